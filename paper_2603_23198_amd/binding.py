"""ctypes binding of libsfl (include/sfl.h). Argument marshalling only.

Every function here has the name of the C entry point it calls and forwards
device pointers (torch tensors' data_ptr()) and the current HIP stream; the operators
around the layer also check the tensors' types, sizes and contiguity. All
arithmetic happens in the HIP kernels of libsfl.so; if the library is missing
or fails to load, importing this module raises (there is no fallback path). The
extension module `_marshal.so` turns tensors into checked pointers for the operators
around the layer, and only those need it.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, c_char_p, c_double, c_int, c_int32, c_int64, c_size_t, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SFL_LIB", os.path.join(_HERE, "libsfl.so"))

if not os.path.exists(LIB_PATH):
    raise ImportError(f"libsfl.so not found at {LIB_PATH}; build it with "
                      "`python -m paper_2603_23198_amd.build` (or __graft_entry__.build())")
_lib = ctypes.CDLL(LIB_PATH)


class _NotBuilt:
    """Stands for the extension module `_marshal` where it cannot be loaded: the layer's entry points
    do without it, those that take checked tensors raise ImportError."""

    def __init__(self, why):
        self._why = why

    def ptr(self, *_):
        raise ImportError(f"the binding's extension module _marshal.so cannot be loaded ({self._why}); build it with "
                          "`python -m paper_2603_23198_amd.build` (or __graft_entry__.build())")

    space = grads = ptr


try:
    from . import _marshal
except ImportError as e:
    _marshal = _NotBuilt(e)

SFL_F32, SFL_BF16 = 0, 1
SFL_OK, SFL_E_ARG, SFL_E_UNSUPPORTED, SFL_E_WORKSPACE, SFL_E_HIP = 0, -1, -2, -3, -4
BUF_NAMES = ["val", "idx", "cnt", "row_nnz", "row_ovf", "ovf_rows", "n_ovf", "ell_val", "ell_idx", "ovf_dense"]

EXPORTED = ["sfl_status_string", "sfl_version", "sfl_twell_buffer_sizes", "sfl_pack_twell",
            "sfl_workspace_size", "sfl_ffn_forward", "sfl_up_projection", "sfl_ffn_backward",
            "sfl_dense_ffn_baseline", "sfl_transpose", "sfl_pack_down_weights", "sfl_track_active_units",
            "sfl_reinit_dead_units", "sfl_ffn_forward_noalloc", "sfl_bandwidth_probe",
            "sfl_down_projection_rowwise", "sfl_forward_workspace_size", "sfl_backward_workspace_size",
            "sfl_norm_forward", "sfl_norm_backward", "sfl_norm_workspace_size", "sfl_route_forward",
            "sfl_route_backward", "sfl_expert_dispatch", "sfl_expert_workspace_size", "sfl_expert_combine",
            "sfl_expert_combine_backward", "sfl_grad_sumsq", "sfl_grad_workspace_size", "sfl_grad_clip",
            "sfl_route_groups_forward", "sfl_route_groups_backward", "sfl_quant_rows", "sfl_quant_columns",
            "sfl_quant_weights", "sfl_quant_product", "sfl_quant_product_weights", "sfl_adamw_step"]


class SflError(RuntimeError):
    def __init__(self, fn, code):
        msg = _lib.sfl_status_string(code).decode()
        super().__init__(f"{fn} failed: {msg} ({code})")
        self.code = code


class Cfg(Structure):
    _fields_ = [("tile_rows", c_int32), ("tile_cols", c_int32), ("tile_slots", c_int32),
                ("ell_width", c_int32), ("ovf_capacity", c_int32), ("layout", c_int32)]


SFL_TWELL_PLANES, SFL_TWELL_PACKED32 = 0, 1


class Twell(Structure):
    _fields_ = [(n, c_void_p) for n in BUF_NAMES]


class Stats(Structure):
    _fields_ = [("total_nnz", c_int64), ("n_ovf_rows", c_int64), ("n_tile_ovf", c_int64),
                ("l1_sum", c_double), ("capacity_exceeded", c_int32), ("reserved", c_int32)]


class FfnArgs(Structure):
    _fields_ = [("dtype", c_int), ("gated", c_int32), ("T", c_int64), ("d", c_int64), ("f", c_int64),
                ("X", c_void_p), ("W_gate", c_void_p), ("W_up", c_void_p), ("W_down", c_void_p),
                ("W_upT", c_void_p), ("W_gateT", c_void_p), ("W_downT", c_void_p), ("W_down_packed", c_void_p),
                ("W_up_packed", c_void_p),
                ("bias_f", c_void_p), ("shift_t", c_void_p),
                ("cfg", Cfg),
                ("Y", c_void_p), ("twell", Twell), ("stats", c_void_p), ("workspace", c_void_p),
                ("workspace_bytes", c_size_t), ("events", c_void_p), ("n_events", c_int32)]


class BwdArgs(Structure):
    _fields_ = [("dtype", c_int), ("gated", c_int32), ("T", c_int64), ("d", c_int64), ("f", c_int64),
                ("X", c_void_p), ("W_gate", c_void_p), ("W_up", c_void_p), ("W_down", c_void_p),
                ("W_upT", c_void_p), ("W_gateT", c_void_p),
                ("W_down_packed", c_void_p), ("W_up_packed", c_void_p), ("W_gate_packed", c_void_p),
                ("bias_f", c_void_p), ("shift_t", c_void_p),
                ("dY", c_void_p), ("cfg", Cfg), ("saved", Twell), ("lambda_l1", c_double),
                ("dX", c_void_p), ("dW_gate", c_void_p), ("dW_up", c_void_p), ("dW_down", c_void_p),
                ("workspace", c_void_p), ("workspace_bytes", c_size_t), ("events", c_void_p), ("n_events", c_int32)]


SFL_NORM_PRE, SFL_NORM_POST = 1, 2


class NormArgs(Structure):
    _fields_ = [("dtype", c_int), ("norms", c_int32), ("T", c_int64), ("d", c_int64), ("eps", ctypes.c_float),
                ("res_scale", ctypes.c_float), ("X", c_void_p), ("Y", c_void_p), ("w_pre", c_void_p),
                ("w_post", c_void_p), ("gate_c", c_void_p), ("gate_t", c_void_p), ("X_out", c_void_p), ("N", c_void_p)]


class NormBwdArgs(Structure):
    _fields_ = [("dtype", c_int), ("norms", c_int32), ("T", c_int64), ("d", c_int64), ("eps", ctypes.c_float),
                ("res_scale", ctypes.c_float), ("X_out", c_void_p), ("Y", c_void_p), ("w_pre", c_void_p),
                ("w_post", c_void_p), ("gate_c", c_void_p), ("gate_t", c_void_p), ("dX_out", c_void_p),
                ("dN", c_void_p), ("dX", c_void_p), ("dY", c_void_p), ("dw_pre", c_void_p), ("dw_post", c_void_p),
                ("dgate_c", c_void_p), ("dgate_t", c_void_p), ("workspace", c_void_p), ("workspace_bytes", c_size_t)]


class Grad(Structure):
    _fields_ = [("src", c_void_p), ("dst", c_void_p), ("n", c_int64), ("dtype", c_int32), ("reserved", c_int32)]


SFL_BF16_FAST = 0x101  # of the products' results
SFL_SCORE_SIGMOID, SFL_SCORE_SOFTMAX = 0, 1
SFL_MOMENTS_F32, SFL_MOMENTS_8BIT = 0, 1


class RouteGroupsArgs(Structure):
    _fields_ = [("dtype", c_int), ("score", c_int32), ("T", c_int64), ("E", c_int32), ("k", c_int32),
                ("groups", c_int32), ("group_k", c_int32), ("group_top", c_int32), ("normalise", c_int32),
                ("scale", ctypes.c_float), ("logits", c_void_p), ("bias", c_void_p), ("expert", c_void_p),
                ("weight", c_void_p)]


class RouteGroupsBwdArgs(Structure):
    _fields_ = [("dtype", c_int), ("score", c_int32), ("T", c_int64), ("E", c_int32), ("k", c_int32),
                ("normalise", c_int32), ("scale", ctypes.c_float), ("logits", c_void_p), ("expert", c_void_p),
                ("dweight", c_void_p), ("dlogits", c_void_p)]


class QuantArgs(Structure):
    _fields_ = [("dtype", c_int), ("E", c_int32), ("T", c_int64), ("d", c_int64), ("columns", c_int64),
                ("X", c_void_p), ("where", c_void_p), ("offsets", c_void_p), ("Q", c_void_p), ("S", c_void_p),
                ("Qt", c_void_p), ("St", c_void_p)]


class Adamw(Structure):
    _fields_ = [("param", c_void_p), ("grad", c_void_p), ("half", c_void_p), ("m", c_void_p), ("v", c_void_p),
                ("m_scale", c_void_p), ("v_scale", c_void_p), ("n", c_int64), ("weight_decay", ctypes.c_float),
                ("param_dtype", c_int32), ("grad_dtype", c_int32), ("moments", c_int32)]


class AdamwCfg(Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double),
                ("max_norm", c_double), ("seed", ctypes.c_uint32), ("reserved", ctypes.c_uint32),
                ("step", c_void_p), ("lr_scale", c_void_p), ("sumsq", c_void_p), ("norm", c_void_p)]


_lib.sfl_status_string.restype = c_char_p
_lib.sfl_status_string.argtypes = [c_int]
_lib.sfl_version.restype = c_char_p
_lib.sfl_twell_buffer_sizes.argtypes = [c_int64, c_int64, c_int, POINTER(Cfg), POINTER(c_size_t)]
_lib.sfl_pack_twell.argtypes = [c_void_p, c_int64, c_int64, c_int, POINTER(Cfg), POINTER(Twell), c_void_p, c_void_p]
_lib.sfl_workspace_size.argtypes = [c_void_p, c_int, POINTER(c_size_t)]
_lib.sfl_forward_workspace_size.argtypes = [POINTER(FfnArgs), c_int32, POINTER(c_size_t)]
_lib.sfl_backward_workspace_size.argtypes = [POINTER(BwdArgs), POINTER(c_size_t)]
_lib.sfl_ffn_forward.argtypes = [POINTER(FfnArgs), c_void_p]
_lib.sfl_ffn_forward_noalloc.argtypes = [POINTER(FfnArgs), c_void_p]
_lib.sfl_down_projection_rowwise.argtypes = [POINTER(FfnArgs), c_int32, c_void_p]
_lib.sfl_bandwidth_probe.argtypes = [c_void_p, c_void_p, c_size_t, c_int32, c_void_p, POINTER(c_size_t), c_void_p]
_lib.sfl_up_projection.argtypes = [POINTER(FfnArgs), c_void_p, c_void_p]
_lib.sfl_ffn_backward.argtypes = [POINTER(BwdArgs), c_void_p]
_lib.sfl_dense_ffn_baseline.argtypes = [POINTER(FfnArgs), c_void_p]
_lib.sfl_transpose.argtypes = [c_void_p, c_void_p, c_int64, c_int64, c_int32, c_void_p]
_lib.sfl_pack_down_weights.argtypes = [c_void_p, c_void_p, c_int64, c_int64, c_void_p]
_lib.sfl_track_active_units.argtypes = [POINTER(Twell), c_int64, c_int64, c_int, POINTER(Cfg), c_int64, c_void_p,
                                        c_void_p]
_lib.sfl_reinit_dead_units.argtypes = [c_void_p, c_int, c_int64, c_int64, c_int32, c_void_p, c_int64, ctypes.c_float,
                                       ctypes.c_float, c_void_p, c_void_p]
_lib.sfl_norm_forward.argtypes = [POINTER(NormArgs), c_void_p]
_lib.sfl_norm_backward.argtypes = [POINTER(NormBwdArgs), c_void_p]
_lib.sfl_norm_workspace_size.argtypes = [c_int64, c_int64, c_int, POINTER(c_size_t)]
_lib.sfl_route_forward.argtypes = [c_void_p, c_int, c_int64, c_int32, c_int32, c_int32, ctypes.c_float, c_void_p,
                                   c_void_p, c_void_p]
_lib.sfl_route_backward.argtypes = [c_void_p, c_int, c_int64, c_int32, c_int32, c_int32, ctypes.c_float, c_void_p,
                                    c_void_p, c_void_p, c_void_p]
_lib.sfl_expert_dispatch.argtypes = [c_void_p, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int, c_int64,
                                     c_int64, c_void_p, c_void_p, c_size_t, c_void_p]
_lib.sfl_expert_workspace_size.argtypes = [c_int64, c_int32, c_int32, POINTER(c_size_t)]
_lib.sfl_expert_combine.argtypes = [c_void_p, c_int, c_int64, c_int64, c_int32, c_void_p, c_int64, c_void_p, c_void_p,
                                    c_void_p]
_lib.sfl_expert_combine_backward.argtypes = [c_void_p, c_void_p, c_int, c_int64, c_int64, c_int32, c_void_p, c_int64,
                                             c_void_p, c_void_p, c_void_p, c_void_p]
_lib.sfl_grad_sumsq.argtypes = [POINTER(Grad), c_int32, c_void_p, c_void_p, c_size_t, c_void_p]
_lib.sfl_grad_workspace_size.argtypes = [POINTER(Grad), c_int32, POINTER(c_size_t)]
_lib.sfl_grad_clip.argtypes = [POINTER(Grad), c_int32, c_void_p, ctypes.c_float, c_void_p, c_void_p]
_lib.sfl_route_groups_forward.argtypes = [POINTER(RouteGroupsArgs), c_void_p]
_lib.sfl_route_groups_backward.argtypes = [POINTER(RouteGroupsBwdArgs), c_void_p]
_lib.sfl_quant_rows.argtypes = [POINTER(QuantArgs), c_void_p]
_lib.sfl_quant_columns.argtypes = [c_int64, c_int32, POINTER(c_int64)]
_lib.sfl_quant_weights.argtypes = [c_void_p, c_int, c_int64, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p]
_lib.sfl_quant_product.argtypes = [c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_int32, c_int64, c_void_p,
                                   c_int, c_void_p, c_void_p]
_lib.sfl_quant_product_weights.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_int64, c_int64,
                                           c_void_p, c_int32, c_int, c_void_p, c_void_p]
_lib.sfl_adamw_step.argtypes = [POINTER(Adamw), c_int32, POINTER(AdamwCfg), c_void_p]
for _n in EXPORTED[2:]:
    getattr(_lib, _n).restype = c_int


def _check(fn, code):
    if code != SFL_OK:
        raise SflError(fn, code)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# torch's handle of the current stream without the Stream object around it (2.9 against 0.3 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_CODES = {torch.float32: SFL_F32, torch.bfloat16: SFL_BF16, "f32": SFL_F32, "bf16": SFL_BF16}


def dtype_code(dtype):
    code = _CODES.get(dtype)
    if code is not None:
        return code
    if dtype in ("bf16", torch.bfloat16, SFL_BF16):
        return SFL_BF16
    if dtype in ("f32", torch.float32, SFL_F32):
        return SFL_F32
    raise ValueError(dtype)


def make_cfg(tile_cols=256, tile_slots=32, ell_width=128, ovf_capacity=0, tile_rows=0, layout=0, **_):
    return Cfg(tile_rows, tile_cols, tile_slots, ell_width, ovf_capacity, layout)


def sfl_version():
    return _lib.sfl_version().decode()


def sfl_status_string(code):
    return _lib.sfl_status_string(code).decode()


def sfl_twell_buffer_sizes(T, f, dtype, cfg):
    out = (c_size_t * len(BUF_NAMES))()
    _check("sfl_twell_buffer_sizes", _lib.sfl_twell_buffer_sizes(T, f, dtype_code(dtype), ctypes.byref(cfg), out))
    return list(out)


def alloc_twell(T, f, dtype, cfg, device="cuda", with_ell=True, with_dense=True):
    """Caller-side allocation (torch) of the packed-activation buffers, as dict of tensors."""
    sizes = sfl_twell_buffer_sizes(T, f, dtype, cfg)
    act = torch.bfloat16 if dtype_code(dtype) == SFL_BF16 else torch.float32
    es = 2 if act == torch.bfloat16 else 4
    packed = cfg.layout == SFL_TWELL_PACKED32
    kinds = {"val": torch.int32 if packed else act, "idx": torch.int16, "cnt": torch.int32, "row_nnz": torch.int32,
             "row_ovf": torch.uint8, "ovf_rows": torch.int32, "n_ovf": torch.int32,
             "ell_val": act, "ell_idx": torch.int16, "ovf_dense": act}
    item = {"val": 4 if packed else es, "idx": 2, "cnt": 4, "row_nnz": 4, "row_ovf": 1, "ovf_rows": 4, "n_ovf": 4,
            "ell_val": es, "ell_idx": 2, "ovf_dense": es}
    bufs = {}
    for name, nbytes in zip(BUF_NAMES, sizes):
        if (name in ("ell_val", "ell_idx") and not with_ell) or (name == "ovf_dense" and not with_dense) or \
                (packed and name in ("idx", "cnt")):
            bufs[name] = None
            continue
        n = max(1, nbytes // item[name])
        bufs[name] = torch.empty(n, dtype=kinds[name], device=device)
    return bufs


def _twell_struct(bufs):
    return Twell(*[_ptr(bufs.get(n)) for n in BUF_NAMES])


def sfl_pack_twell(Z, dtype, cfg, bufs, stats=None, stream=None):
    T, f = Z.shape
    tw = _twell_struct(bufs)
    _check("sfl_pack_twell", _lib.sfl_pack_twell(_ptr(Z), T, f, dtype_code(dtype), ctypes.byref(cfg),
                                                 ctypes.byref(tw), _ptr(stats), _stream(stream)))


def alloc_stats(device="cuda"):
    return torch.zeros(ctypes.sizeof(Stats), dtype=torch.uint8, device=device)


def read_stats(stats_tensor):
    raw = bytes(stats_tensor.cpu().numpy().tobytes())
    s = Stats.from_buffer_copy(raw)
    return {n: getattr(s, n) for n, _ in Stats._fields_ if n != "reserved"}


def ffn_args(X, W_up, W_down, cfg, *, Y=None, bufs=None, W_gate=None, W_upT=None, W_gateT=None, W_downT=None,
             W_down_packed=None, W_up_packed=None, bias_f=None, shift_t=None, stats=None, workspace=None,
             events=None):
    T, d = X.shape
    f = W_down.shape[0]
    a = FfnArgs()
    a.dtype = dtype_code(X.dtype)
    a.gated = 1 if W_gate is not None else 0
    a.T, a.d, a.f = T, d, f
    a.X, a.W_gate, a.W_up, a.W_down, a.W_upT = _ptr(X), _ptr(W_gate), _ptr(W_up), _ptr(W_down), _ptr(W_upT)
    a.W_gateT, a.W_downT = _ptr(W_gateT), _ptr(W_downT)
    a.W_down_packed, a.W_up_packed = _ptr(W_down_packed), _ptr(W_up_packed)
    a.bias_f, a.shift_t = _ptr(bias_f), _ptr(shift_t)
    a.cfg = cfg
    a.Y = _ptr(Y)
    if bufs is not None:
        a.twell = _twell_struct(bufs)
    a.stats = _ptr(stats)
    if workspace is not None:
        a.workspace = _ptr(workspace)
        a.workspace_bytes = workspace.numel() * workspace.element_size()
    if events is not None:
        a._events_keepalive = events
        a.events = ctypes.cast(events, c_void_p).value
        a.n_events = len(events)
    return a


def sfl_workspace_size(args, kind=0):
    out = c_size_t(0)
    _check("sfl_workspace_size", _lib.sfl_workspace_size(ctypes.byref(args), kind, ctypes.byref(out)))
    return out.value


def sfl_forward_workspace_size(args, dense=False):
    out = c_size_t(0)
    _check("sfl_forward_workspace_size", _lib.sfl_forward_workspace_size(ctypes.byref(args), 1 if dense else 0,
                                                                          ctypes.byref(out)))
    return out.value


def sfl_backward_workspace_size(args):
    out = c_size_t(0)
    _check("sfl_backward_workspace_size", _lib.sfl_backward_workspace_size(ctypes.byref(args), ctypes.byref(out)))
    return out.value


def sfl_ffn_forward(args, stream=None):
    _check("sfl_ffn_forward", _lib.sfl_ffn_forward(ctypes.byref(args), _stream(stream)))


def sfl_ffn_forward_noalloc(args, stream=None):
    _check("sfl_ffn_forward_noalloc", _lib.sfl_ffn_forward_noalloc(ctypes.byref(args), _stream(stream)))


def sfl_up_projection(args, Z, stream=None):
    _check("sfl_up_projection", _lib.sfl_up_projection(ctypes.byref(args), _ptr(Z), _stream(stream)))


def sfl_dense_ffn_baseline(args, stream=None):
    _check("sfl_dense_ffn_baseline", _lib.sfl_dense_ffn_baseline(ctypes.byref(args), _stream(stream)))


def bwd_args(X, W_up, W_down, dY, cfg, saved_bufs, lambda_l1, dX, dW_up, dW_down, *, W_upT=None, W_down_packed=None,
             W_up_packed=None, W_gate=None, W_gateT=None, W_gate_packed=None, dW_gate=None, bias_f=None,
             shift_t=None, workspace=None, events=None):
    T, d = X.shape
    f = W_down.shape[0]
    a = BwdArgs()
    a.dtype = dtype_code(X.dtype)
    a.T, a.d, a.f = T, d, f
    a.X, a.W_up, a.W_down, a.W_upT, a.dY = _ptr(X), _ptr(W_up), _ptr(W_down), _ptr(W_upT), _ptr(dY)
    a.W_down_packed, a.W_up_packed = _ptr(W_down_packed), _ptr(W_up_packed)
    a.gated = 1 if W_gate is not None else 0
    a.W_gate, a.W_gateT, a.W_gate_packed = _ptr(W_gate), _ptr(W_gateT), _ptr(W_gate_packed)
    a.bias_f, a.shift_t, a.dW_gate = _ptr(bias_f), _ptr(shift_t), _ptr(dW_gate)
    a.cfg = cfg
    a.saved = _twell_struct(saved_bufs)
    a.lambda_l1 = float(lambda_l1)
    a.dX, a.dW_up, a.dW_down = _ptr(dX), _ptr(dW_up), _ptr(dW_down)
    if workspace is not None:
        a.workspace = _ptr(workspace)
        a.workspace_bytes = workspace.numel() * workspace.element_size()
    if events is not None:
        a._events_keepalive = events
        a.events = ctypes.cast(events, c_void_p).value
        a.n_events = len(events)
    return a


def sfl_ffn_backward(args, stream=None):
    _check("sfl_ffn_backward", _lib.sfl_ffn_backward(ctypes.byref(args), _stream(stream)))


def sfl_pack_down_weights(W_down, out, stream=None):
    f, d = W_down.shape
    _check("sfl_pack_down_weights", _lib.sfl_pack_down_weights(_ptr(W_down), _ptr(out), f, d, _stream(stream)))


def sfl_track_active_units(bufs, T, f, dtype, cfg, step, last_active, stream=None):
    tw = _twell_struct(bufs)
    _check("sfl_track_active_units", _lib.sfl_track_active_units(ctypes.byref(tw), T, f, dtype_code(dtype),
                                                                 ctypes.byref(cfg), int(step), _ptr(last_active),
                                                                 _stream(stream)))


def sfl_reinit_dead_units(W, last_active, step, lam, sigma, noise, units_on_rows=False, stream=None):
    rows, cols = W.shape
    _check("sfl_reinit_dead_units", _lib.sfl_reinit_dead_units(_ptr(W), dtype_code(W.dtype), rows, cols,
                                                               1 if units_on_rows else 0, _ptr(last_active),
                                                               int(step), float(lam), float(sigma), _ptr(noise),
                                                               _stream(stream)))


def sfl_down_projection_rowwise(args, split, stream=None):
    _check("sfl_down_projection_rowwise", _lib.sfl_down_projection_rowwise(ctypes.byref(args), split, _stream(stream)))


def sfl_bandwidth_probe(src, dst=None, reps=1, sink=None, nbytes=None, stream=None):
    """Copy (dst given) or L2/HBM read probe (dst None); returns the bytes moved."""
    moved = c_size_t(0)
    n = src.numel() * src.element_size() if nbytes is None else nbytes
    _check("sfl_bandwidth_probe", _lib.sfl_bandwidth_probe(_ptr(src), _ptr(dst), n, reps, _ptr(sink),
                                                           ctypes.byref(moved), _stream(stream)))
    return moved.value


def sfl_transpose(inp, out, stream=None):
    rows, cols = inp.shape
    _check("sfl_transpose", _lib.sfl_transpose(_ptr(inp), _ptr(out), rows, cols, inp.element_size(),
                                               _stream(stream)))


# ---- around the layer: norms, router, experts, gradient clipping ----
# These take the tensors themselves, so shapes, types and contiguity are checked here.
# Device pointer of a contiguous device tensor of n elements of a type (SFL_F32, SFL_BF16 or one of
# those below), in rows of so many where a fourth argument says so; None for None; ValueError for
# any other.
_buf = _marshal.ptr
_space = _marshal.space  # (device pointer, bytes) of a contiguous device tensor, or (None, 0) for None
_F32, _BF16, _I32, _F64, _F8, _U8, _I64 = SFL_F32, SFL_BF16, 2, 3, 4, 5, 6


def sfl_norm_forward(X, Y=None, *, X_out=None, N=None, norms=SFL_NORM_PRE | SFL_NORM_POST, w_pre=None, w_post=None,
                     gate_c=None, gate_t=None, res_scale=1.0, eps=1e-6, stream=None):
    T, d = X.shape
    dt, n = dtype_code(X.dtype), T * d
    a = NormArgs(dt, norms, T, d, eps, res_scale, _buf(X, dt, n, d), _buf(Y, dt, n, d), _buf(w_pre, _F32, d),
                 _buf(w_post, _F32, d), _buf(gate_c, _F32, d), _buf(gate_t, _F32, T), _buf(X_out, dt, n, d),
                 _buf(N, dt, n, d))
    _check("sfl_norm_forward", _lib.sfl_norm_forward(a, _stream(stream)))


def sfl_norm_workspace_size(T, d, dtype):
    out = c_size_t(0)
    _check("sfl_norm_workspace_size", _lib.sfl_norm_workspace_size(T, d, dtype_code(dtype), out))
    return out.value


def sfl_norm_backward(X_out, Y, dX_out, dN=None, *, dX=None, dY=None, dw_pre=None, dw_post=None, dgate_c=None,
                      dgate_t=None, norms=SFL_NORM_PRE | SFL_NORM_POST, w_pre=None, w_post=None, gate_c=None,
                      gate_t=None, res_scale=1.0, eps=1e-6, workspace=None, stream=None):
    like = X_out if X_out is not None else dX_out
    if like is None:
        like = next((t for t in (Y, dN, dX) if t is not None), None)
    if like is None:
        raise ValueError("sfl_norm_backward: no tensor of rows gives the sizes")
    T, d = like.shape
    dt, n = dtype_code(like.dtype), T * d
    a = NormBwdArgs(dt, norms, T, d, eps, res_scale, _buf(X_out, dt, n, d), _buf(Y, dt, n, d),
                    _buf(w_pre, _F32, d), _buf(w_post, _F32, d), _buf(gate_c, _F32, d), _buf(gate_t, _F32, T),
                    _buf(dX_out, dt, n, d), _buf(dN, dt, n, d), _buf(dX, dt, n, d), _buf(dY, dt, n, d),
                    _buf(dw_pre, _F32, d), _buf(dw_post, _F32, d), _buf(dgate_c, _F32, d), _buf(dgate_t, _F32, T),
                    *_space(workspace))
    _check("sfl_norm_backward", _lib.sfl_norm_backward(a, _stream(stream)))


def sfl_route_forward(logits, expert, weight, *, normalise=True, scale=1.0, stream=None):
    (T, E), k, dt = logits.shape, expert.shape[1], dtype_code(logits.dtype)
    _check("sfl_route_forward",
           _lib.sfl_route_forward(_buf(logits, dt, T * E, E), dt, T, E, k, 1 if normalise else 0, scale,
                                  _buf(expert, _I32, T * k, k), _buf(weight, _F32, T * k, k), _stream(stream)))


def sfl_route_backward(logits, expert, dweight, dlogits, *, normalise=True, scale=1.0, stream=None):
    (T, E), k, dt = logits.shape, expert.shape[1], dtype_code(logits.dtype)
    _check("sfl_route_backward",
           _lib.sfl_route_backward(_buf(logits, dt, T * E, E), dt, T, E, k, 1 if normalise else 0, scale,
                                   _buf(expert, _I32, T * k, k), _buf(dweight, _F32, T * k, k),
                                   _buf(dlogits, dt, T * E, E), _stream(stream)))


def sfl_expert_workspace_size(T, k, E):
    out = c_size_t(0)
    _check("sfl_expert_workspace_size", _lib.sfl_expert_workspace_size(T, k, E, out))
    return out.value


def sfl_expert_dispatch(expert, E, pos, offsets, *, X=None, Xs=None, workspace=None, stream=None):
    T, k = expert.shape
    n, dt, d, rows, px, ps = T * k, SFL_F32, 1, 0, None, None
    like = X if X is not None else Xs
    if like is not None:  # one of the two alone is for the entry point to judge
        d, rows, dt = like.shape[1], 0 if Xs is None else Xs.shape[0], dtype_code(like.dtype)
        px, ps = _buf(X, dt, T * d, d), _buf(Xs, dt, rows * d, d)
    ws, ws_bytes = _space(workspace)
    _check("sfl_expert_dispatch",
           _lib.sfl_expert_dispatch(_buf(expert, _I32, n, k), T, k, E, _buf(pos, _I32, n, k),
                                    _buf(offsets, _I32, E + 1), px, dt, d, rows, ps, ws, ws_bytes, _stream(stream)))


def sfl_expert_combine(Ys, pos, Y, *, weight=None, stream=None):
    (T, k), (rows, d), dt = pos.shape, Ys.shape, dtype_code(Ys.dtype)
    _check("sfl_expert_combine",
           _lib.sfl_expert_combine(_buf(Ys, dt, rows * d, d), dt, T, d, k, _buf(pos, _I32, T * k, k), rows,
                                   _buf(weight, _F32, T * k, k), _buf(Y, dt, T * d, d), _stream(stream)))


def sfl_expert_combine_backward(dY, Ys, pos, weight, *, dYs=None, dweight=None, stream=None):
    (T, k), d, dt = pos.shape, dY.shape[1], dtype_code(dY.dtype)
    like = dYs if Ys is None else Ys
    if like is None and dweight is not None:
        raise ValueError("sfl_expert_combine_backward: dweight needs Ys")
    rows = 0 if like is None else like.shape[0]
    _check("sfl_expert_combine_backward",
           _lib.sfl_expert_combine_backward(_buf(dY, dt, T * d, d), _buf(Ys, dt, rows * d, d), dt, T, d, k,
                                            _buf(pos, _I32, T * k, k), rows, _buf(weight, _F32, T * k, k),
                                            _buf(dYs, dt, rows * d, d), _buf(dweight, _F32, T * k, k), _stream(stream)))


def grad_list(grads, out=None):
    """The list of gradients that the sfl_grad_* calls take; it keeps the tensors alive. out: where
    the clipped gradients go, in place if None."""
    rows = _marshal.grads(grads, out)
    a = (Grad * len(grads)).from_buffer(rows) if rows else (Grad * 0)()
    a._keepalive = (tuple(grads), None if out is None else tuple(out))  # the caller's lists may change
    return a


def sfl_grad_workspace_size(grads):
    out = c_size_t(0)
    _check("sfl_grad_workspace_size", _lib.sfl_grad_workspace_size(grads, len(grads), out))
    return out.value


def sfl_grad_sumsq(grads, sumsq, *, workspace=None, stream=None):
    _check("sfl_grad_sumsq", _lib.sfl_grad_sumsq(grads, len(grads), _buf(sumsq, _F64, 1), *_space(workspace),
                                                 _stream(stream)))


def sfl_grad_clip(grads, sumsq, max_norm, norm=None, *, stream=None):
    _check("sfl_grad_clip", _lib.sfl_grad_clip(grads, len(grads), _buf(sumsq, _F64, 1), max_norm,
                                               _buf(norm, _F32, 1), _stream(stream)))


# ---- many routed experts in 8 bits: router with groups, quantisation, products, AdamW ----
_SCORES = {"sigmoid": SFL_SCORE_SIGMOID, "softmax": SFL_SCORE_SOFTMAX}


def _up(n, m):
    return -(-n // m) * m


def _score(score):
    code = _SCORES.get(score)
    if code is None:
        raise ValueError(f"unknown score {score!r}: 'sigmoid' or 'softmax'")
    return code


def sfl_route_groups_forward(logits, expert, weight, *, bias=None, score="sigmoid", groups=1, group_k=1, group_top=1,
                             normalise=True, scale=1.0, stream=None):
    (T, E), k, dt = logits.shape, expert.shape[1], dtype_code(logits.dtype)
    a = RouteGroupsArgs(dt, _score(score), T, E, k, groups, group_k, group_top, 1 if normalise else 0, scale,
                        _buf(logits, dt, T * E, E), _buf(bias, _F32, E), _buf(expert, _I32, T * k, k),
                        _buf(weight, _F32, T * k, k))
    _check("sfl_route_groups_forward", _lib.sfl_route_groups_forward(a, _stream(stream)))


def sfl_route_groups_backward(logits, expert, dweight, dlogits, *, score="sigmoid", normalise=True, scale=1.0,
                              stream=None):
    (T, E), k, dt = logits.shape, expert.shape[1], dtype_code(logits.dtype)
    a = RouteGroupsBwdArgs(dt, _score(score), T, E, k, 1 if normalise else 0, scale, _buf(logits, dt, T * E, E),
                           _buf(expert, _I32, T * k, k), _buf(dweight, _F32, T * k, k), _buf(dlogits, dt, T * E, E))
    _check("sfl_route_groups_backward", _lib.sfl_route_groups_backward(a, _stream(stream)))


def sfl_quant_columns(T, E=1):
    out = c_int64(0)
    _check("sfl_quant_columns", _lib.sfl_quant_columns(T, E, out))
    return out.value


def _codes(Q, S, rows, width, scale_rows):
    """Pointers of codes of so many rows and bytes a row, and of their scales."""
    per = _up(width // 128, 4)
    return _buf(Q, _F8, rows * width, width), _buf(S, _U8, scale_rows * per, per)


def sfl_quant_rows(X, Q=None, S=None, *, Qt=None, St=None, where=None, offsets=None, stream=None):
    (T, d), dt = X.shape, dtype_code(X.dtype)
    E = 1 if offsets is None else offsets.numel() - 1
    columns = 0 if Qt is None else Qt.shape[1]
    a = QuantArgs(dt, E, T, d, columns, _buf(X, dt, T * d, d), _buf(where, dt, T * d, d), _buf(offsets, _I32, E + 1),
                  *_codes(Q, S, T, _up(d, 128), T), *_codes(Qt, St, d, columns, d))
    _check("sfl_quant_rows", _lib.sfl_quant_rows(a, _stream(stream)))


def sfl_quant_weights(W, Q=None, S=None, *, Qt=None, St=None, stream=None):
    R, C = W.shape[-2:]
    E, dt = W.shape[0] if W.dim() == 3 else 1, dtype_code(W.dtype)
    r, c = _up(R, 128), _up(C, 128)
    _check("sfl_quant_weights",
           _lib.sfl_quant_weights(_buf(W, dt, E * R * C, C), dt, E, R, C, *_codes(Q, S, E * R, c, E * (r // 128)),
                                  *_codes(Qt, St, E * C, r, E * (c // 128)), _stream(stream)))


def _result(dt, fast):
    """The type of a product's result; fast: bf16 from the 8-bit matrix instruction, which drops what lies 13 bits
    below the largest of eight neighbouring products."""
    if fast and dt != SFL_BF16:
        raise ValueError("fast products have bf16 results")
    return SFL_BF16_FAST if fast else dt


def sfl_quant_product(Q, S, W, Ws, Y, *, offsets=None, fast=False, stream=None):
    (rows, K), N, dt = Q.shape, W.shape[-2], dtype_code(Y.dtype)
    result = _result(dt, fast)
    E = W.shape[0] if W.dim() == 3 else 1
    if offsets is not None and offsets.numel() != E + 1:
        raise ValueError(f"offsets of {E} experts are {E + 1}, got {offsets.numel()}")
    q, s = _codes(Q, S, rows, K, rows)
    w, ws = _codes(W, Ws, E * N, K, E * (_up(N, 128) // 128))
    _check("sfl_quant_product",
           _lib.sfl_quant_product(q, s, rows, K, w, ws, E, N, _buf(offsets, _I32, E + 1), result,
                                  _buf(Y, dt, rows * N, N), _stream(stream)))


def sfl_quant_product_weights(Yt, Ys, Xt, Xs, dW, *, rows=None, offsets=None, fast=False, stream=None):
    """rows: the tokens of the one run without offsets (with them, they say how many there are)."""
    (N, columns), K, dt = Yt.shape, Xt.shape[0], dtype_code(dW.dtype)
    result = _result(dt, fast)
    E = 1 if offsets is None else offsets.numel() - 1
    if rows is None:
        if offsets is None:
            raise ValueError("sfl_quant_product_weights: rows or offsets are needed")
        rows = columns
    yt, ys = _codes(Yt, Ys, N, columns, N)
    xt, xs = _codes(Xt, Xs, K, columns, K)
    _check("sfl_quant_product_weights",
           _lib.sfl_quant_product_weights(yt, ys, N, xt, xs, K, rows, columns, _buf(offsets, _I32, E + 1), E,
                                          result, _buf(dW, dt, E * N * K, K), _stream(stream)))


def adamw_list(params, grads, m, v, *, halves=None, m_scales=None, v_scales=None, weight_decay=0.0):
    """The list of tensors that sfl_adamw_step takes; it keeps them alive. Moments are fp32, or
    float8_e4m3fn with uint8 scales of one for each 128 elements. weight_decay: one for all, or one
    for each tensor; halves: bf16 copies, None for no copy (of all, or of single tensors)."""
    n = len(params)
    none = [None] * n
    halves, m_scales, v_scales = halves or none, m_scales or none, v_scales or none
    decay = [weight_decay] * n if isinstance(weight_decay, (int, float)) else list(weight_decay)
    lists = (params, grads, m, v, halves, m_scales, v_scales, decay)
    if any(len(x) != n for x in lists):
        raise ValueError("the lists of sfl_adamw_step need one entry for each parameter")
    a = (Adamw * n)()
    for i, (p, g, mi, vi, half, ms, vs, wd) in enumerate(zip(*lists)):
        e, pd, gd = p.numel(), dtype_code(p.dtype), dtype_code(g.dtype)
        small = mi.dtype == torch.float8_e4m3fn
        kind, blocks = (_F8, -(-e // 128)) if small else (_F32, 0)
        if not small and (ms is not None or vs is not None):
            raise ValueError("fp32 moments have no scales")
        a[i] = Adamw(_buf(p, pd, e), _buf(g, gd, e), _buf(half, _BF16, e), _buf(mi, kind, e), _buf(vi, kind, e),
                     _buf(ms, _U8, blocks), _buf(vs, _U8, blocks), e, wd, pd, gd,
                     SFL_MOMENTS_8BIT if small else SFL_MOMENTS_F32)
    a._keepalive = [tuple(x) for x in lists]  # the caller's lists may change
    return a


def sfl_adamw_step(tensors, step, *, lr, beta1=0.9, beta2=0.999, eps=1e-8, sumsq=None, max_norm=None, norm=None,
                   lr_scale=None, seed=0, stream=None):
    """max_norm: needed with sumsq; math.inf clips nothing (and leaves a step out where the norm is not finite)."""
    if sumsq is not None and max_norm is None:
        raise ValueError("sfl_adamw_step: sumsq needs max_norm (math.inf for no clipping)")
    cfg = AdamwCfg(lr, beta1, beta2, eps, max_norm or 0.0, seed & 0xffffffff, 0, _buf(step, _I64, 1),
                   _buf(lr_scale, _F32, 1), _buf(sumsq, _F64, 1), _buf(norm, _F32, 1))
    _check("sfl_adamw_step", _lib.sfl_adamw_step(tensors, len(tensors), cfg, _stream(stream)))


# ---- HIP events through the runtime library torch already loaded (for stage timing) ----
_hip = None


def _hiprt():
    global _hip
    if _hip is None:
        for name in ("libamdhip64.so.7", "libamdhip64.so"):
            try:
                _hip = ctypes.CDLL(name)
                break
            except OSError:
                continue
        if _hip is None:
            raise OSError("libamdhip64 not found")
        _hip.hipEventCreate.argtypes = [POINTER(c_void_p)]
        _hip.hipEventElapsedTime.argtypes = [POINTER(ctypes.c_float), c_void_p, c_void_p]
        _hip.hipEventSynchronize.argtypes = [c_void_p]
        _hip.hipEventDestroy.argtypes = [c_void_p]
    return _hip


def create_events(n):
    """Array of n hipEvent_t handles (ctypes array of c_void_p) for the `events` argument."""
    hip = _hiprt()
    arr = (c_void_p * n)()
    for i in range(n):
        e = c_void_p()
        if hip.hipEventCreate(ctypes.byref(e)) != 0:
            raise RuntimeError("hipEventCreate failed")
        arr[i] = e
    return arr


def event_ms(events, i, j):
    hip = _hiprt()
    hip.hipEventSynchronize(events[j])
    ms = ctypes.c_float()
    if hip.hipEventElapsedTime(ctypes.byref(ms), events[i], events[j]) != 0:
        raise RuntimeError("hipEventElapsedTime failed")
    return ms.value
