"""What the binding of the operators around the layer does before a launch, as far as that needs no
GPU."""
import ctypes
import gc
import types
import weakref

import pytest
import torch

from paper_2603_23198_amd import binding as b


@pytest.mark.parametrize("kind", [list, tuple])
def test_a_list_of_gradients_keeps_its_tensors(monkeypatch, kind):
    """Also when the caller's own lists change: the calls follow the pointers that were taken."""
    rows = lambda grads, out: bytearray(len(grads) * ctypes.sizeof(b.Grad))  # noqa: E731
    monkeypatch.setattr(b, "_marshal", types.SimpleNamespace(grads=rows))
    grads, out = (kind(torch.zeros(n) for n in (3, 5)) for _ in range(2))
    held = [weakref.ref(t) for t in (*grads, *out)]
    handle = b.grad_list(grads, out)
    if kind is list:
        grads.clear()
        out[0] = out[1] = None
    del grads, out
    gc.collect()
    assert all(r() is not None for r in held)
    del handle
    gc.collect()
    assert all(r() is None for r in held)


def test_a_workspace_that_the_kernels_cannot_use_is_refused():
    with pytest.raises(ValueError, match="on the CPU"):
        b._space(torch.empty(64, dtype=torch.uint8))
    with pytest.raises(ValueError, match="not contiguous"):
        b._space(torch.empty((8, 8), dtype=torch.uint8).t()[1:])
    with pytest.raises(TypeError):
        b._space(0x1000)
    assert b._space(None) == (None, 0)


class Recorded:
    """Stands for the library and for tensors' pointers: device tensors need no device then, and the
    C entry points' own checks still run."""

    def __init__(self, monkeypatch):
        monkeypatch.setattr(b, "_buf", lambda t, *_: None if t is None else 0x1000)
        monkeypatch.setattr(b, "_space", lambda t: (None, 0) if t is None else (0x1000, 1 << 30))
        monkeypatch.setattr(b, "_stream", lambda s: None)
        self.monkeypatch, self.calls = monkeypatch, {}

    def stub(self, name):
        """The entry point's arguments instead of a launch."""
        class Lib:
            def __getattr__(_, n):
                return (lambda *a: self.calls.setdefault(n, a) and 0) if n == name else getattr(b_lib, n)
        b_lib = b._lib
        self.monkeypatch.setattr(b, "_lib", Lib())


def refused(call):
    with pytest.raises((b.SflError, ValueError)) as e:
        call()
    assert getattr(e.value, "code", b.SFL_E_ARG) == b.SFL_E_ARG


def test_dispatch_takes_both_of_rows_and_copies_or_neither(monkeypatch):
    r = Recorded(monkeypatch)
    i, off = torch.zeros((4, 2), dtype=torch.int32), torch.zeros(9, dtype=torch.int32)
    X, Xs = torch.zeros(4, 16), torch.zeros(8, 16)
    refused(lambda: b.sfl_expert_dispatch(i, 8, i, off, Xs=Xs))
    r.stub("sfl_expert_dispatch")
    # no copies wanted: the header allows Xs = NULL where there are no rows
    b.sfl_expert_dispatch(i, 8, i, off, X=X)
    a = r.calls["sfl_expert_dispatch"]
    assert a[6] is not None and a[8] == 16 and a[9] == 0 and a[10] is None


def test_norm_backward_without_the_stored_rows(monkeypatch):
    """The header asks for X_out only with SFL_NORM_PRE and takes a missing dX_out for zeros."""
    r = Recorded(monkeypatch)
    rows, w = torch.zeros(4, 16), torch.zeros(16)
    refused(lambda: b.sfl_norm_backward(None, rows, None, rows, dX=rows, workspace=w))  # SFL_NORM_PRE needs X_out
    with pytest.raises(ValueError):
        b.sfl_norm_backward(None, None, None, norms=0, dgate_c=w, workspace=w)  # nothing says how many rows
    r.stub("sfl_norm_backward")
    for kw in (dict(Y=rows, dY=rows, dw_post=w), dict(Y=None, dX=rows)):
        r.calls.clear()
        b.sfl_norm_backward(None, kw.pop("Y"), None, norms=b.SFL_NORM_POST if "dY" in kw else 0, workspace=w, **kw)
        a = r.calls["sfl_norm_backward"][0]
        assert (a.T, a.d, a.dtype, a.X_out, a.dX_out) == (4, 16, b.SFL_F32, None, None)


def test_combine_backward_without_rows(monkeypatch):
    r = Recorded(monkeypatch)
    dY, pos, w = torch.zeros(4, 16), torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, 2)
    refused(lambda: b.sfl_expert_combine_backward(dY, None, pos, w, dweight=w))
    refused(lambda: b.sfl_expert_combine_backward(dY, None, pos, w, dweight=w, dYs=torch.zeros(8, 16)))
    r.stub("sfl_expert_combine_backward")
    b.sfl_expert_combine_backward(dY, None, pos, w)  # neither gradient is wanted
    assert r.calls["sfl_expert_combine_backward"][7] == 0
