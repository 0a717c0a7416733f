"""Argument checks of the operators around the layer that need no GPU: they are made before any
launch, in C for sizes and pointers and in the binding for tensors."""
import ctypes

import pytest
import torch

from paper_2603_23198_amd import binding as b

P = 0x1000  # a pointer that is never followed
lib = b._lib


def norm(**kw):
    a = b.NormArgs()
    a.dtype, a.norms, a.T, a.d, a.eps, a.res_scale = b.SFL_BF16, 3, 4, 64, 1e-6, 1.0
    a.X = a.Y = a.X_out = a.N = P
    for n, v in kw.items():
        setattr(a, n, v)
    return lib.sfl_norm_forward(ctypes.byref(a), None)


def norm_bwd(**kw):
    a = b.NormBwdArgs()
    a.dtype, a.norms, a.T, a.d, a.eps, a.res_scale = b.SFL_BF16, 3, 4, 64, 1e-6, 1.0
    a.X_out = a.Y = a.dX_out = a.dN = a.dX = a.workspace = P
    a.workspace_bytes = 1 << 30
    for n, v in kw.items():
        setattr(a, n, v)
    return lib.sfl_norm_backward(ctypes.byref(a), None)


@pytest.mark.parametrize("call", [norm, norm_bwd])
def test_norm_sizes_and_options(call):
    for kw in (dict(dtype=7), dict(norms=4), dict(norms=-1), dict(T=-1), dict(d=0), dict(d=-5), dict(eps=-1.0),
               dict(eps=float("nan")), dict(Y=None), dict(norms=2, w_pre=P), dict(norms=1, w_post=P),
               dict(norms=1, Y=None, gate_c=P), dict(norms=1, Y=None, gate_t=P), dict(T=1 << 60, d=64)):
        assert call(**kw) == b.SFL_E_ARG, kw
    assert call(d=16385) == b.SFL_E_UNSUPPORTED


def test_norm_buffers():
    assert lib.sfl_norm_forward(None, None) == b.SFL_E_ARG and lib.sfl_norm_backward(None, None) == b.SFL_E_ARG
    for kw in (dict(X=None), dict(N=None), dict(norms=2), dict(norms=2, N=None, X_out=None)):
        assert norm(**kw) == b.SFL_E_ARG, kw
    assert norm(T=0, X=None, Y=None, X_out=None, N=None) == b.SFL_OK
    for kw in (dict(X_out=None), dict(norms=2, dN=P), dict(norms=2, dN=None, dw_pre=P), dict(norms=1, dw_post=P),
               dict(norms=1, Y=None, dY=P), dict(norms=1, Y=None, dgate_c=P), dict(norms=1, Y=None, dgate_t=P)):
        assert norm_bwd(**kw) == b.SFL_E_ARG, kw
    need = b.sfl_norm_workspace_size(4, 64, "bf16")
    assert need > 0
    assert norm_bwd(workspace_bytes=need - 1) == b.SFL_E_WORKSPACE and norm_bwd(workspace=None) == b.SFL_E_WORKSPACE
    out = ctypes.c_size_t(0)
    assert lib.sfl_norm_workspace_size(4, 64, 1, None) == b.SFL_E_ARG
    assert lib.sfl_norm_workspace_size(4, 16385, 1, ctypes.byref(out)) == b.SFL_E_UNSUPPORTED
    assert lib.sfl_norm_workspace_size(-1, 64, 1, ctypes.byref(out)) == b.SFL_E_ARG


def test_route():
    def f(logits=P, dtype=0, T=4, E=8, k=2, norm=1, expert=P, weight=P):
        return lib.sfl_route_forward(logits, dtype, T, E, k, norm, 1.0, expert, weight, None)

    def g(logits=P, dtype=0, T=4, E=8, k=2, norm=1, expert=P, dweight=P, dlogits=P):
        return lib.sfl_route_backward(logits, dtype, T, E, k, norm, 1.0, expert, dweight, dlogits, None)

    for call in (f, g):
        for kw in (dict(dtype=3), dict(T=-1), dict(E=0), dict(k=0), dict(k=9), dict(norm=2), dict(logits=None),
                   dict(expert=None)):
            assert call(**kw) == b.SFL_E_ARG, kw
        for kw in (dict(E=1025), dict(E=100, k=65), dict(T=1 << 31)):
            assert call(**kw) == b.SFL_E_UNSUPPORTED, kw
        assert call(T=0, logits=None, expert=None) == b.SFL_OK
    assert f(weight=None) == g(dweight=None) == g(dlogits=None) == b.SFL_E_ARG


def test_experts():
    def there(expert=P, T=4, k=2, E=8, pos=P, offsets=P, X=P, dtype=1, d=64, rows=8, Xs=P, ws=P, n=1 << 30):
        return lib.sfl_expert_dispatch(expert, T, k, E, pos, offsets, X, dtype, d, rows, Xs, ws, n, None)

    def back(Ys=P, dtype=1, T=4, d=64, k=2, pos=P, rows=8, w=P, Y=P):
        return lib.sfl_expert_combine(Ys, dtype, T, d, k, pos, rows, w, Y, None)

    def grad(dY=P, Ys=P, dtype=1, T=4, d=64, k=2, pos=P, rows=8, w=P, dYs=P, dw=P):
        return lib.sfl_expert_combine_backward(dY, Ys, dtype, T, d, k, pos, rows, w, dYs, dw, None)

    for call in (there, back, grad):
        for kw in (dict(dtype=9), dict(T=-1), dict(k=0), dict(d=0), dict(rows=-1), dict(pos=None)):
            assert call(**kw) == b.SFL_E_ARG, kw
        for kw in (dict(k=65), dict(T=1 << 30, k=2)):
            assert call(**kw) == b.SFL_E_UNSUPPORTED, kw
    for kw in (dict(expert=None), dict(offsets=None), dict(E=0), dict(Xs=None), dict(X=None)):
        assert there(**kw) == b.SFL_E_ARG, kw
    assert there(E=1025) == b.SFL_E_UNSUPPORTED
    for kw in (dict(Ys=None), dict(Y=None)):
        assert back(**kw) == b.SFL_E_ARG, kw
    for kw in (dict(Ys=None), dict(dY=None)):
        assert grad(**kw) == b.SFL_E_ARG, kw
    assert back(T=0, pos=None, Y=None, Ys=None) == grad(T=0, pos=None, dY=None) == b.SFL_OK
    need = b.sfl_expert_workspace_size(16384, 8, 64)
    if need:
        assert there(T=16384, k=8, E=64, ws=None) == b.SFL_E_WORKSPACE
        assert there(T=16384, k=8, E=64, n=need - 1) == b.SFL_E_WORKSPACE
    out = ctypes.c_size_t(0)
    assert lib.sfl_expert_workspace_size(4, 2, 0, ctypes.byref(out)) == b.SFL_E_ARG
    assert lib.sfl_expert_workspace_size(4, 2, 8, None) == b.SFL_E_ARG
    assert lib.sfl_expert_workspace_size(4, 2, 2000, ctypes.byref(out)) == b.SFL_E_UNSUPPORTED


def test_gradients():
    one = (b.Grad * 1)((P, None, 10, 0, 0))
    for bad in ((P, None, -1, 0, 0), (None, None, 5, 0, 0), (P, None, 5, 6, 0)):
        l = (b.Grad * 1)(bad)
        assert lib.sfl_grad_sumsq(l, 1, P, P, 1 << 20, None) == b.SFL_E_ARG
        assert lib.sfl_grad_clip(l, 1, P, 1.0, P, None) == b.SFL_E_ARG
    assert lib.sfl_grad_sumsq(None, 1, P, P, 1 << 20, None) == lib.sfl_grad_sumsq(one, -1, P, P, 9, None) == b.SFL_E_ARG
    assert lib.sfl_grad_sumsq(one, 1, None, P, 1 << 20, None) == b.SFL_E_ARG
    assert lib.sfl_grad_sumsq(one, 1, P, None, 1 << 20, None) == b.SFL_E_WORKSPACE
    assert lib.sfl_grad_sumsq(one, 1, P, P, b.sfl_grad_workspace_size(one) - 1, None) == b.SFL_E_WORKSPACE
    for m in (-1.0, float("nan")):
        assert lib.sfl_grad_clip(one, 1, P, m, P, None) == b.SFL_E_ARG
    assert lib.sfl_grad_clip(one, 1, None, 1.0, P, None) == b.SFL_E_ARG
    assert lib.sfl_grad_workspace_size(one, 1, None) == b.SFL_E_ARG


def test_the_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4, 64)
    for bad in (torch.zeros(4, 63), torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, 4).t()):
        with pytest.raises(ValueError):
            b.sfl_norm_forward(x, bad, X_out=x, N=x, stream=0)
    i = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        b.sfl_route_forward(x, i.long(), torch.zeros(4, 2), stream=0)
    with pytest.raises(ValueError):
        b.sfl_expert_dispatch(i, 8, i, torch.zeros(8, dtype=torch.int32), stream=0)
    with pytest.raises(ValueError):
        b.sfl_expert_combine(x, i, torch.zeros(4, 64, dtype=torch.bfloat16), stream=0)
    with pytest.raises(ValueError):
        b.grad_list([torch.zeros(4, 4).t()[1:]])
    with pytest.raises(ValueError):
        b.grad_list([x], [torch.zeros(3)])
    with pytest.raises(ValueError):
        b.grad_list([torch.zeros(3, dtype=torch.float64)])
