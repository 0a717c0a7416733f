"""The operators around the layer run together: the routed stack of examples/routed_block.py against
a float64 model of it, its training, and its calls under graph capture.

Bounds of the model comparison. About six bf16 tensors are stored per block in each direction, each
rounded with a relative rms error of about 2^-9: with two blocks, outputs carry sqrt(12) 2^-9 = 0.7 %
and are held to the layer's own 2 %. In the gradients a pre-activation within that error of zero may
be active on one side only: a fraction of about 0.8 * 0.7 % = 0.6 % of the active units, which moves
their gradient by sqrt(0.006) = 8 %; with the roundings, 10 %."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("routed_block", os.path.join(ROOT, "examples", "routed_block.py"))
rb = importlib.util.module_from_spec(spec)
spec.loader.exec_module(rb)


def model64(m, X, choices):
    """The stack in float64 with autograd on the CPU, taking the choices of experts as given."""
    leaf = lambda t: t.detach().cpu().double().requires_grad_()  # noqa: E731
    P = [{n: leaf(m.halves[i][n] if n in m.halves[i] else p) for n, p in blk.items()} for i, blk in enumerate(m.blocks)]
    w_out, x0 = leaf(m.w_out), leaf(X)
    norm = lambda v: v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    x, out = x0, None
    n = norm(x) * P[0]["w_pre"]
    for i, p in enumerate(P):
        e = choices[i].cpu().long()
        w = torch.softmax((n @ p["router"]).gather(1, e), 1)
        y = torch.zeros_like(x)
        for j in range(m.E):
            t, s = (e == j).nonzero(as_tuple=True)
            y = y.index_add(0, t, w[t, s][:, None] * (torch.relu(n[t] @ p["W_up"][j]) @ p["W_down"][j]))
        x = m.res_scale * x + p["gate_c"] * (norm(y) * p["w_post"])
        n = norm(x) * (P[i + 1]["w_pre"] if i + 1 < len(P) else w_out)
    return n, P, w_out, x0


def rel(a, ref):
    a, ref = a.detach().cpu().double(), ref.detach()
    return float((a - ref).norm() / ref.norm())


@pytest.mark.parametrize("T,E,k", [(96, 4, 2), (33, 8, 3), (1, 4, 1), (700, 4, 2)])
def test_stack_against_float64(T, E, k):
    m = rb.RoutedStack(2, 512, 256, E, k, res_scale=0.8, seed=T)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    X = torch.randn((T, 512), generator=g, device="cuda").bfloat16()
    dN = torch.randn((T, 512), generator=g, device="cuda").bfloat16()
    out, state = m.forward(X)
    dX = m.backward(state, dN)
    want, P, w_out, x0 = model64(m, X, [s["expert"] for s in state["layers"]])
    assert rel(out, want) < 0.02
    (want * dN.cpu().double()).sum().backward()
    assert rel(dX, x0.grad) < 0.1
    assert rel(m.dw_out, w_out.grad) < 0.1
    for grads, p in zip(m.grads, P):
        for n, v in p.items():
            if n == "router" and k == 1:
                assert grads[n].abs().max() <= 1e-6  # one choice has weight one, whatever its logit
            else:
                assert rel(grads[n], v.grad) < 0.1, n


def test_training_lowers_the_loss_and_clips():
    losses = rb.main(["--tokens", "256", "--width", "512", "--hidden", "512", "--experts", "4", "--steps", "12",
                      "--lr", "3"])
    assert losses[-1] < losses[0]
    m = rb.RoutedStack(1, 512, 256, 4, 2)
    X = torch.randn((64, 512), device="cuda").bfloat16()
    out, state = m.forward(X)
    m.backward(state, torch.ones_like(out))
    before = torch.cat([t.reshape(-1) for t in m.all_grads()]).double()
    norm = m.step(0.0, 1e-3)
    after = torch.cat([t.reshape(-1) for t in m.all_grads()]).double()
    assert abs(norm.item() - before.norm().item()) <= 1e-6 * before.norm().item()
    assert abs(after.norm().item() - 1e-3) <= 1e-9


def test_under_graph_capture():
    """Every operator's launches recorded once and replayed on new inputs, with eager work between
    the replays, against eager calls."""
    T, d, E, k = 3000, 512, 16, 2
    new = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    X, Y, X_out, N, dX, dY = (new(T, d) for _ in range(6))
    logits, w, dw, dl = new(T, E, dt=torch.float32), new(T, k, dt=torch.float32), new(T, k, dt=torch.float32), new(T, E, dt=torch.float32)
    e, pos, off = new(T, k, dt=torch.int32), new(T, k, dt=torch.int32), new(E + 1, dt=torch.int32)
    Xs, dYs, back = new(T * k, d), new(T * k, d), new(T, d)
    g, q, norm = torch.zeros(d, device="cuda"), new(1, dt=torch.float64), new(1, dt=torch.float32)
    ws = torch.empty(max(b.sfl_norm_workspace_size(T, d, "bf16"), b.sfl_expert_workspace_size(T, k, E)),
                     dtype=torch.uint8, device="cuda")
    grads = b.grad_list([dX, dw], [dY, dl.view(-1)[:T * k]])
    gws = torch.empty(b.sfl_grad_workspace_size(grads), dtype=torch.uint8, device="cuda")

    def work():
        b.sfl_norm_forward(X, Y, X_out=X_out, N=N)
        b.sfl_route_forward(logits, e, w)
        b.sfl_expert_dispatch(e, E, pos, off, X=N, Xs=Xs, workspace=ws)
        b.sfl_expert_combine(Xs, pos, back, weight=w)
        b.sfl_expert_combine_backward(X, Xs, pos, w, dYs=dYs, dweight=dw)
        b.sfl_norm_backward(X_out, Y, X, back, dX=dX, dY=dY, dw_post=g, workspace=ws)
        b.sfl_route_backward(logits, e, dw, dl)
        b.sfl_grad_sumsq(grads, q, workspace=gws)
        b.sfl_grad_clip(grads, q, 1.0, norm)

    outs = (X_out, N, e, w, pos, off, Xs, back, dYs, dw, dX, dY, g, dl, q, norm)
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in range(4):
        r = torch.Generator(device="cuda")
        r.manual_seed(seed)
        for t in (X, Y, logits):
            t.copy_(torch.randn(t.shape, generator=r, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        work()
        torch.cuda.synchronize()
        for a, c in zip(got, outs):
            assert torch.equal(a.view(torch.uint8), c.view(torch.uint8))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_step_whose_norm_is_not_finite_changes_nothing(bad):
    m = rb.RoutedStack(1, 512, 256, 4, 2)
    for g in m.all_grads():
        g.fill_(1.0)
    m.grads[0]["W_up"][1, 3, 7] = bad
    params = [p for blk in m.blocks for p in blk.values()] + [m.w_out]
    halves = [h for half in m.halves for h in half.values()]
    before = [t.clone() for t in params + halves]
    norm = m.step(0.1, 1.0)
    assert not norm.isfinite().item()
    assert all(torch.equal(a, t) for a, t in zip(before, params + halves))
    m.grads[0]["W_up"].fill_(1.0)
    assert m.step(0.1, 1.0).isfinite().item()
    assert not any(torch.equal(a, t) for a, t in zip(before, params))
