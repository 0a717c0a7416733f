"""The operators for many routed experts in 8 bits as they are used together: one feed-forward block of
8-bit experts with its router, forward and backward, and a step of the optimiser, all captured into one
graph; against the same block in float64."""
import numpy as np
import pytest
import torch

from block_util import U32, U_BF16, same_bits
from oracle import routed as o
from paper_2603_23198_amd import binding as b
from routed_util import F8, up

pytestmark = pytest.mark.gpu

ROUTE = dict(score="sigmoid", scale=2.0)
GROUPS = dict(groups=4, group_k=2, group_top=2)


class Block:
    """T tokens of width d, E experts of hidden width f, k choices; every buffer made once."""

    def __init__(self, T, d, f, E, k, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        dev, bf = "cuda", torch.bfloat16
        self.T, self.d, self.f, self.E, self.k = T, d, f, E, k
        R = self.R = T * k  # rows in expert order

        def normal(*shape, std=1.0):
            return torch.randn(shape, generator=g, device=dev) * std

        self.X, self.dY = normal(T, d).bfloat16(), normal(T, d, std=0.1).bfloat16()
        self.logits, self.bias = normal(T, E), normal(E, std=0.1)
        self.W1, self.W2 = normal(E, f, d, std=d ** -0.5), normal(E, d, f, std=f ** -0.5)  # [out][in]
        e = lambda *s, t=bf: torch.empty(s, dtype=t, device=dev)  # noqa: E731
        i32, f32, u8 = torch.int32, torch.float32, torch.uint8
        self.expert, self.weight, self.pos, self.offsets = e(T, k, t=i32), e(T, k, t=f32), e(T, k, t=i32), e(E + 1, t=i32)
        self.ws = e(max(1, b.sfl_expert_workspace_size(T, k, E)), t=u8)
        columns = b.sfl_quant_columns(R, E)

        def rows(n):
            return [e(R, up(n), t=F8), e(R, up(up(n) // 128, 4), t=u8)]

        def cols(n):
            return [e(n, columns, t=F8), e(n, columns // 128, t=u8)]

        def matrix(r, c):
            return [e(E, r, up(c), t=F8), e(E, up(r) // 128, up(up(c) // 128, 4), t=u8)]

        self.Xs, self.H, self.Ys, self.Y = e(R, d), e(R, f), e(R, d), e(T, d)
        self.xq, self.xt, self.hq, self.ht = rows(d), cols(d), rows(f), cols(f)
        self.w1, self.w1t, self.w2, self.w2t = matrix(f, d), matrix(d, f), matrix(d, f), matrix(f, d)
        self.dYs, self.dH, self.dXs, self.dX = e(R, d), e(R, f), e(R, d), e(T, d)
        self.dyq, self.dyt, self.dhq, self.dht = rows(d), cols(d), rows(f), cols(f)
        self.dweight, self.dlogits = e(T, k, t=f32), e(T, E, t=f32)
        self.dW1, self.dW2 = e(E, f, d, t=f32), e(E, d, f, t=f32)
        self.sumsq, self.norm = e(1, t=torch.float64), e(1, t=f32)
        params, grads = [self.W1, self.W2], [self.dW1, self.dW2]
        self.grads = b.grad_list(grads)
        self.gws = e(max(1, b.sfl_grad_workspace_size(self.grads)), t=u8)
        self.m = [torch.zeros(p.numel(), dtype=u8, device=dev).view(F8) for p in params]
        self.v = [torch.zeros(p.numel(), dtype=u8, device=dev).view(F8) for p in params]
        self.ms = [torch.full((up(p.numel()) // 128,), 127, dtype=u8, device=dev) for p in params]
        self.vs = [s.clone() for s in self.ms]
        self.list = b.adamw_list(params, grads, self.m, self.v, m_scales=self.ms, v_scales=self.vs, weight_decay=0.01)
        self.step_number = torch.tensor([1], device=dev)

    def forward(self):
        of = dict(offsets=self.offsets)
        b.sfl_quant_weights(self.W1, *self.w1, Qt=self.w1t[0], St=self.w1t[1])
        b.sfl_quant_weights(self.W2, *self.w2, Qt=self.w2t[0], St=self.w2t[1])
        b.sfl_route_groups_forward(self.logits, self.expert, self.weight, bias=self.bias, **ROUTE, **GROUPS)
        b.sfl_expert_dispatch(self.expert, self.E, self.pos, self.offsets, X=self.X, Xs=self.Xs, workspace=self.ws)
        b.sfl_quant_rows(self.Xs, *self.xq, Qt=self.xt[0], St=self.xt[1], **of)
        b.sfl_quant_product(*self.xq, *self.w1, self.H, **of)
        b.sfl_quant_rows(self.H, *self.hq, Qt=self.ht[0], St=self.ht[1], where=self.H, **of)  # with the ReLU
        b.sfl_quant_product(*self.hq, *self.w2, self.Ys, **of)
        b.sfl_expert_combine(self.Ys, self.pos, self.Y, weight=self.weight)

    def backward(self):
        of = dict(offsets=self.offsets)
        b.sfl_expert_combine_backward(self.dY, self.Ys, self.pos, self.weight, dYs=self.dYs, dweight=self.dweight)
        b.sfl_quant_rows(self.dYs, *self.dyq, Qt=self.dyt[0], St=self.dyt[1], **of)
        b.sfl_quant_product(*self.dyq, *self.w2t, self.dH, **of)
        b.sfl_quant_product_weights(*self.dyt, *self.ht, self.dW2, **of)
        b.sfl_quant_rows(self.dH, *self.dhq, Qt=self.dht[0], St=self.dht[1], where=self.H, **of)
        b.sfl_quant_product(*self.dhq, *self.w1t, self.dXs, **of)
        b.sfl_quant_product_weights(*self.dht, *self.xt, self.dW1, **of)
        b.sfl_expert_combine(self.dXs, self.pos, self.dX)
        b.sfl_route_groups_backward(self.logits, self.expert, self.dweight, self.dlogits, **ROUTE)

    def step(self):
        b.sfl_grad_sumsq(self.grads, self.sumsq, workspace=self.gws)
        b.sfl_adamw_step(self.list, self.step_number, lr=1e-3, sumsq=self.sumsq, max_norm=1.0, norm=self.norm, seed=4)

    def run(self):
        self.forward()
        self.backward()
        self.step()

    def state(self):
        return [self.W1, self.W2, *self.m, *self.v, *self.ms, *self.vs]

    def outputs(self):
        # of the codes those of the rows; some of the columns are not written
        return [self.expert, self.weight, self.Y, self.dX, self.dW1, self.dW2, self.dlogits, self.norm, *self.state()]


def host(t):
    return t.detach().cpu().double().numpy()


def quant_rows(x):
    q, e = o.quant(x)
    return o.held(q, e)[:, :x.shape[1]]


def quant_matrix(w):
    q, e = o.quant_square(w)
    return o.held(q, e, 128)[:, :w.shape[1]]


def near(got, want, rel, name):
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert off < rel, f"{name}: {off}"


def test_block_against_float64():
    """Every stage from the stage before it as the library left it, so that no difference of one is
    amplified by a later one's codes; sizes that fill no block and no tile."""
    T, d, f, E, k = 150, 200, 330, 8, 2
    s = Block(T, d, f, E, k)
    W = [host(s.W1), host(s.W2)]
    s.forward()
    s.backward()
    torch.cuda.synchronize()
    X, logits, dY = host(s.X), host(s.logits), host(s.dY)
    expert, weight = o.route_groups(logits, k, bias=host(s.bias), **ROUTE, **GROUPS)
    np.testing.assert_array_equal(s.expert.cpu().numpy(), expert)
    order = np.argsort(expert.reshape(-1), kind="stable")
    tokens = order // k
    of = np.concatenate([[0], np.cumsum(np.bincount(expert.reshape(-1), minlength=E))])
    np.testing.assert_array_equal(s.offsets.cpu().numpy(), of)
    got = {n: host(getattr(s, n)) for n in ("H", "Ys", "Y", "dYs", "dH", "dXs", "dX", "dW1", "dW2", "dweight", "dlogits")}
    # the 8-bit instruction and one bf16 rounding, against the result as a whole
    bf16 = U_BF16 + 2.0 ** -11
    on = got["H"] > 0
    relu, dH = np.where(on, got["H"], 0), np.where(on, got["dH"], 0)
    for e in range(E):
        at = slice(of[e], of[e + 1])
        if of[e] == of[e + 1]:
            assert not got["dW1"][e].any() and not got["dW2"][e].any()
            continue
        w1, w2, x = quant_matrix(W[0][e]), quant_matrix(W[1][e]), X[tokens[at]]
        near(got["H"][at], quant_rows(x) @ w1.T, bf16, "H")
        near(got["Ys"][at], quant_rows(relu[at]) @ w2.T, bf16, "Ys")
        near(got["dH"][at], quant_rows(got["dYs"][at]) @ w2, bf16, "dH")
        near(got["dXs"][at], quant_rows(dH[at]) @ w1, bf16, "dXs")
        turn = lambda a: quant_rows(np.ascontiguousarray(a.T))  # noqa: E731
        near(got["dW2"][e], turn(got["dYs"][at]) @ turn(relu[at]).T, 400 * U32, "dW2")
        near(got["dW1"][e], turn(dH[at]) @ turn(x).T, 400 * U32, "dW1")
    # and the whole against the block without 8 bits: each product's operands are off by at most 2^-4 of
    # themselves, at random; two products behind one another, and what a sign of H decides
    Y = np.zeros((T, d))
    for r, slot in enumerate(order):
        t, j = divmod(slot, k)
        e = expert[t, j]
        Y[t] += weight[t, j] * (W[1][e] @ np.maximum(W[0][e] @ X[t], 0))
    near(got["Y"], Y, 2.0 ** -4, "Y")
    near(got["dlogits"], o.route_groups_backward(logits, expert, got["dweight"], **ROUTE), 100 * U32, "dlogits")


def test_the_gradient_follows_differences():
    """Along the block's own gradient, in 8 bits, the loss of the block in float64 falls as the gradient's
    norm says, to the accuracy that 8 bits leave."""
    T, d, f, E, k = 96, 128, 256, 8, 2
    s = Block(T, d, f, E, k, seed=3)
    W1, W2 = host(s.W1), host(s.W2)
    s.forward()
    s.backward()
    torch.cuda.synchronize()
    X, dY = host(s.X), host(s.dY)
    expert, weight = host(s.expert).astype(int), host(s.weight)
    dW1, dW2 = host(s.dW1), host(s.dW2)

    def loss(by):
        total = 0.0
        for t in range(T):
            for j in range(k):
                e = expert[t, j]
                h = np.maximum((W1[e] + by * dW1[e]) @ X[t], 0)
                total += weight[t, j] * dY[t] @ ((W2[e] + by * dW2[e]) @ h)
        return total

    slope = (loss(1e-6) - loss(-1e-6)) / 2e-6
    norm2 = (dW1 ** 2).sum() + (dW2 ** 2).sum()
    assert abs(slope / norm2 - 1) < 2.0 ** -4


def test_the_whole_block_in_one_graph():
    """Captured with the expert's loads on the device and replayed on batches of other loads: the bits of
    the eager calls, parameters and moments carried from step to step."""
    a, e = (Block(150, 200, 330, 8, 2, seed=7) for _ in range(2))
    a.run()
    e.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for step in range(2, 6):
        X, logits = torch.randn((150, 200), generator=g, device="cuda"), torch.randn((150, 8), generator=g, device="cuda")
        logits[:, 3] += 2 * (step - 3)  # a favourite, then an expert that few take
        for s in (a, e):
            s.X.copy_(X)
            s.logits.copy_(logits)
            s.step_number.fill_(step)
        graph.replay()
        e.run()
        torch.cuda.synchronize()
        for x, y in zip(a.outputs(), e.outputs()):
            assert same_bits(x, y)
        assert a.norm.isfinite().item()
