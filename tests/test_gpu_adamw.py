"""Steps of AdamW against the float64 definition."""
import numpy as np
import pytest
import torch

from block_util import DT, Out, U32, U_BF16, same_bits, stored
from oracle import routed as o
from paper_2603_23198_amd import binding as b
from routed_util import Bytes, F8, up

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8)


class Tensor:
    """One entry of a list, its values in float64 and where they go."""

    def __init__(self, rng, n, param="f32", grad="f32", small=False, half=True, decay=0.0, first=False, shift=0):
        self.n, self.param, self.small, self.decay = n, param, small, decay
        self.p = Out((n,), DT[param], shift)
        P, self.p0 = stored(rng.normal(size=n), param)
        self.p.t.copy_(P)
        G, self.g = stored(rng.normal(size=n) * np.exp(rng.normal(size=n)), grad)
        self.G = Out((n,), DT[grad], shift)
        self.G.t.copy_(G)
        self.half = Out((n,), torch.bfloat16, shift) if half and param == "f32" else None
        m = np.zeros(n) if first else rng.normal(size=n) * 0.3
        v = np.zeros(n) if first else rng.random(size=n) + 0.1
        if not small:
            self.m, self.v = Out((n,), torch.float32, shift), Out((n,), torch.float32, shift)
            M, self.m0 = stored(m, "f32")
            V, self.v0 = stored(v, "f32")
            self.m.t.copy_(M)
            self.v.t.copy_(V)
            self.scales = [None, None]
            return
        self.m, self.v = Bytes((n,), F8), Bytes((n,), F8)
        self.scales = [Bytes((up(n) // 128,)) for _ in range(2)]
        self.held = []
        for x, codes, scale in ((m, self.m, self.scales[0]), (np.sqrt(v), self.v, self.scales[1])):
            q, e = o.quant(x[None])
            codes.bytes.copy_(torch.from_numpy(q[0, :n]))
            scale.bytes.copy_(torch.from_numpy((e[0] + 127).astype(np.uint8)))
            self.held.append(o.held(q, e)[0, :n])
        self.m0, self.v0 = self.held[0], self.held[1] ** 2

    def check(self, t, c=1.0, place=0, seed=0, lr=None):
        h = dict(HYPER, lr=HYPER["lr"] if lr is None else lr)
        p, m, v = o.adamw(self.p0, self.g, self.m0, self.v0, t, weight_decay=self.decay, c=c, **h)
        # fp32 has nothing between 0 and 2^-149: squares under half of that are zero there
        v = np.where(v < 2.0 ** -150, 0, v)
        # moments: each product and sum rounds once, and beta, 1 - beta and c do
        gm, gv = np.abs(0.1 * c * self.g), 0.001 * (c * self.g) ** 2
        tol_m = 6 * U32 * (np.abs(0.9 * self.m0) + gm)
        tol_v = 9 * U32 * (0.999 * self.v0 + gv)
        # the step: its moments' errors (a root halves a relative one), two corrections, a quotient, a sum with
        # eps, a root: ten roundings; then decay, a sum, lr and the difference
        size = np.sqrt(v / (1 - 0.999 ** t)) + h["eps"]
        with np.errstate(invalid="ignore", divide="ignore"):
            rel_v = np.where(v > 0, tol_v / v, 0)
        step = np.abs(m / (1 - 0.9 ** t)) / size
        tol_p = h["lr"] * (tol_m / (1 - 0.9 ** t) / size + step * (rel_v + 12 * U32) + 4 * U32 * self.decay * np.abs(self.p0))
        tol_p = tol_p + 2 * U32 * (np.abs(self.p0) + np.abs(p)) + 1e-37
        self.near(self.p, p, tol_p, self.param)
        if self.half is not None:
            self.near(self.half, p, tol_p, "bf16")
        if not self.small:
            self.near(self.m, m, tol_m + 1e-37, "f32")
            self.near(self.v, v, tol_v + 1e-37, "f32")
            return
        bits = o.noise(place + np.arange(self.n), t, seed)
        root = np.sqrt(v)
        with np.errstate(invalid="ignore", divide="ignore"):
            tol_root = np.where(v > 0, tol_v / (2 * root), 0) + U32 * root
        for x, tol, codes, scale, noise, least in ((m, tol_m, self.m, self.scales[0], bits[0], False),
                                                   (root, tol_root, self.v, self.scales[1], bits[1], True)):
            got, s = codes.values(), scale.values().astype(np.int64) - 127
            wide = np.zeros(up(self.n))
            wide[:self.n] = np.abs(x)
            top = wide.reshape(-1, 128).max(1)
            # the largest magnitude may lie within its error of where the scale changes
            lo, hi = (np.array([o.scale_exponent(a) for a in top * by]) for by in (1 - 1e-6, 1 + 1e-6))
            assert ((s == lo) | (s == hi)).all()
            e = np.repeat(s, 128)[:self.n].astype(np.float64)
            want, sure = o.drawn(x, noise, e, least)
            value = o.from_e4m3(got) * 2.0 ** e
            step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(x) / 2.0 ** e, 2.0 ** -30))), -6) - 3 + e)
            # where the sum of x and its noise, in steps, lies within x's own error of a whole step, either
            # may come. (x's error is that of its terms: where beta m and (1 - beta) g nearly cancel, it is
            # far more than a rounding of x.) The sum of at most 9 steps in fp32 rounds by 2^-21.
            off = (value != want) & (sure > tol / step + 2.0 ** -20)
            assert not off.any(), (off.sum(), np.flatnonzero(off)[:5])
            assert (np.abs(value - x) <= step * 1.001).all()

    def near(self, out, want, tol, dt):
        if dt == "bf16":
            tol = tol + U_BF16 * (np.abs(want) + tol)
        err = np.abs(out.values() - want)
        assert (err <= tol).all(), (dt, (err / tol).max())


def step(ts, t, **kw):
    some = lambda f: [f(x) for x in ts]  # noqa: E731
    scales = [some(lambda x, i=i: None if x.scales[i] is None else x.scales[i].t) for i in range(2)]
    lst = b.adamw_list(some(lambda x: x.p.t), some(lambda x: x.G.t), some(lambda x: x.m.t), some(lambda x: x.v.t),
                       halves=some(lambda x: None if x.half is None else x.half.t), m_scales=scales[0],
                       v_scales=scales[1], weight_decay=some(lambda x: x.decay))
    number = torch.tensor([t], device="cuda")
    b.sfl_adamw_step(lst, number, **HYPER | kw)
    return lst, number


def places(ts):
    return np.cumsum([0] + [up(x.n) for x in ts])


@pytest.mark.parametrize("small", [False, True])
@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_types_and_sizes(small, param, grad):
    for n in (1, 2, 3, 127, 128, 129, 1023, 2048, 2049, 5000):
        rng = np.random.default_rng(n)
        for t in (1, 2, 1000):
            x = Tensor(rng, n, param, grad, small, half=t != 2, decay=0.1 * (t - 1), first=t == 1, shift=n % 4)
            step([x], t, seed=5)
            x.check(t, seed=5)


@pytest.mark.parametrize("count", [1, 2, 7, 37, 38, 39, 90])
def test_lists(count):
    """Mixed types, tensors without elements, more tensors than one launch takes."""
    rng = np.random.default_rng(count)
    ts = [Tensor(rng, int(rng.integers(0, 700)) * (i % 5 > 0), "bf16" if i % 4 == 3 else "f32", "bf16" if i % 3 else "f32",
                 i % 2 > 0, half=i % 7 > 2, decay=0.1 * (i % 3), shift=i % 3) for i in range(count)]
    step(ts, 9, seed=count)
    for x, at in zip(ts, places(ts)):
        x.check(9, place=int(at), seed=count)


def test_a_long_tensor():
    rng = np.random.default_rng(3)
    ts = [Tensor(rng, 300001, small=True), Tensor(rng, 200003, grad="bf16")]
    step(ts, 4)
    for x, at in zip(ts, places(ts)):
        x.check(4, place=int(at))


@pytest.mark.parametrize("small", [False, True])
def test_clipping_on_the_device(small):
    rng = np.random.default_rng(4)
    for factor in (0.5, 2.0):
        ts = [Tensor(rng, n, small=small) for n in (300, 1000)]
        norm = np.sqrt(sum((x.g ** 2).sum() for x in ts))
        sumsq, out = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
        grads = b.grad_list([x.G.t for x in ts])
        ws = torch.empty(b.sfl_grad_workspace_size(grads), dtype=torch.uint8, device="cuda")
        b.sfl_grad_sumsq(grads, sumsq, workspace=ws)
        step(ts, 3, sumsq=sumsq, max_norm=norm * factor, norm=out)
        assert abs(out.item() / norm - 1) < 1e-6
        for x, at in zip(ts, places(ts)):
            x.check(3, min(1.0, factor), place=int(at))


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_norm_that_is_not_finite_changes_nothing(bad):
    rng = np.random.default_rng(5)
    ts = [Tensor(rng, 300, small=s) for s in (False, True)]
    keep = [[t.clone() for t in (x.p.t, x.half.t, x.m.t, x.v.t)] for x in ts]
    scales = [s.t.clone() for s in ts[1].scales]
    out = torch.empty(1, device="cuda")
    step(ts, 3, sumsq=torch.tensor([bad], dtype=torch.float64, device="cuda"), max_norm=1.0, norm=out)
    assert not out.isfinite().item()
    for x, old in zip(ts, keep):
        assert all(same_bits(a, w) for a, w in zip((x.p.t, x.half.t, x.m.t, x.v.t), old))
    assert all(same_bits(a.t, w) for a, w in zip(ts[1].scales, scales))


def test_an_empty_list_gives_the_norm():
    out = torch.empty(1, device="cuda")
    b.sfl_adamw_step(b.adamw_list([], [], [], []), torch.tensor([1], device="cuda"), lr=1.0,
                     sumsq=torch.tensor([9.0], dtype=torch.float64, device="cuda"), max_norm=1.0, norm=out)
    assert out.item() == 3.0


def test_a_learning_rate_on_the_device():
    rng = np.random.default_rng(6)
    x = Tensor(rng, 500)
    step([x], 7, lr_scale=torch.tensor([0.25], device="cuda"))
    x.check(7, lr=HYPER["lr"] * 0.25)


def test_steps_below_one_count_as_one():
    rng = np.random.default_rng(7)
    for t in (0, -3):
        x = Tensor(rng, 200, small=True, first=True)
        step([x], t)
        x.check(1)


def test_small_moments():
    """Blocks of zeros, one element far above the others, elements that underflow a block's scale: a root
    above zero stays above zero, zeros stay zeros."""
    rng = np.random.default_rng(8)
    x = Tensor(rng, 512, small=True, first=True)
    g = np.zeros(512)
    g[128:256] = rng.normal(size=128) * 1e-9
    g[130] = 1e3
    g[256:384] = 1e-30
    g[400] = -1e-3
    x.G.t.copy_(torch.from_numpy(g))
    x.g = x.G.t.double().cpu().numpy()
    step([x], 1)
    x.check(1)
    root = o.from_e4m3(x.v.values())
    assert ((root > 0) == (0.001 * x.g ** 2 >= 2.0 ** -149)).all() and (root > 0).sum() == 129


def test_gradients_that_are_not_finite():
    """Without a norm that stops the step they reach their own elements only."""
    rng = np.random.default_rng(9)
    for small in (False, True):
        x = Tensor(rng, 400, small=small)
        keep = x.g.copy()
        bad = [3, 130, 399]
        x.G.t[bad] = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda")
        step([x], 2)
        p = x.p.values()
        # an infinite gradient gives an infinite second moment: 0/0 or inf/inf
        np.testing.assert_array_equal(np.flatnonzero(np.isnan(p)), bad)
        for codes in (x.m, x.v):
            v = o.from_e4m3(codes.values()) if small else codes.values()
            np.testing.assert_array_equal(np.flatnonzero(~np.isfinite(v)), bad)
        good = np.setdiff1d(np.arange(400), bad)
        want = o.adamw(x.p0[good], keep[good], x.m0[good], x.v0[good], 2, **HYPER)[0]
        np.testing.assert_allclose(p[good], want, rtol=1e-5, atol=1e-6)


def test_places_beyond_32_bits():
    """The noise goes by the place in the whole list: as if a tensor of 2^32 elements came before."""
    places32 = np.array([0, 1, (1 << 32) - 1, 1 << 32, (1 << 33) + 5])
    low = o.noise(places32 & 0xffffffff, 3, 1)
    high = o.noise(places32, 3, 1)
    assert (low[0][:3] == high[0][:3]).all() and (low[0][3:] != high[0][3:]).any()


def test_repeats_and_graphs():
    """Captured steps whose number and gradients change: bit for bit the eager ones."""
    rng = np.random.default_rng(10)

    def make():
        r = np.random.default_rng(10)
        return [Tensor(r, n, small=s, grad="bf16", decay=0.1) for n, s in ((700, True), (500, False))]

    a, e = make(), make()
    lst, number = step(a, 1, seed=3)
    lst2, number2 = step(e, 1, seed=3)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.sfl_adamw_step(lst, number, seed=3, **HYPER)
    for t in range(2, 6):
        for x, y in zip(a, e):
            G = torch.from_numpy(rng.normal(size=x.n)).cuda()
            x.G.t.copy_(G)
            y.G.t.copy_(G)
        number.fill_(t)
        number2.fill_(t)
        g.replay()
        b.sfl_adamw_step(lst2, number2, seed=3, **HYPER)
        torch.cuda.synchronize()
        for x, y in zip(a, e):
            assert same_bits(x.p.t, y.p.t) and same_bits(x.half.t, y.half.t)
            assert same_bits(x.m.t.view(torch.uint8), y.m.t.view(torch.uint8))
            assert same_bits(x.v.t.view(torch.uint8), y.v.t.view(torch.uint8))


def test_moments_in_8_bits_follow_those_in_32():
    """Drawn rounding keeps slow averages moving: after gradients of one size come ones of a tenth, and the
    roots fall with them as in 32 bits (a nearest rounding would leave them where they were)."""
    n = 128 * 40
    p = [torch.zeros(n, device="cuda") for _ in range(2)]
    g = torch.empty(n, device="cuda")
    m32, v32 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m8, v8 = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    ms, vs = (torch.full((n // 128,), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    lst = b.adamw_list([p[0], p[1]], [g, g], [m32, m8], [v32, v8], m_scales=[None, ms], v_scales=[None, vs])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for t in range(1, 601):
        g.copy_(torch.randn(n, generator=gen, device="cuda") * (1.0 if t <= 100 else 0.1))
        b.sfl_adamw_step(lst, torch.tensor([t], device="cuda"), lr=1e-3, beta2=0.99, seed=2)
    root8 = v8.float() * torch.exp2(vs.float() - 127).repeat_interleave(128)
    ratio = (root8.square().mean() / v32.mean()).sqrt().item()
    # a code is off by a step of at most 1/8; 5120 elements average what the draws add
    assert 0.85 < ratio < 1.15, ratio


@pytest.mark.parametrize("byte", [0, 1, 127, 254, 255])
def test_moments_of_zero_codes_and_any_scale(byte):
    """Before the first step the codes are zeros, and their scales may be anything."""
    rng = np.random.default_rng(byte)
    for n in (5000, 130):
        x = Tensor(rng, n, small=True, first=True)
        for s in x.scales:
            s.bytes.fill_(byte)
        step([x], 1, seed=2)
        x.check(1, seed=2)


def test_the_step_is_a_quotient_rounded_once():
    """beta1 = beta2 = 0, lr = 1 and parameters of zero: m = g and sqrt(v) = |g| without a rounding, so is
    |g| + eps, and the new parameter is -g / (|g| + eps)."""
    rng = np.random.default_rng(12)
    n = 40000
    g = (rng.integers(1, 1 << 11, size=n) * rng.choice([-1.0, 1.0], size=n)).astype(np.float32)
    p, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    lst = b.adamw_list([p], [torch.from_numpy(g).cuda()], [m], [v])
    b.sfl_adamw_step(lst, torch.tensor([1], device="cuda"), lr=1.0, beta1=0.0, beta2=0.0, eps=2.0 ** -8)
    np.testing.assert_array_equal(p.cpu().numpy(), -(g / (np.abs(g) + np.float32(2.0 ** -8))))


def test_quotients_beyond_fp32():
    """m / eps above every fp32 number is an infinite step, one by an infinite root none, inf / inf NaN."""
    inf = float("inf")
    m, v = torch.tensor([1e30, -1e30, 1.0, -inf, inf]).cuda(), torch.tensor([0.0, 0.0, inf, 0.0, inf]).cuda()
    p, g = torch.ones(5, device="cuda"), torch.zeros(5, device="cuda")
    b.sfl_adamw_step(b.adamw_list([p], [g], [m], [v]), torch.tensor([3], device="cuda"), lr=1e-3, eps=1e-30)
    np.testing.assert_array_equal(p.cpu().numpy(), [-inf, inf, 1, inf, np.nan])


def test_a_norm_that_clips_nothing():
    """max_norm = inf: the norm is written and looked at, the gradients are as they are."""
    rng = np.random.default_rng(13)
    x = Tensor(rng, 700)
    out = torch.empty(1, device="cuda")
    step([x], 3, sumsq=torch.tensor([1e6], dtype=torch.float64, device="cuda"), max_norm=float("inf"), norm=out)
    assert out.item() == 1e3
    x.check(3)
