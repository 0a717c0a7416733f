"""Calls whose work items pass 2^32, the most of one HIP launch: they go in several launches. The
inputs are mostly zeros or unused, so that only the few rows that matter are made and compared."""
import pytest
import torch

from tests.block_util import same_bits

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")


@pytest.fixture(autouse=True)
def released():
    """The next test finds the memory free again."""
    yield
    torch.cuda.empty_cache()


def room(nbytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes + (4 << 30):
        pytest.skip(f"needs {nbytes >> 30} GiB of device memory")


def test_expert_rows():
    """2^24 tokens and more at a workgroup of 256 per token: six of them have a row."""
    T, d = (1 << 24) + 5, 1032
    room(2 * T * d)
    at = torch.tensor([0, 70_000, (1 << 24) - 2, (1 << 24) - 1, 1 << 24, T - 1], device="cuda")
    n = len(at)
    expert = torch.full((T, 1), -1, dtype=torch.int32, device="cuda")
    expert[at] = torch.tensor([[0], [1], [0], [1], [0], [1]], dtype=torch.int32, device="cuda")
    want_pos = torch.tensor([0, 3, 1, 4, 2, 5], device="cuda")
    rows = torch.randn((n, d), device="cuda").bfloat16()
    wide = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    wide[at] = rows
    pos, off = torch.empty_like(expert), torch.empty(3, dtype=torch.int32, device="cuda")
    Xs = torch.full((n, d), -77, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(b.sfl_expert_workspace_size(T, 1, 2), dtype=torch.uint8, device="cuda")
    b.sfl_expert_dispatch(expert, 2, pos, off, X=wide, Xs=Xs, workspace=ws)
    assert off.tolist() == [0, 3, 6]
    assert torch.equal(pos[at, 0].long(), want_pos) and int((pos >= 0).sum()) == n
    assert same_bits(Xs[want_pos], rows)

    dYs, dw = torch.full_like(Xs, -77), torch.full((T, 1), -77.0, device="cuda")
    weight = torch.zeros((T, 1), device="cuda")
    weight[at, 0] = torch.tensor([0.5, 2.0, -1.0, 4.0, 0.25, 1.0], device="cuda")
    b.sfl_expert_combine_backward(wide, Xs, pos, weight, dYs=dYs, dweight=dw)
    assert same_bits(dYs[want_pos], (rows.float() * weight[at]).bfloat16())
    dot = rows.double().square().sum(1)  # within d / 64 + 32 fp32 roundings
    assert ((dw[at, 0].double() - dot).abs() <= (d / 64 + 32) * 2.0 ** -24 * dot).all()
    assert int((dw != 0).sum()) == n

    wide.fill_(-77)
    b.sfl_expert_combine(Xs, pos, wide, weight=weight)
    assert same_bits(wide[at], (rows.float() * weight[at]).bfloat16())
    wide[at] = 0
    assert not any(part.any() for part in wide.split(1 << 20))


@pytest.mark.parametrize("E", [130, 300])
def test_router(E):
    """2^26 tokens at a wave per token, against calls of a few of them."""
    T, k = (1 << 26) + 3, 2
    room(2 * 2 * T * E + 4 * 4 * T * k)
    if E == 130:
        logits = torch.empty((T, E), dtype=torch.bfloat16, device="cuda").normal_()
    else:  # 40 GB: the same rows again and again
        logits = torch.randn((1 << 10, E), device="cuda").bfloat16().repeat((1 << 16) + 1, 1)[:T]
    dweight = torch.randn((T, k), device="cuda")
    expert, weight = torch.full((T, k), -7, dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    dlogits = torch.full_like(logits, -77)
    b.sfl_route_forward(logits, expert, weight)
    b.sfl_route_backward(logits, expert, dweight, dlogits)
    assert int((expert < 0).sum()) == 0
    for z in (9, 1 << 25, (1 << 26) - 4, (1 << 26) - 3, 1 << 26, T):
        s = slice(z - 9, z)
        e, w, dl = expert[s].clone(), weight[s].clone(), dlogits[s].clone()
        b.sfl_route_forward(logits[s], e.zero_(), w.zero_())
        b.sfl_route_backward(logits[s], e, dweight[s], dl.zero_())
        assert torch.equal(e, expert[s]) and same_bits(w, weight[s]) and same_bits(dl, dlogits[s])


def test_one_gradient():
    """A tensor of more shares than the scaling pass has workgroups in a launch."""
    share, n = 4096, (1 << 36) + 77
    room(2 * n)
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    most = ((1 << 32) - 1) // 256 * share
    at = sorted({0, 1, share, n // 2, most - 1, most, most + 1, n - most - 1, n - most, n - most + 1, n - share, n - 1})
    for i in at:
        g[i] = 2.0
    grads = b.grad_list([g])
    q = torch.empty(1, dtype=torch.float64, device="cuda")
    norm = torch.empty(1, device="cuda")
    b.sfl_grad_sumsq(grads, q, workspace=torch.empty(b.sfl_grad_workspace_size(grads), dtype=torch.uint8, device="cuda"))
    assert q.item() == 4.0 * len(at)
    b.sfl_grad_clip(grads, q, norm.copy_(q.sqrt() / 4).item(), norm)
    assert abs(norm.item() - q.sqrt().item()) <= 2.0 ** -23 * norm.item()
    assert [g[i].item() for i in at] == [0.5] * len(at)
    for i in at:
        g[i] = 0
    assert not any(part.any() for part in g.split(1 << 31))


def test_many_large_gradients():
    """Ranges whose shares pass a launch of the sum together (one tensor, listed again and again; an
    allowed norm above theirs leaves it as it is)."""
    n, times = (1 << 31) + 9, 70
    room(2 * n)
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[n // 3], g[n - 1] = 1.0, 2.0, 2.0
    grads = b.grad_list([g] * times)
    q, norm = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    b.sfl_grad_sumsq(grads, q, workspace=torch.empty(b.sfl_grad_workspace_size(grads), dtype=torch.uint8, device="cuda"))
    assert q.item() == 9.0 * times
    b.sfl_grad_clip(grads, q, 1e6, norm)
    assert abs(norm.item() - (9.0 * times) ** 0.5) <= 2.0 ** -23 * norm.item()
    assert [g[i].item() for i in (0, n // 3, n - 1)] == [1.0, 2.0, 2.0]
