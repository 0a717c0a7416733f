"""Workspace sizes never fall as a call grows: one allocation for the largest batch or the longest
list serves every smaller one."""
import pytest

from paper_2603_23198_amd import binding as b

P = 0x1000  # a pointer that is never followed


@pytest.mark.parametrize("k", [1, 2, 3, 8, 64])
def test_expert_order(k):
    # around one launch's slots, whole tiles and every step of a workgroup's run of slots
    at = sorted({max(0, s // k + i) for s in (0, 1024, 2048, 4096, *(262144 * n for n in range(1, 12)), (1 << 31) - 1 - 64)
                 for i in (-1025, -1024, -2, -1, 0, 1, 2, 1023, 1024, 1025)})
    at = [T for T in at if T <= ((1 << 31) - 1) // k]
    for E in (1, 64, 1024):
        sizes = [b.sfl_expert_workspace_size(T, k, E) for T in at]
        assert sizes == sorted(sizes), (E, [(T, s) for T, s, n in zip(at, sizes, sizes[1:]) if n < s])


def test_expert_order_takes_the_workspace_of_a_larger_batch():
    for T in (1025, 1024 * 128, 1024 * 256):
        larger = max(b.sfl_expert_workspace_size(T + n, 2, 64) for n in (1, 1000, 1 << 20))
        assert b.sfl_expert_workspace_size(T, 2, 64) <= larger


def grad_bytes(lens):
    l = (b.Grad * len(lens))(*[(P, None, n, b.SFL_F32, 0) for n in lens])
    return b.sfl_grad_workspace_size(l)


def test_gradients():
    steps = [(1 << p) + i for p in (11, 20, 21, 22, 23, 26, 33) for i in (-4097, -4096, -1, 0, 1, 2047, 2048, 2049, 4096, 8192)]
    for beside in ([], [1], [5, 3000, 0, 70000], [(1 << 20) + 7], [3] * 500):
        sizes = [grad_bytes(beside + [n]) for n in sorted(steps) if n >= 0]
        assert sizes == sorted(sizes), beside
    for n in (1, 2048, 2049, 100_000, (1 << 20) + 1, 1 << 21):  # more and more tensors
        sizes = [grad_bytes([n] * m) for m in range(0, 130)]
        assert sizes == sorted(sizes), n


def test_gradients_parts_of_a_list():
    lens = [1 << 20, 3, 70_000, 0, 1 << 21, 4097, 1 << 22, 11]
    whole = grad_bytes(lens)
    assert all(grad_bytes(lens[i:j]) <= whole for i in range(len(lens)) for j in range(i, len(lens) + 1))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norms(dt):
    for d in (1, 64, 130, 640, 1003, 4096, 8200, 16384):
        sizes = [b.sfl_norm_workspace_size(T, d, dt) for T in (*range(0, 70), 511, 512, 513, 8191, 8192, 8193, 1 << 20)]
        assert sizes == sorted(sizes), d


def test_alignment():
    """Workspaces hold fp32 sums, int32 counts and fp64 sums: 4, 4 and 8 bytes."""
    norm = b.NormBwdArgs()
    norm.dtype, norm.norms, norm.T, norm.d, norm.eps, norm.res_scale = b.SFL_BF16, 3, 4, 64, 1e-6, 1.0
    norm.X_out = norm.Y = norm.dX_out = norm.dN = norm.dX = P
    norm.workspace_bytes = 1 << 30
    one = (b.Grad * 1)((P, None, 10, 0, 0))
    for by in (1, 2, 3):
        norm.workspace = P + by
        assert b._lib.sfl_norm_backward(norm, None) == b.SFL_E_ARG
        assert b._lib.sfl_expert_dispatch(P, 16384, 8, 64, P, P, None, 0, 1, 0, None, P + by, 1 << 30, None) == b.SFL_E_ARG
    for by in range(1, 8):
        assert b._lib.sfl_grad_sumsq(one, 1, P, P + by, 1 << 20, None) == b.SFL_E_ARG


def test_a_workspace_that_is_not_needed_may_lie_anywhere():
    """(On the CPU the launch itself is what fails.)"""
    assert b._lib.sfl_expert_dispatch(P, 4, 2, 8, P, P, None, 0, 1, 0, None, None, 0, None) != b.SFL_E_ARG
