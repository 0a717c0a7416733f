"""Helpers of the tests of the operators for many routed experts in 8 bits."""
import numpy as np
import torch

from oracle import routed as o

F8 = torch.float8_e4m3fn


def up(n, m=128):
    return -(-n // m) * m


def run_offsets(loads, first=0):
    of = np.cumsum([first] + list(loads))
    return of.tolist(), torch.tensor(of, dtype=torch.int32, device="cuda")


class Bytes:
    """An output of single bytes (codes or scales), filled with a sentinel between sentinel bands of 64."""

    def __init__(self, shape, dtype=torch.uint8, fill=0xA5):
        n = int(np.prod(shape))
        self.raw = torch.full((n + 128,), fill, dtype=torch.uint8, device="cuda")
        self.fill, self.bytes = fill, self.raw[64:64 + n].view(shape)
        self.t = self.bytes.view(dtype)

    def values(self):
        assert (self.raw[:64] == self.fill).all() and (self.raw[-64:] == self.fill).all(), "written out of bounds"
        return self.bytes.cpu().numpy()


def row_outputs(T, d):
    return Bytes((T, up(d)), F8), Bytes((T, up(up(d) // 128, 4)))


def column_outputs(d, columns):
    return Bytes((d, columns), F8), Bytes((d, columns // 128))


def same_codes(got, want):
    """Equal codes; any NaN for a NaN."""
    nan = want & 127 == 127
    assert (got[nan] & 127 == 127).all()
    np.testing.assert_array_equal(got[~nan], want[~nan])


def codes_on_gpu(codes, e, rows_per_scale=1):
    """Codes [rows][n] and exponents [rows][blocks] (numpy) as the products take them, and their
    values in float64."""
    s = np.full((e.shape[0], up(e.shape[1], 4)), 127, dtype=np.uint8)
    s[:, :e.shape[1]] = e + 127
    return (torch.from_numpy(codes).cuda().view(F8), torch.from_numpy(s).cuda(), o.held(codes, e, rows_per_scale))
