"""Helpers of the tests of the operators around the layer: inputs of both types as the device
holds them, outputs between guard bands, and the rounding-error bound they are held to."""
import numpy as np
import torch

from oracle import bf16

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
PAD = 64  # guard elements on each side of an output


def stored(a, dt):
    """float64 array -> (device tensor of type dt, the float64 values it holds)."""
    a = np.ascontiguousarray(a, dtype=np.float32)
    if dt == "f32":
        return torch.from_numpy(a).cuda(), a.astype(np.float64)
    bits = bf16.to_bf16_bits(a.astype(np.float64))
    return (torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16),
            bf16.from_bf16_bits(bits).astype(np.float64))


def f32(a):
    """float64 array (or None) -> (fp32 device tensor, its values)."""
    return (None, None) if a is None else stored(a, "f32")


def shifted(t, by=1):
    """The same values, contiguous, `by` elements into a larger buffer (element alignment only)."""
    if t is None:
        return None
    big = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    v = big[by:].view(t.shape)
    v.copy_(t)
    return v


class Out:
    """An output tensor filled with a sentinel, between sentinel bands of PAD + `by` elements."""

    def __init__(self, shape, dtype, by=0):
        n = int(np.prod(shape))
        self.raw = torch.full((n + 2 * PAD + by,), -77, dtype=dtype, device="cuda")
        self.at = PAD + by
        self.t = self.raw[self.at:self.at + n].view(shape)

    def values(self):
        """On the host in float64, after checking the bands."""
        n = self.t.numel()
        assert (self.raw[:self.at] == -77).all() and (self.raw[self.at + n:] == -77).all(), "written out of bounds"
        return self.t.detach().cpu().double().numpy()


U32, U_BF16 = 2.0 ** -24, 2.0 ** -8  # half a unit in the last of 24 and of 8 significant bits, at worst


def assert_rounded(got, ref, scale, dt, terms, name=""):
    """|got - ref| within what `terms` fp32 roundings of terms of total magnitude `scale` can add
    up to, and one rounding to dt."""
    tol = terms * U32 * np.asarray(scale) + 1e-37
    if dt == "bf16":
        tol = tol + U_BF16 * (np.abs(ref) + tol)
    err = np.abs(np.asarray(got) - ref)
    bad = ~(err <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, err / tol, 0)), err.shape)
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} out of bounds; at {i} got {np.asarray(got)[i]} "
                             f"want {np.asarray(ref)[i]} tolerance {np.asarray(tol)[i]}")


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
