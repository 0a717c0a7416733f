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
