"""How the 4-bit and balance calls make their outputs: what torch was asked to do with new memory is done, on the CPU."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2405_01943_b200 import binding as b


@pytest.fixture
def direct(monkeypatch):
    """The direct allocation, stood in for by one that shows in its values."""
    monkeypatch.setattr(b, "_cuda_empty", lambda shape, strides, dtype: torch.full(shape, 9.0, dtype=dtype))


def _made():
    return b._empty(torch.zeros(4), None, (3, 2), (2, 1), torch.float32)


def test_new_memory_is_filled_under_deterministic_algorithms(direct):
    assert bool((_made() == 9).all())                                  # the direct way, where nothing was asked for
    torch.use_deterministic_algorithms(True)
    try:
        assert bool(torch.isnan(_made()).all())                        # torch fills new memory with NaN
    finally:
        torch.use_deterministic_algorithms(False)
    assert bool((_made() == 9).all())


def test_a_dispatch_mode_sees_the_allocation(direct):
    seen = []

    class Mode(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(func)
            return func(*args, **(kwargs or {}))

    with Mode():
        out = _made()
    assert out.shape == (3, 2) and any("new_empty" in str(f) for f in seen)
