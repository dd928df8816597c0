"""How the 4-bit and balance calls make their outputs: what torch was asked to do with new memory is done, and buffers have the
sizes that the library fills, on the CPU."""
import ctypes

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200 import build


@pytest.fixture
def direct(monkeypatch):
    """The direct allocation, stood in for by one that shows in its values."""
    monkeypatch.setattr(b, "_cuda_empty", lambda shape, strides, dtype: torch.full(shape, 9.0, dtype=dtype))


def _made():
    return b._maker(torch.zeros(4), None)((3, 2), (2, 1), torch.float32)


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


class _Device(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 0


@pytest.mark.parametrize("dims", [2, 3])
@pytest.mark.parametrize("rows,K", [(0, 1), (1, 1), (1, 4096), (127, 31), (128, 32), (128, 128), (129, 129), (3, 33), (300, 257)])
def test_quantisation_allocates_what_the_library_fills(monkeypatch, dims, rows, K):
    build.build()
    lib, calls = b.load(), []

    class Library:
        def __getattr__(self, name):
            return getattr(lib, name) if name.endswith("_bytes") else lambda *a: calls.append(a) or b.OK

    monkeypatch.setattr(b, "load", lambda: Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    G = 3 if dims == 3 else 1
    codes, scales = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.dass_mx4_bytes(rows, K, ctypes.byref(codes), ctypes.byref(scales)) == b.OK
    X = torch.zeros(((G,) if dims == 3 else ()) + (rows, K), dtype=torch.bfloat16)
    for direct in (True, False):                                       # both ways to allocate: a plain tensor takes the direct one
        asked = []

        def empty(shape, strides, dtype):
            asked.append(shape)
            out = torch.empty_strided(shape, strides, dtype=dtype)
            assert out.is_contiguous()
            return out.as_subclass(_Device)

        monkeypatch.setattr(b, "_cuda_empty", empty)
        x = X.as_subclass(_Device)
        with monkeypatch.context() as m:
            if direct:
                m.setattr(b, "_maker", lambda t, stream: empty)
            q = b.mx4_quantize(x)
        assert bool(asked) == direct
        assert q.codes.numel() == G * codes.value and q.scales.numel() == G * scales.value and q.shape == X.shape
        assert q.codes.is_contiguous() and q.scales.is_contiguous()
        assert b._mx4(q, "q", 0) == (q.codes.data_ptr(), q.scales.data_ptr())
        if rows:
            assert calls[-1][7:9] == (q.codes.data_ptr(), q.scales.data_ptr())
