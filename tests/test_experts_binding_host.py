"""What the mixture-of-experts bindings refuse before they reach the library, on CPU tensors and stand-ins."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b

CPU = torch.device("cpu")


def test_rows_used_is_the_last_of_the_offsets():
    """The address of the number of rows in use: never one outside the tensor."""
    offsets = torch.zeros(5, dtype=torch.int32)
    assert b._rows_used(offsets, CPU) == offsets.data_ptr() + 16
    assert b._rows_used(offsets[:1], CPU) == offsets.data_ptr()
    assert b._rows_used(None, CPU) is None
    for bad in (offsets[:0], offsets.long(), offsets[::2], offsets.view(1, 5)):
        with pytest.raises(ValueError):
            b._rows_used(bad, CPU)


class OnDevice(torch.Tensor):
    """A tensor that passes for a CUDA tensor; the library below notes calls and makes none."""
    is_cuda = True

    def get_device(self):
        return 0


class Library:
    def __init__(self, lib):
        self.lib, self.calls = lib, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.lib, name)
        return lambda *args: self.calls.append(name) or b.OK


def _on_device(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def library(monkeypatch):
    lib = Library(b.load())
    monkeypatch.setattr(b, "load", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(b, "_stream", lambda stream: 0)
    return lib


def test_a_workspace_has_to_be_device_memory(library):
    calls = [lambda w: b.expert_sort(_on_device(5000, 2, dtype=torch.int32), 8, workspace=w), lambda w: b.feature_sumsq(_on_device(64, 32), workspace=w),
             lambda w: b.select_unstructured(_on_device(64, 32), _on_device(64), b.AXIS_ROWS, 0.5, 0.5, b.AXIS_ROWS, workspace=w)]
    for call in calls:
        library.calls.clear()
        call(_on_device(1 << 20, dtype=torch.uint8))
        assert len(library.calls) == 1
        for bad in (torch.zeros(1 << 20, dtype=torch.uint8), _on_device(1 << 20), _on_device(1 << 20, dtype=torch.uint8)[::2]):
            with pytest.raises(ValueError):
                call(bad)
        assert len(library.calls) == 1


class Stream:
    cuda_stream, device_index = 1 << 20, 1


def test_tensors_of_another_device_than_the_current_one(library, monkeypatch):
    """The library launches on the current device: a call with another device's tensors, or another device's stream, is refused."""
    ids, X, Ys, W = _on_device(4, 2, dtype=torch.int32), _on_device(4, 8), _on_device(8, 8), _on_device(8, 8)
    out = {n: _on_device(*shape, dtype=t) for n, shape, t in (("k", (4, 2), torch.float32), ("off", (9,), torch.int32), ("slot", (4, 2), torch.int32),
                                                              ("src", (8,), torch.int32), ("X", (4, 8), torch.float32), ("Ys", (8, 8), torch.float32))}
    calls = [lambda s: b.route_topk(X, 2, expert=ids, weight=out["k"], stream=s), lambda s: b.route_topk_backward(X, ids, out["k"], dlogits=out["X"], stream=s),
             lambda s: b.expert_sort(ids, 8, offsets=out["off"], slot=out["slot"], source=out["src"], stream=s),
             lambda s: b.expert_gather(X, ids, Xs=out["Ys"], stream=s), lambda s: b.expert_combine(Ys, ids, Y=out["X"], stream=s),
             lambda s: b.expert_combine_backward(X, Ys, ids, dYs=out["Ys"], dweight=out["k"], stream=s), lambda s: b.linear(X, W, Y=out["X"], stream=s)]
    older = [lambda: b.feature_sumsq(X), lambda: b.norm_finalize(_on_device(8, dtype=torch.float64)),
             lambda: b.score_nm(W, _on_device(8), b.AXIS_ROWS, 0.5, 2, 4, b.AXIS_ROWS)]
    for call in calls:
        call(None)
        with pytest.raises(ValueError):
            call(Stream())
    for call in older:
        call()
    made = len(library.calls)
    assert made == len(calls) + len(older)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError):
            call(None)
    for call in older:
        with pytest.raises(ValueError):
            call()
    assert len(library.calls) == made


def test_no_tokens_need_no_buffers():
    """T = 0 is a valid request: an empty tensor has no address."""
    lib = b.load()
    assert lib.dass_route_topk(None, 0, 8, 8, b.BF16, 2, b.ROUTE_CHOSEN, None, None, None) == b.OK
    assert lib.dass_route_topk_backward(None, 0, 8, 8, b.BF16, 2, b.ROUTE_ALL, None, None, None, 8, None) == b.OK
    assert lib.dass_expert_gather(None, 0, 16, 16, b.BF16, None, 2, None, None, None, 0, 16, None) == b.OK
    assert lib.dass_expert_combine(None, 0, 16, 16, b.BF16, None, 0, 2, None, None, 0, None, 16, None) == b.OK
    assert lib.dass_linear(None, 0, 64, 64, 1 << 20, None, 32, 64, 0, None, None, b.ACT_NONE, None, 0, None, 32, b.BF16, None, 1, None) == b.OK
    assert lib.dass_route_topk(None, 0, 8, 7, b.BF16, 2, b.ROUTE_CHOSEN, None, None, None) == 2     # sizes are still looked at
