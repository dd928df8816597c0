"""The memory that a call with `stream=` allocates belongs to that stream: what the caller's current stream allocates next never
shares it, and it is not reused there while the current stream may still read it.  The library calls are recorded and not
made, so that nothing runs on memory in doubt."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Recorder:
    """The library with its launching calls replaced by notes of the addresses they got."""

    def __init__(self, lib):
        self.lib, self.addresses = lib, set()

    def __getattr__(self, name):
        if name.endswith("_bytes") or name in ("dass_status_string",):
            return getattr(self.lib, name)

        def call(*args):
            self.addresses |= {a for a in args if isinstance(a, int) and a > 1 << 32}
            return b.OK
        return call


def _z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device=DEV)


T, K, E, D, N = 5000, 2, 8, 64, 96
CALLS = {
    "route_topk": lambda z, s: b.route_topk(z["logits"], K, stream=s),
    "route_topk_backward": lambda z, s: b.route_topk_backward(z["logits"], z["ids"], z["w"], stream=s),
    "expert_sort": lambda z, s: b.expert_sort(z["ids"], E, stream=s),
    "expert_gather": lambda z, s: b.expert_gather(z["X"], z["ids"], stream=s),
    "expert_combine": lambda z, s: b.expert_combine(z["Ys"], z["ids"], stream=s),
    "expert_combine_backward": lambda z, s: b.expert_combine_backward(z["X"], z["Ys"], z["ids"], stream=s),
    "linear": lambda z, s: b.linear(z["X"], z["W"], stream=s),
    "norm_finalize": lambda z, s: b.norm_finalize(z["sumsq"], stream=s),
    "score_nm": lambda z, s: b.score_nm(z["W"], z["norm"], b.AXIS_ROWS, 0.5, 2, 4, b.AXIS_ROWS, stream=s),
    "compress_nm": lambda z, s: b.compress_nm(z["W"], z["mask"], 2, 4, b.AXIS_ROWS, stream=s),
    "prune_nm": lambda z, s: b.prune_nm(z["W"], z["norm"], b.AXIS_ROWS, 0.5, 2, 4, b.AXIS_ROWS, stream=s),
    "select_unstructured": lambda z, s: b.select_unstructured(z["W"], z["norm"], b.AXIS_ROWS, 0.5, 0.5, b.AXIS_ROWS, stream=s),
    "feature_sumsq": lambda z, s: b.feature_sumsq(z["X"], stream=s),
    "mlp_forward": lambda z, s: b.mlp_forward(z["X"], z["W"], z["W"], z["Wd"], b.ACT_SILU, stream=s),
}


@pytest.fixture(scope="module")
def inputs():
    z = {"logits": _z(T, E), "ids": _z(T, K, dtype=torch.int32), "w": _z(T, K), "X": _z(T, D), "Ys": _z(T * K, D), "W": _z(N, D), "Wd": _z(D, N),
         "norm": _z(N), "sumsq": _z(N, dtype=torch.float64), "mask": _z(N, b.mask_words_per_row(D), dtype=torch.int32)}
    torch.cuda.synchronize()
    return z


def _spans(tensors):
    return [(t.untyped_storage().data_ptr(), t.untyped_storage().nbytes()) for t in tensors if t is not None]


def _tensors(out):
    return [] if out is None else [out] if isinstance(out, torch.Tensor) else [t for t in out if t is not None]


def _allocated_now(sizes):
    """Allocations of these sizes on the current stream, several of each, as (address, bytes); all held until the end."""
    kept = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(8)]
    return kept, [(t.data_ptr(), t.numel()) for t in kept]


def _recorded(monkeypatch, inputs, call, s):
    """The outputs of a call on s, and the addresses of all that it allocated."""
    own = {t.untyped_storage().data_ptr() for t in inputs.values()}
    rec = Recorder(b.load())
    monkeypatch.setattr(b, "load", lambda: rec)
    outs = _tensors(call(inputs, s))
    monkeypatch.undo()
    return outs, {a for a in rec.addresses if a not in own}


@pytest.mark.parametrize("name", CALLS)
def test_released_memory_stays_with_the_calls_stream(monkeypatch, inputs, name):
    outs, made = _recorded(monkeypatch, inputs, CALLS[name], torch.cuda.Stream())
    assert made, "the call allocated nothing"
    sizes = sorted({n for _, n in _spans(outs)} | {1 << 9, 1 << 12, 1 << 16})
    outs.clear()                                                       # the workspace is released already
    kept, now = _allocated_now(sizes)
    for a in made:
        assert not any(lo <= a < lo + n for lo, n in now), "memory of a call on another stream was handed to the current stream"


@pytest.mark.parametrize("name", CALLS)
def test_outputs_outlive_their_use_on_the_current_stream(monkeypatch, inputs, name):
    s = torch.cuda.Stream()
    outs, _ = _recorded(monkeypatch, inputs, CALLS[name], s)
    spans = _spans(outs)
    torch.cuda._sleep(100_000_000)                                     # tens of milliseconds of work on the current stream
    outs.clear()
    with torch.cuda.stream(s):
        again = [torch.empty(n, dtype=torch.uint8, device=DEV) for _, n in spans]
    for t in again:
        assert not any(lo <= t.data_ptr() < lo + n for lo, n in spans), "memory that the current stream may still read was reused"
    torch.cuda.synchronize()


def test_the_order_on_a_busy_stream_is_right(inputs):
    """The case in earnest: the call waits behind other work of its stream while the current stream allocates and writes."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    ids = torch.randint(0, 64, (20000, 4), generator=g, device=DEV, dtype=torch.int32)
    want = b.expert_sort(ids, 64)
    s = torch.cuda.Stream()
    need = b.expert_sort_workspace_bytes(20000, 4, 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
    got = b.expert_sort(ids, 64, stream=s)
    junk = [torch.full((need,), 0x7f, dtype=torch.uint8, device=DEV) for _ in range(200)]
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and len(junk) == 200


def test_sums_start_from_zero_on_the_calls_stream(monkeypatch, inputs):
    """feature_sumsq fills its sums itself: on the stream of the call, not on one that the call does not wait for."""
    s, where, ones = torch.cuda.Stream(), [], inputs["X"] + 1.0
    torch.cuda.synchronize()
    zeros = torch.Tensor.new_zeros
    monkeypatch.setattr(torch.Tensor, "new_zeros", lambda *a, **k: where.append(torch.cuda.current_stream()) or zeros(*a, **k))
    got = b.feature_sumsq(ones, stream=s)
    torch.cuda.synchronize()
    assert where == [s] and bool((got == T).all())
