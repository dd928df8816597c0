"""The router's balance loss, its counts and its gradient against 64-bit definitions and differences."""
import numpy as np
import pytest
import torch

import expert_reference as eref
import mx4_reference as ref
from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200 import build

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
both = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


def _inputs(T, E, k, dtype, seed=0, masked=0.2, drop=0.2, pad=0, wild=False):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(T, E)) * 3
    x[rng.random((T, E)) < masked] = -np.inf
    if T > 3:
        x[1] = -np.inf
        x[2, E // 2] = np.nan
        x[3, 0] = np.inf
    base = torch.full((T, E + pad), 9.0, dtype=dtype, device=DEV)
    logits = base[:, pad // 2:pad // 2 + E]
    logits.copy_(torch.from_numpy(x))
    ids = rng.integers(0, E, (T, k))
    ids[rng.random(T) < drop] = -1
    ids[rng.random((T, k)) < 0.1] = -1
    if wild:
        ids = np.where(rng.random((T, k)) < 0.3, rng.integers(-2 ** 31, 2 ** 31, (T, k)), ids)
    return logits, torch.from_numpy(ids.astype(np.int32)).to(DEV)


def _check(got, want, bound, what):
    err = np.abs(got - want)
    assert np.all(err <= bound), f"{what}: worst {float((err / bound).max()):.3g} of the bound at {np.argwhere(err > bound)[:3].tolist()}"


def _both_ways(logits, ids, dtype, dloss=0.37, add=False):
    T, E = logits.shape
    k = ids.shape[1]
    x, idn = eref.f64(logits), ids.cpu().numpy()
    loss, counts, share = b.route_balance(logits, ids)
    wl, wc, ws, p, counted = ref.balance(x, idn)
    assert np.array_equal(counts.cpu().numpy(), wc)
    bs = ref.share_bound(x, ws, T, E)
    _check(eref.f64(share), ws, bs, "share")
    f = wc[:E] / (max(1, wc[E]) * k)
    _check(np.array(eref.f64(loss)), wl, E * float(f @ bs) + (E + 6) * ref.EPS24 * abs(wl) + 1e-37, "loss")
    scale = torch.tensor(dloss, device=DEV)
    other = (torch.randn((T, E), device=DEV) * 1e-3).to(dtype) if add else None
    d = b.route_balance_backward(logits, ids, counts, dloss=scale, add=other)
    on = eref.f64(other) if add else None
    want = ref.balance_gradient(p, counted, wc, k, float(scale)) + (on if add else 0.0)
    _check(eref.f64(d), want, ref.gradient_bound(x, p, wc, k, float(scale), dtype, on), "gradient")
    return loss, counts, share, d


SHAPES = [(1, 1, 1), (1, 8, 2), (5, 4, 4), (33, 7, 3), (128, 8, 2), (100, 60, 8), (700, 16, 1), (1000, 128, 8), (65, 257, 9), (2049, 33, 5), (300, 512, 4),
          (9, 1000, 32), (77, 1024, 6), (20011, 12, 2)]


@both
@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("pad", [0, 5], ids=["dense", "odd-pitch"])
def test_loss_counts_and_gradient(T, E, k, dtype, pad):
    logits, ids = _inputs(T, E, k, dtype, pad=pad)
    _both_ways(logits, ids, dtype, add=pad > 0)


@both
def test_choices_out_of_range_are_no_choices(dtype):
    for T, E, k in ((40, 20, 3), (5000, 64, 4)):
        logits, ids = _inputs(T, E, k, dtype, wild=True)
        _both_ways(logits, ids, dtype)


@both
def test_no_tokens_and_only_padding_tokens(dtype):
    for T in (0, 5, 3000):
        logits = torch.randn((T, 24), device=DEV).to(dtype)
        ids = torch.full((T, 2), -1, dtype=torch.int32, device=DEV)
        loss, counts, share = b.route_balance(logits, ids)
        assert float(loss) == 0 and int(counts.abs().sum()) == 0 and bool((share == 0).all())
        d = b.route_balance_backward(logits, ids, counts)
        assert d.shape == (T, 24) and bool((d == 0).all())
        other = torch.randn((T, 24), device=DEV).to(dtype)
        assert torch.equal(b.route_balance_backward(logits, ids, counts, add=other), other)


@both
def test_even_loads_give_one_and_one_expert_alone_gives_their_number(dtype):
    E, k = 16, 2
    ids = torch.arange(64 * k, device=DEV, dtype=torch.int32).view(64, k) % E
    loss, counts, share = b.route_balance(torch.zeros((64, E), dtype=dtype, device=DEV), ids)
    assert abs(float(loss) - 1.0) < 1e-6 and counts[:E].tolist() == [8] * E and int(counts[E]) == 64
    far = torch.full((64, E), -200.0, device=DEV).to(dtype)
    far[:, 3] = 0
    assert abs(float(b.route_balance(far, torch.full((64, 1), 3, dtype=torch.int32, device=DEV))[0]) - E) < 1e-5


def test_gradient_against_differences():
    """Central differences of the 64-bit loss at fixed choices: the step's own error is below 1e-8 of the loss."""
    logits, ids = _inputs(24, 10, 3, F32, masked=0.0, drop=0.3)
    logits[1:4] = torch.randn((3, 10), device=DEV)
    x, idn = eref.f64(logits), ids.cpu().numpy()
    counts = b.route_balance(logits, ids)[1]
    d = eref.f64(b.route_balance_backward(logits, ids, counts))
    h = 1e-5
    for t in range(24):
        for e in range(10):
            up, down = x.copy(), x.copy()
            up[t, e] += h
            down[t, e] -= h
            want = (ref.balance(up, idn)[0] - ref.balance(down, idn)[0]) / (2 * h)
            assert abs(d[t, e] - want) < 1e-8 + 1e-5 * abs(want), (t, e)


@both
def test_counts_of_several_batches(dtype):
    """Two batches with their counts summed have the gradient of both at once."""
    logits, ids = _inputs(600, 40, 4, dtype)
    counts = b.route_balance(logits, ids)[1]
    halves = [b.route_balance(logits[s], ids[s].contiguous())[1] for s in (slice(0, 250), slice(250, 600))]
    assert torch.equal(halves[0] + halves[1], counts)
    whole = b.route_balance_backward(logits, ids, counts)
    parts = [b.route_balance_backward(logits[s], ids[s].contiguous(), counts) for s in (slice(0, 250), slice(250, 600))]
    assert torch.equal(torch.cat(parts), whole)


@both
def test_outputs_given_in_place_equal_bits_streams_and_capture(dtype):
    for T, E in ((100, 8), (9000, 96)):
        logits, ids = _inputs(T, E, 2, dtype)
        loss, counts, share = b.route_balance(logits, ids)
        out = torch.empty((), device=DEV), torch.empty(E + 1, dtype=torch.int32, device=DEV), torch.empty(E, device=DEV)
        ws = torch.empty(b.route_balance_workspace_bytes(T, E) + 16, dtype=torch.uint8, device=DEV)
        again = b.route_balance(logits, ids, *out, workspace=ws)
        assert again[0] is out[0] and torch.equal(again[0], loss) and torch.equal(again[1], counts) and torch.equal(again[2], share)
        other = torch.randn((T, E), device=DEV).to(dtype)
        want = b.route_balance_backward(logits, ids, counts, add=other)
        assert b.route_balance_backward(logits, ids, counts, add=other, dlogits=other) is other and torch.equal(other, want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        l2, c2, s2 = b.route_balance(logits, ids, stream=side)
        d2 = b.route_balance_backward(logits, ids, c2, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(l2, loss) and torch.equal(d2, b.route_balance_backward(logits, ids, counts))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            l3, c3, s3 = b.route_balance(logits, ids)
            d3 = b.route_balance_backward(logits, ids, c3)
        logits.copy_(_inputs(T, E, 2, dtype, seed=9)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(l3, b.route_balance(logits, ids)[0]) and torch.equal(d3, b.route_balance_backward(logits, ids, c3))


@both
def test_every_access_stays_inside(dtype):
    with b.library(build.build_bounds_check()):
        b.bounds_report()
        for T, E, k in ((1, 1, 1), (33, 7, 3), (100, 60, 8), (65, 257, 9), (9, 1000, 32), (3000, 40, 2)):
            for pad in (0, 5):
                logits, ids = _inputs(T, E, k, dtype, pad=pad, wild=True)
                counts = b.route_balance(logits, ids)[1]
                b.route_balance_backward(logits, ids, counts, add=logits)
        rep = b.bounds_report()
    assert rep["violations"] == 0, rep
