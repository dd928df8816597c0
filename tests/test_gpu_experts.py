"""The mixture-of-experts operators (router, sort by expert, rows in and out, gradients) against plain 64-bit definitions."""
import numpy as np
import pytest
import torch

import expert_reference as ref
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
both = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
INF = float("inf")


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed), device=DEV) * scale).to(dtype)


def _pitched(t, extra, lead=0, fill=float("nan")):
    """The same matrix inside a wider one, so that its pitch is not its length (what lies around it is NaN)."""
    base = torch.full((t.shape[0], lead + t.shape[1] + extra), fill, dtype=t.dtype, device=t.device)
    view = base[:, lead:lead + t.shape[1]]
    view.copy_(t)
    return view


def _logits(T, E, dtype, seed, special=True):
    x = torch.randn((T, E), generator=_gen(seed), device=DEV) * 2
    if special and E > 2:
        u = torch.rand((T, E), generator=_gen(seed + 1), device=DEV)
        x = torch.where(u < 0.2, x.round(), x)                       # ties
        x = torch.where(u > 0.93, torch.full_like(x, -INF), x)       # masked experts
        x = torch.where(u > 0.98, torch.full_like(x, float("nan")), x)
        low = float(torch.finfo(dtype).min)
        rows = [torch.full((E,), -INF), torch.full((E,), float("nan")), torch.full((E,), low), torch.zeros(E),
                torch.tensor([low] + [-INF] * (E - 1)), torch.tensor([-INF] * (E - 1) + [1.5]),
                torch.tensor([0.0, -0.0] * (E // 2) + [0.0] * (E % 2)), torch.tensor([-0.0, 0.0] * (E // 2) + [0.0] * (E % 2)),
                torch.tensor([1.0] * (E - 1) + [INF]), torch.tensor([INF] * E)]
        for i, r in enumerate(rows):
            if i < T - 1:
                x[i] = r.to(DEV)
    return x.to(dtype)


# ------------------------------------------------------------------------------------------------ router

ROUTE_SIZES = [(1, 1, 1), (1, 8, 2), (3, 7, 7), (13, 8, 1), (40, 5, 3), (33, 16, 4), (64, 33, 6), (130, 60, 8), (257, 64, 6),
               (100, 100, 32), (70, 128, 8), (31, 200, 8), (50, 256, 8), (19, 257, 9), (20, 500, 32), (17, 1000, 5), (12, 1024, 32)]


@both
@pytest.mark.parametrize("T,E,k", ROUTE_SIZES)
@pytest.mark.parametrize("over_all", [False, True], ids=["chosen", "all"])
@pytest.mark.parametrize("extra,lead", [(0, 0), (5, 3)], ids=["dense", "pitched"])
def test_route_forward_and_gradient(dtype, T, E, k, over_all, extra, lead):
    logits = _logits(T, E, dtype, seed=T * 7 + E)
    x = _pitched(logits, extra, lead) if extra else logits
    ids, w = b.route_topk(x, k, renormalise=not over_all)
    want_ids, want_w = ref.route(ref.f64(logits), k, over_all)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    rel = ref.route_weight_bound(ref.f64(logits), E)
    got = ref.f64(w)
    # below the smallest normal f32 a result may be flushed or rounded coarsely: an absolute 2^-126
    assert np.all(np.abs(got - want_w) <= rel * np.abs(want_w) + 2.0 ** -126)

    dw = _randn((T, k), F32, seed=3)
    dl = b.route_topk_backward(x, ids, dw, renormalise=not over_all)
    want = ref.route_gradient(ref.f64(logits), k, over_all, ref.f64(dw))
    # p (dw - s): p to rel; s a sum of k products of weights to rel and f32 sums; one rounding
    big = np.abs(ref.f64(dw)).max()
    _, p_any = ref.route(ref.f64(logits), E, over_all=True)
    bound = (2 * rel + (k + 4) * ref.EPS24) * 2 * big + ref.HALF_ULP[dtype] * np.abs(want) + 2.0 ** -120
    assert np.all(np.abs(ref.f64(dl) - want) <= bound)
    masked = ~(ref.f64(logits) > -np.inf)
    assert np.all(ref.f64(dl)[masked] == 0)


@pytest.mark.parametrize("over_all", [False, True], ids=["chosen", "all"])
def test_route_gradient_against_differences(over_all):
    T, E, k = 6, 12, 3
    logits = _logits(T, E, F32, seed=5, special=False)
    ids, _ = b.route_topk(logits, k, renormalise=not over_all)
    dw = _randn((T, k), F32, seed=6)
    dl = ref.f64(b.route_topk_backward(logits, ids, dw, renormalise=not over_all))
    x, chosen, g, h = ref.f64(logits), ids.cpu().numpy(), ref.f64(dw), 1e-5
    for t in range(T):
        for e in range(E):
            up, dn = x[t].copy(), x[t].copy()
            up[e] += h
            dn[e] -= h
            diff = ((ref.route_weights_of(up, chosen[t], over_all) - ref.route_weights_of(dn, chosen[t], over_all)) * g[t]).sum() / (2 * h)
            assert abs(dl[t, e] - diff) <= 1e-5 * max(1.0, np.abs(g[t]).max())     # h^2 of the difference, f32 of the kernel


def test_route_gradient_skips_ids_outside():
    logits = _logits(4, 16, F32, seed=8, special=False)
    ids = torch.tensor([[-1, -1], [16, 2], [3, -5], [1 << 30, -(1 << 31)]], dtype=torch.int32, device=DEV)
    for renorm in (True, False):
        dl = b.route_topk_backward(logits, ids, torch.ones(4, 2, device=DEV), renormalise=renorm)
        assert bool(torch.isfinite(dl).all())
        assert bool((dl[0] == 0).all()) and bool((dl[3] == 0).all())


def test_route_empty_and_refusals():
    empty = torch.empty((0, 8), device=DEV)
    ids, w = b.route_topk(empty, 2)
    assert ids.shape == (0, 2) and w.shape == (0, 2)
    assert b.route_topk_backward(empty, ids, w).shape == (0, 8)
    x = torch.zeros((4, 8), device=DEV)
    with pytest.raises(b.DassError):
        b.route_topk(x, 9)                                           # more than there are
    with pytest.raises(b.DassError):
        b.route_topk(x, 0)
    with pytest.raises(b.DassError):
        b.route_topk(torch.zeros((4, 1025), device=DEV), 2)
    with pytest.raises(b.DassError):
        b.route_topk(torch.zeros((4, 64), device=DEV), 33)
    with pytest.raises(TypeError):
        b.route_topk(x.double(), 2)
    with pytest.raises(ValueError):
        b.route_topk(x.t(), 2)
    with pytest.raises(ValueError):
        b.route_topk(x.cpu(), 2)
    with pytest.raises(ValueError):
        b.route_topk(x, 2, expert=torch.empty((4, 2), dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        b.route_topk_backward(x, torch.zeros((4, 2), dtype=torch.int32, device=DEV), torch.zeros((4, 3), device=DEV))


# ------------------------------------------------------------------------------------------------ order

SORT_SIZES = [(1, 1, 1), (1, 2, 8), (7, 3, 5), (100, 2, 8), (1000, 1, 1024), (682, 6, 64), (683, 6, 64), (4096, 1, 3), (4097, 1, 3),
              (5000, 4, 60), (3001, 32, 256), (20000, 8, 1000), (70001, 5, 17)]


def _sorted_matches(ids, E):
    offsets, slot, source = b.expert_sort(ids, E)
    flat = ids.cpu().numpy().reshape(-1).astype(np.int64)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    end = int((key < E).sum())
    want_slot = np.full(flat.size, -1, np.int32)
    want_slot[order[:end]] = np.arange(end)
    assert np.array_equal(offsets.cpu().numpy(), np.searchsorted(key[order], np.arange(E + 1)).astype(np.int32))
    assert np.array_equal(slot.cpu().numpy().reshape(-1), want_slot)
    assert np.array_equal(source.cpu().numpy(), np.concatenate([order[:end], np.full(flat.size - end, -1)]).astype(np.int32))
    return offsets, slot, source


@pytest.mark.parametrize("T,k,E", SORT_SIZES)
@pytest.mark.parametrize("kind", ["uniform", "skewed", "one", "dropped", "none", "wild"])
def test_expert_sort(T, k, E, kind):
    g = _gen(T + k + E)
    ids = torch.randint(0, E, (T, k), generator=g, device=DEV, dtype=torch.int32)
    u = torch.rand((T, k), generator=g, device=DEV)
    if kind == "skewed":
        ids = torch.where(u < 0.8, torch.full_like(ids, E - 1), ids)
    elif kind == "one":
        ids.fill_(E // 2)
    elif kind == "dropped":
        ids = torch.where(u < 0.5, torch.full_like(ids, -1), ids)
    elif kind == "none":
        ids.fill_(-1)
    elif kind == "wild":
        ids = torch.where(u < 0.2, torch.full_like(ids, E), torch.where(u < 0.4, torch.full_like(ids, -(1 << 31)), ids))
        ids = torch.where(u > 0.9, torch.full_like(ids, (1 << 31) - 1), ids)
    _sorted_matches(ids, E)


def test_expert_sort_matches_the_definition():
    ids = torch.randint(-1, 6, (50, 3), generator=_gen(1), device=DEV, dtype=torch.int32)
    for got, want in zip(b.expert_sort(ids, 5), ref.sort(ids.cpu().numpy(), 5)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_expert_sort_empty_and_refusals():
    offsets, slot, source = b.expert_sort(torch.empty((0, 2), dtype=torch.int32, device=DEV), 7)
    assert bool((offsets == 0).all()) and offsets.numel() == 8 and slot.shape == (0, 2) and source.numel() == 0
    ids = torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    for E in (0, 1025):
        with pytest.raises(b.DassError):
            b.expert_sort(ids, E)
    with pytest.raises(b.DassError):
        b.expert_sort(torch.zeros((4, 33), dtype=torch.int32, device=DEV), 8)
    with pytest.raises(ValueError):
        b.expert_sort(ids.long(), 8)
    with pytest.raises(ValueError):
        b.expert_sort(torch.zeros((2, 4), dtype=torch.int32, device=DEV).t(), 8)
    many = torch.zeros((5000, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(b.DassError):
        b.expert_sort(many, 8, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))


# ------------------------------------------------------------------------------------------------ rows

ROW_SIZES = [(1, 1, 1, 1), (1, 2, 8, 64), (5, 3, 4, 7), (33, 2, 8, 257), (64, 6, 60, 128), (300, 8, 16, 72), (17, 32, 64, 1000), (9, 5, 3, 4104)]
LAYOUTS = pytest.mark.parametrize("extra,lead", [(0, 0), (8, 8), (3, 1)], ids=["dense", "aligned", "odd"])


def _case(T, k, E, drop, seed):
    g = _gen(seed)
    ids = torch.randint(0, E, (T, k), generator=g, device=DEV, dtype=torch.int32)
    ids = torch.where(torch.rand((T, k), generator=g, device=DEV) < drop, torch.full_like(ids, -1), ids)
    if T > 3:
        ids[T // 2] = -1                                              # a token that no expert gets
    return ids, b.expert_sort(ids, E)


@both
@pytest.mark.parametrize("T,k,E,d", ROW_SIZES)
@pytest.mark.parametrize("drop", [0.0, 0.3, 1.0])
@LAYOUTS
def test_gather_and_its_gradient(dtype, T, k, E, d, drop, extra, lead):
    ids, (offsets, slot, source) = _case(T, k, E, drop, seed=T + d)
    X = _randn((T, d), dtype, 1)
    x = _pitched(X, extra, lead) if extra else X
    out = None
    if extra:
        base = torch.full((T * k, lead + d + extra), 7.0, dtype=dtype, device=DEV)
        out = base[:, lead:lead + d]
    Xs = b.expert_gather(x, slot, offsets, Xs=out)
    end = int(offsets[-1])
    want = torch.zeros((T * k, d), dtype=dtype, device=DEV)
    want[:end] = X[source[:end].long() // k]
    assert torch.equal(Xs, want)
    if extra:
        assert bool((base[:, :lead] == 7).all()) and bool((base[:, lead + d:] == 7).all())

    dXs = _randn((T * k, d), dtype, 2)
    dXs[end:] = float("nan")                                          # rows of no expert have no part
    g = _pitched(dXs, extra, lead) if extra else dXs
    dX = b.expert_gather_backward(g, slot)
    val, mag = ref.combine(ref.f64(dXs), slot.cpu().numpy(), None, None)
    assert np.all(np.abs(ref.f64(dX) - val) <= (k + 1) * ref.EPS24 * mag + ref.HALF_ULP[dtype] * (np.abs(val) + (k + 1) * ref.EPS24 * mag))


@both
@pytest.mark.parametrize("T,k,E,d", ROW_SIZES)
@pytest.mark.parametrize("with_residual", [False, True])
@LAYOUTS
def test_combine_and_its_gradient(dtype, T, k, E, d, with_residual, extra, lead):
    ids, (offsets, slot, _) = _case(T, k, E, 0.2, seed=T + d)
    end = int(offsets[-1])
    Ys, w = _randn((T * k, d), dtype, 1), torch.rand((T, k), generator=_gen(2), device=DEV)
    Ys[end:] = float("nan")
    w = torch.where(slot < 0, torch.full_like(w, float("nan")), w)    # the weights of dropped choices have no part
    R = _randn((T, d), dtype, 3) if with_residual else None
    pit = (lambda t: _pitched(t, extra, lead)) if extra else (lambda t: t)
    Y = b.expert_combine(pit(Ys), slot, w, residual=pit(R) if with_residual else None)
    s = slot.cpu().numpy()
    val, mag = ref.combine(ref.f64(Ys), s, ref.f64(w), ref.f64(R) if with_residual else None)
    f32 = (2 * k + 2) * ref.EPS24 * mag
    assert np.all(np.abs(ref.f64(Y) - val) <= f32 + ref.HALF_ULP[dtype] * (np.abs(val) + f32))
    if with_residual:                                                 # in place
        again = R.clone()
        b.expert_combine(pit(Ys), slot, w, residual=again, Y=again)
        assert torch.equal(again, Y)

    dY = _randn((T, d), dtype, 4)
    out = None
    if extra:
        base = torch.full((T * k, lead + d + extra), 7.0, dtype=dtype, device=DEV)
        out = base[:, lead:lead + d]
    dYs, dw = b.expert_combine_backward(pit(dY), pit(Ys), slot, w, offsets, dYs=out)
    want, want_w, mag_w = ref.combine_gradient(ref.f64(dY), ref.f64(Ys), s, ref.f64(w))
    assert np.all(np.abs(ref.f64(dYs) - want) <= (2 * ref.EPS24 + ref.HALF_ULP[dtype]) * np.abs(want))
    assert np.all(np.abs(ref.f64(dw) - want_w) <= (d + 2) * ref.EPS24 * mag_w)
    if extra:
        assert bool((base[:, :lead] == 7).all()) and bool((base[:, lead + d:] == 7).all())
    only_w = b.expert_combine_backward(pit(dY), pit(Ys), slot, w, want_rows=False)
    only_r = b.expert_combine_backward(pit(dY), pit(Ys), slot, w, offsets, want_weight=False)
    assert only_w[0] is None and torch.equal(only_w[1], dw) and only_r[1] is None and torch.equal(only_r[0], dYs)


def test_combine_gradient_against_differences():
    T, k, d = 4, 2, 6
    _, (offsets, slot, _) = _case(T, k, 3, 0.0, seed=3)
    Ys, w, dY = _randn((T * k, d), F32, 1), torch.rand((T, k), generator=_gen(2), device=DEV), _randn((T, d), F32, 4)
    dYs, dw = (ref.f64(v) for v in b.expert_combine_backward(dY, Ys, slot, w, offsets))
    s, y64, w64, g = slot.cpu().numpy(), ref.f64(Ys), ref.f64(w), ref.f64(dY)
    loss = lambda y, q: (ref.combine(y, s, q, None)[0] * g).sum()     # noqa: E731  (linear in each: the difference is exact but for rounding)
    for at in np.ndindex(T, k):
        q = w64.copy()
        q[at] += 1.0
        assert abs(loss(y64, q) - loss(y64, w64) - dw[at]) <= 1e-5
    for at in np.ndindex(T * k, d):
        y = y64.copy()
        y[at] += 1.0
        assert abs(loss(y, w64) - loss(y64, w64) - dYs[at]) <= 1e-5


def test_slots_outside_the_rows_are_skipped():
    X = _randn((4, 16), F32, 1)
    slot = torch.tensor([[0, 5], [-1, 6], [1 << 30, -(1 << 31)], [3, 2]], dtype=torch.int32, device=DEV)
    Xs = torch.full((6, 16), 9.0, device=DEV)
    b.expert_gather(X, slot, Xs=Xs)
    assert torch.equal(Xs[0], X[0]) and torch.equal(Xs[5], X[0]) and torch.equal(Xs[3], X[3]) and torch.equal(Xs[2], X[3])
    assert bool((Xs[1] == 9).all()) and bool((Xs[4] == 9).all())      # named by no slot, no offsets given: left alone
    Y = b.expert_combine(Xs, slot)
    assert torch.equal(Y[1], torch.zeros(16, device=DEV)) and torch.equal(Y[0], Xs[0] + Xs[5])
    dYs, dw = b.expert_combine_backward(X, Xs, slot, dYs=torch.full((6, 16), 9.0, device=DEV))
    assert bool((dYs[1] == 9).all()) and bool((dw[1] == 0).all()) and bool((dw[2] == 0).all())
    wild = torch.tensor([0, -7, 1 << 30], dtype=torch.int32, device=DEV)   # "rows used" beyond the rows, and negative
    b.expert_gather(X, slot, wild, Xs=Xs)
    b.expert_gather(X, torch.full_like(slot, -1), wild[:2].contiguous(), Xs=Xs)
    assert bool((Xs == 0).all())


def test_gather_with_weights_is_the_gradient_of_combine():
    _, (offsets, slot, _) = _case(40, 3, 8, 0.2, seed=9)
    dY, w = _randn((40, 72), BF16, 1), torch.rand((40, 3), generator=_gen(2), device=DEV)
    rows = b.expert_gather(dY, slot, offsets, weight=w)
    assert torch.equal(rows, b.expert_combine_backward(dY, rows, slot, w, offsets)[0])


def test_rows_without_tokens_and_refusals():
    none = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    X0 = torch.empty((0, 16), device=DEV)
    assert b.expert_gather(X0, none).shape == (0, 16)
    assert b.expert_combine(X0, none).shape == (0, 16)
    assert b.expert_combine_backward(X0, X0, none)[1].shape == (0, 2)
    Xs = torch.ones((5, 16), device=DEV)
    b.expert_gather(X0, none, torch.zeros(3, dtype=torch.int32, device=DEV), Xs=Xs)
    assert bool((Xs == 0).all())
    X, slot = torch.zeros((4, 16), device=DEV), torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    assert bool((b.expert_combine(X0, slot) == 0).all())              # no rows at all
    with pytest.raises(ValueError):
        b.expert_gather(X[:3], slot)
    with pytest.raises(ValueError):
        b.expert_gather(X, slot, Xs=torch.zeros((8, 15), device=DEV))
    with pytest.raises(ValueError):
        b.expert_gather(X, slot, Xs=torch.zeros((8, 16), device=DEV, dtype=BF16))
    with pytest.raises(ValueError):
        b.expert_gather(X.t(), torch.zeros((16, 2), dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        b.expert_combine(X, slot, weight=torch.zeros((4, 3), device=DEV))
    with pytest.raises(ValueError):
        b.expert_combine(X, slot, residual=torch.zeros((5, 16), device=DEV))
    with pytest.raises(TypeError):
        b.expert_gather(X.half(), slot)
    with pytest.raises(b.DassError):
        b.expert_combine_backward(X, X, slot, want_rows=False, want_weight=False)
    with pytest.raises(b.DassError):
        b.expert_gather(X, torch.zeros((4, 33), dtype=torch.int32, device=DEV))


def test_rows_past_32_bit_offsets():
    """Element offsets beyond 2^31 on the sorted side, the last rows checked."""
    rows, d = (1 << 31) // 4096 + 64, 4096
    Ys = torch.empty((rows, d), dtype=BF16, device=DEV)
    T = 32
    X = _randn((T, d), BF16, 1)
    slot = torch.arange(rows - T, rows, dtype=torch.int32, device=DEV).view(T, 1)
    b.expert_gather(X, slot, Xs=Ys)
    assert torch.equal(Ys[-T:], X)
    assert torch.equal(b.expert_combine(Ys, slot), X)


def test_another_stream_and_repeatable():
    s = torch.cuda.Stream()
    logits = _logits(5000, 64, BF16, seed=1)
    X = _randn((5000, 136), BF16, 2)
    torch.cuda.synchronize()

    def once(stream):
        ids, w = b.route_topk(logits, 6, stream=stream)
        offsets, slot, source = b.expert_sort(ids, 64, stream=stream)
        Xs = b.expert_gather(X, slot, offsets, stream=stream)
        Y = b.expert_combine(Xs, slot, w, stream=stream)
        dYs, dw = b.expert_combine_backward(X, Xs, slot, w, offsets, stream=stream)
        dl = b.route_topk_backward(logits, ids, dw, stream=stream)
        return ids, w, offsets, slot, source, Xs, Y, dYs, dw, dl

    here = once(None)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        there = once(s)
    s.synchronize()
    for p, q in zip(here, there):
        assert torch.equal(p, q)
