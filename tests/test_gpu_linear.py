"""The matrix product with bias, activation, gating product and residual, dense and per expert, against 64 bits."""
import numpy as np
import pytest
import torch

import expert_reference as ref
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
both = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
ACTS = {"none": b.ACT_NONE, **b.ACT_BY_NAME}


def _randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _up8(n):
    return (n + 7) // 8 * 8


def _matrix(shape, dtype, seed, scale=1.0, pad=0, fill=float("nan")):
    """A matrix (or a stack of them) whose pitch is a multiple of 8 elements; the padding holds NaN."""
    ld = _up8(shape[-1]) + pad
    base = torch.full(shape[:-1] + (ld,), fill, dtype=dtype, device=DEV)
    view = base[..., :shape[-1]]
    view.copy_(_randn(shape, dtype, seed, scale))
    return view


def _check(Y, want, bound):
    err = np.abs(ref.f64(Y) - want)
    assert np.all(err <= bound), f"worst {float((err / bound).max()):.3g} of the bound at {np.unravel_index((err / bound).argmax(), err.shape)}"


OPTIONS = [dict(act="none"), dict(act="none", bias=True, residual=True), dict(act="gelu_tanh", bias=True), dict(act="silu", glu=True),
           dict(act="relu", glu=True, bias=True, residual=True), dict(act="silu", residual=True), dict(act="none", glu=True, bias=True)]


def _dense(T, K, N, dtype, act="none", bias=False, glu=False, residual=False, pad=0):
    X, W = _matrix((T, K), dtype, 1, pad=pad), _matrix((N, K), dtype, 2, K ** -0.5, pad=pad)
    V = _matrix((N, K), dtype, 3, K ** -0.5, pad=pad) if glu else None
    bw = _randn((N,), dtype, 4) if bias else None
    bv = _randn((N,), dtype, 5) if bias and glu else None
    R = _matrix((T, N), dtype, 6, pad=pad) if residual else None
    out = None
    if pad:
        base = torch.full((T, N + 5), 7.0, dtype=dtype, device=DEV)
        out = base[:, 2:2 + N]
    Y = b.linear(X, W, bias=bw, act=ACTS[act], W_up=V, bias_up=bv, residual=R, Y=out)
    c = lambda t: None if t is None else ref.f64(t)                   # noqa: E731
    want, bound = ref.linear(c(X), c(W), c(bw), act, c(V), c(bv), c(R), dtype)
    _check(Y, want, bound)
    if pad:
        assert bool((base[:, :2] == 7).all()) and bool((base[:, 2 + N:] == 7).all())
    b.linear_status()
    return X, W, V, bw, bv, R, Y


@both
@pytest.mark.parametrize("T,K,N", [(1, 8, 1), (1, 64, 33), (1, 1024, 4096), (2, 72, 128), (7, 520, 344), (16, 256, 688), (17, 264, 130),
                                   (33, 96, 257), (64, 200, 512), (65, 128, 127), (129, 72, 300), (300, 392, 520), (513, 64, 129)])
@pytest.mark.parametrize("options", OPTIONS, ids=lambda o: "-".join([o["act"]] + [k for k in o if k != "act"]))
def test_dense(T, K, N, dtype, options):
    _dense(T, K, N, dtype, **options)


@both
@pytest.mark.parametrize("T,K,N", [(1, 3, 5), (5, 70, 33), (40, 1001, 131), (260, 133, 390)])
def test_odd_lengths_pitches_and_an_output_off_alignment(T, K, N, dtype):
    _dense(T, K, N, dtype, act="silu", glu=True, bias=True, residual=True, pad=16)
    _dense(T, K, N, dtype, act="none", bias=True, residual=True, pad=8)


@both
@pytest.mark.parametrize("T,K,N", [(1, 12800, 264), (40, 12288, 200), (2100, 320, 1100), (1024, 2048, 520)])
def test_long_contractions_and_many_tiles(T, K, N, dtype):
    if dtype == F32 and T * K * N > 2 ** 30:
        pytest.skip("the 64-bit reference of one type is enough at this size")
    _dense(T, K, N, dtype, act="gelu_tanh", bias=True, residual=True)
    _dense(T, K, N, dtype, act="silu", glu=True)


def _grouped(counts, K, N, dtype, act="none", bias=False, glu=False, residual=False, tail=0, head=0, poison=True):
    G, n = len(counts), head + sum(counts) + tail
    edges = head + np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(edges, dtype=torch.int32, device=DEV)
    X = _matrix((n, K), dtype, 1)
    if poison:
        X[edges[-1]:] = float("nan")                                  # rows of no expert have no part
        X[:head] = float("inf")
    W = _matrix((G, N, K), dtype, 2, K ** -0.5)
    V = _matrix((G, N, K), dtype, 3, K ** -0.5) if glu else None
    bw = _randn((G, N), dtype, 4) if bias else None
    bv = _randn((G, N), dtype, 5) if bias and glu else None
    R = _randn((n, N), dtype, 6) if residual else None
    Y = b.linear(X, W, bias=bw, act=ACTS[act], W_up=V, bias_up=bv, residual=R, offsets=offsets)
    b.linear_status()
    c = lambda t, g=None: None if t is None else ref.f64(t if g is None else t[g])   # noqa: E731
    y = ref.f64(Y)
    assert np.all(y[:edges[0]] == 0) and np.all(y[edges[-1]:] == 0)
    for g in range(G):
        lo, hi = edges[g], edges[g + 1]
        if hi > lo:
            want, bound = ref.linear(c(X)[lo:hi], c(W, g), c(bw, g), act, c(V, g), c(bv, g), c(R)[lo:hi] if residual else None, dtype)
            _check(Y[lo:hi], want, bound)
    return X, W, V, bw, bv, R, offsets, Y


COUNTS = [[1], [0], [0, 0, 3], [5, 0, 1, 2], [1] * 9, [0, 40, 0, 7, 0], [130, 1, 0, 64, 3], [300, 0, 17, 260], [16] * 40, [0] * 70 + [2] + [0] * 30,
          [64, 65, 63, 128, 127, 129, 0, 256, 257]]


@both
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{sum(c)}")
@pytest.mark.parametrize("options", [dict(act="none"), dict(act="silu", glu=True), dict(act="gelu_tanh", glu=True, bias=True, residual=True),
                                     dict(act="relu", bias=True)], ids=["plain", "glu", "all", "relu"])
def test_per_expert(counts, dtype, options):
    _grouped(counts, 136, 200, dtype, **options)


@both
def test_per_expert_rows_of_no_expert(dtype):
    _grouped([3, 0, 5], 64, 72, dtype, act="silu", glu=True, tail=6)
    _grouped([30, 0, 500, 2], 64, 72, dtype, act="silu", glu=True, bias=True, residual=True, tail=300, head=3)
    _grouped([0, 0], 64, 72, dtype, tail=9)


@both
def test_per_expert_stack_that_is_not_contiguous(dtype):
    K, N = 64, 96
    big = _randn((3, 2, N, K), dtype, 1, K ** -0.5)
    offsets = torch.tensor([0, 4, 4, 10], dtype=torch.int32, device=DEV)
    X = _randn((10, K), dtype, 2)
    Y = b.linear(X, big[:, 0], act=b.ACT_SILU, W_up=big[:, 1], offsets=offsets)
    assert torch.equal(Y, b.linear(X, big[:, 0].contiguous(), act=b.ACT_SILU, W_up=big[:, 1].contiguous(), offsets=offsets))


@both
def test_offsets_that_lie_stay_inside(dtype):
    """Offsets that decrease or pass the rows: what is computed is unspecified, every access stays inside (the checked-access
    build looks at that too)."""
    X, W = _randn((50, 64), dtype, 1), _randn((3, 40, 64), dtype, 2)
    for o in ([0, 60, 20, 50], [5, 2, 90, 10], [-9, 1 << 30, -(1 << 31), (1 << 31) - 1], [50, 50, 50, 0]):
        b.linear(X, W, offsets=torch.tensor(o, dtype=torch.int32, device=DEV))
    b.linear_status()


@both
def test_in_place_on_the_residual_and_repeatable(dtype):
    for T in (3, 100, 700):
        X, W, V, bw, bv, R, Y = _dense(T, 136, 264, dtype, act="none", bias=True, residual=True)
        again = R.clone()
        b.linear(X, W, bias=bw, residual=again, Y=again)
        assert torch.equal(again, Y)
        assert torch.equal(b.linear(X, W, bias=bw, residual=R), Y)


def test_infinities_stay_in_their_rows():
    for T, dtype in ((4, BF16), (300, BF16), (40, F32)):
        X, W = _randn((T, 64), dtype, 1), _randn((72, 64), dtype, 2)
        Y = b.linear(X, W, act=b.ACT_SILU)
        X2 = X.clone()
        X2[1, 3], X2[2, 5] = float("inf"), float("nan")
        Y2 = b.linear(X2, W, act=b.ACT_SILU)
        keep = [t for t in range(T) if t not in (1, 2)]
        assert torch.equal(Y[keep], Y2[keep])
        assert not bool(torch.isfinite(Y2[2]).any())


def test_large_arguments_of_the_activations():
    W = torch.eye(8, device=DEV)
    X = torch.tensor([[-1e4, -100.0, -88.0, -20.0, 20.0, 88.0, 100.0, 1e4]], device=DEV)
    for dtype in (BF16, F32):
        for act in ("silu", "gelu_tanh", "relu"):
            Y = ref.f64(b.linear(X.to(dtype), W.to(dtype), act=ACTS[act]))
            with np.errstate(over="ignore"):
                want = ref.act(act, ref.f64(X.to(dtype)))
            assert np.all(np.isfinite(Y))
            assert np.all(np.abs(Y - want) <= 2.0 ** -8 * np.abs(want) + 1e-30)


@pytest.mark.parametrize("T", [2, 600])
def test_another_stream(T):
    s = torch.cuda.Stream()
    X, W = _randn((T, 512), BF16, 1), _randn((384, 512), BF16, 2)
    want = b.linear(X, W, act=b.ACT_SILU)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = b.linear(X, W, act=b.ACT_SILU, stream=s)
    s.synchronize()
    assert torch.equal(want, got)


def test_no_rows_and_refusals():
    X, W = torch.zeros((4, 64), device=DEV), torch.zeros((32, 64), device=DEV)
    assert b.linear(X[:0], W).shape == (0, 32)
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    stack = torch.zeros((2, 32, 64), device=DEV)
    assert b.linear(X[:0], stack, offsets=off).shape == (0, 32)
    bad = [dict(W=W[:, :60]), dict(W=W.to(BF16)), dict(W=W.t()), dict(W=stack), dict(bias=torch.zeros(31, device=DEV)), dict(W_up=W[:16]),
           dict(bias_up=torch.zeros(32, device=DEV)), dict(residual=torch.zeros((3, 32), device=DEV)), dict(Y=torch.zeros((4, 33), device=DEV)),
           dict(W=W.cpu()), dict(W=stack, offsets=off[:2].contiguous()), dict(W=stack, offsets=off.long())]
    for kw in bad:
        with pytest.raises(ValueError):
            b.linear(X, **{"W": W, **kw})
    with pytest.raises(TypeError):
        b.linear(X.half(), W.half())
    with pytest.raises(b.DassError):                                  # a pitch that is not whole 16 bytes
        b.linear(torch.zeros((4, 66), device=DEV)[:, :64], W)
    with pytest.raises(b.DassError):                                  # a base that is not 16-byte aligned
        b.linear(torch.zeros((4, 68), device=DEV)[:, 1:65], W)
    with pytest.raises(b.DassError):
        b.linear(X, W, act=9)
