"""Microscaled 4-bit values on the device: quantisation and back bit for bit, the product against 64 bits."""
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
ACTS = {"none": b.ACT_NONE, **b.ACT_BY_NAME}


def _same_values(got, want):
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


def _check_quantize(X, Q):
    rows, K = X.shape
    codes, scales = ref.quantize(eref.f64(X))
    got = ref.unpack(Q.codes.cpu().numpy())
    assert np.array_equal(Q.scales.cpu().numpy(), ref.tile(scales)), "scales"
    same = (got == codes) | ((got & 7) + (codes & 7) == 0)             # the sign of a zero is free
    assert same.all(), np.argwhere(~same)[:4]
    want = ref.values(codes, scales)[:, :K]
    for dtype in (BF16, F32):
        _same_values(eref.f64(b.mx4_dequantize(Q, dtype)), want)


def _rows(rows, K, dtype, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((rows, K), generator=g, device=DEV) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g, device=DEV).float())
    return x.to(dtype)


@both
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (3, 31), (1, 4096), (127, 33), (128, 128), (129, 129), (5, 257), (300, 1001), (257, 512), (64, 14336)])
def test_quantize(rows, K, dtype):
    X = _rows(rows, K, dtype)
    _check_quantize(X, b.mx4_quantize(X))


@both
def test_quantize_every_middle_and_extreme(dtype):
    """All numbers half way between codes at every scale that occurs, their neighbours, and the ends of the type's range."""
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0])
    rows = []
    for e in list(range(-133, -120)) + [-30, -1, 0, 1, 40, 123, 124, 125]:
        for sign in (1.0, -1.0):
            row = sign * torch.ldexp(torch.cat((mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -7))).double(), torch.tensor(e)).float()
            rows.append(torch.cat((row, torch.ldexp(torch.tensor([4.0, 0.1]).double(), torch.tensor(e)).float())))
    X = torch.stack(rows).to(dtype).to(DEV)
    big = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_normal
    extra = torch.zeros((6, 32), dtype=dtype, device=DEV)
    extra[0, 3], extra[1, :2], extra[2, 0], extra[3, 5], extra[4, 31] = big, torch.tensor([big, -big / 3]), tiny, tiny / 4, -big
    extra[5, 1] = -0.0
    X = torch.cat((X, extra))
    assert X.shape[1] == 32
    _check_quantize(X, b.mx4_quantize(X))


@both
def test_quantize_blocks_with_nan_or_infinity_become_nan_alone(dtype):
    X = _rows(9, 160, dtype)
    X[1, 33], X[2, 159], X[3, 0], X[4, 64:96] = float("nan"), float("inf"), float("-inf"), float("nan")
    Q = b.mx4_quantize(X)
    _check_quantize(X, Q)
    assert int(torch.isnan(b.mx4_dequantize(Q)).sum()) == 4 * 32


@both
@pytest.mark.parametrize("rows,K", [(7, 96), (130, 250)])
def test_quantize_strides_offsets_and_stacks(rows, K, dtype):
    base = _rows(rows, K + 21, dtype)
    for X in (base[:, 3:3 + K], base[:, 8:8 + K], base[::2, :K]):
        _check_quantize(X, b.mx4_quantize(X))
    S = torch.stack([_rows(rows, K, dtype, seed=s) for s in range(3)])
    Q = b.mx4_quantize(S)
    wide = torch.empty((3, rows, K + 9), dtype=dtype, device=DEV)[:, :, 1:1 + K]
    wide.copy_(S)
    Q2 = b.mx4_quantize(wide)
    assert torch.equal(Q.codes, Q2.codes) and torch.equal(Q.scales, Q2.scales)
    out = torch.full((3, rows + 1, K + 2), 7.0, dtype=dtype, device=DEV)
    b.mx4_dequantize(Q, dtype, out=out[:, :rows, 1:1 + K])
    assert bool((out[:, rows] == 7).all()) and bool((out[:, :, 0] == 7).all()) and bool((out[:, :, K + 1:] == 7).all())
    for g in range(3):
        _check_quantize(S[g], b.MX4(Q.codes[g], Q.scales[g], K))
        assert torch.equal(out[g, :rows, 1:1 + K], b.mx4_dequantize(b.MX4(Q.codes[g], Q.scales[g], K), dtype))


def _nearest(x):
    """Rows [n x 32 b] of doubles rounded to 4 bits and back, on the device (for sizes that numpy is slow at)."""
    blocks = x.view(len(x), -1, 32)
    scale = torch.ldexp(torch.ones_like(blocks[:, :, :1]), (torch.frexp(blocks.abs().amax(2, keepdim=True)).exponent - 3).clamp_min(-127))
    y = (blocks / scale).abs().clamp_max(6.0)
    step = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0))
    return (torch.round(y / step) * step * blocks.sign() * scale).view_as(x)       # half to even is the even code: steps are its last bit


@both
@pytest.mark.parametrize("groups,rows,K", [(1, 1100077, 32), (70001, 3, 64), (3, 40000, 96)])
def test_more_rows_and_matrices_than_a_grid_has_places(groups, rows, K, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    X = torch.randn((groups, rows, K), generator=g, device=DEV).to(dtype)
    X = X[0] if groups == 1 else X
    Q = b.mx4_quantize(X)
    got = b.mx4_dequantize(Q, dtype)
    assert torch.equal(got.view(-1, K).double(), _nearest(X.view(-1, K).double()))
    if groups > 1:
        last = b.mx4_quantize(X[-1])
        assert torch.equal(Q.codes[-1], last.codes) and torch.equal(Q.scales[-1], last.scales)


def test_every_code_and_scale():
    """All 16 codes under all 256 scales: exact, infinite only where the value passes bf16's range, NaN for scale 255."""
    codes = np.tile(np.arange(32, dtype=np.uint8) % 16, (256, 1))
    scales = np.arange(256, dtype=np.uint8)[:, None]
    Q = b.MX4(torch.from_numpy(ref.pack(codes)).to(DEV), torch.from_numpy(ref.tile(scales)).to(DEV), 32)
    want = ref.values(codes, scales)
    for dtype in (BF16, F32):
        top = float(torch.finfo(dtype).max)
        _same_values(eref.f64(b.mx4_dequantize(Q, dtype)), np.where(np.abs(want) > top, np.copysign(np.inf, want), want))


def test_no_rows():
    Q = b.mx4_quantize(torch.empty((0, 70), dtype=BF16, device=DEV))
    assert Q.shape == (0, 70) and b.mx4_dequantize(Q).shape == (0, 70)
    W = b.mx4_quantize(_rows(5, 70, BF16))
    assert b.linear_mx4(Q, W).shape == (0, 5) and b.linear_mx4(torch.empty((0, 72), dtype=BF16, device=DEV)[:, :70], W).shape == (0, 5)


# ------------------------------------------------------------------ product
def _mx4(rng, rows, K, low=118, high=124):
    codes, scales, v = ref.random_mx4(rng, rows, K, low, high)
    return b.MX4(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), K), v


def _mx4_stack(rng, G, rows, K):
    parts = [ref.random_mx4(rng, rows, K) for _ in range(G)]
    return b.MX4(torch.from_numpy(np.stack([p[0] for p in parts])).to(DEV), torch.from_numpy(np.stack([p[1] for p in parts])).to(DEV), K), [p[2] for p in parts]


def _randn(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(BF16)


def _pitched(shape, seed):
    """bf16 rows of a pitch of whole 16 bytes whose padding is NaN."""
    base = torch.full((*shape[:-1], (shape[-1] + 7) // 8 * 8 + 8), float("nan"), dtype=BF16, device=DEV)
    base[..., :shape[-1]] = _randn(shape, seed)
    return base[..., :shape[-1]]


def _check(Y, want, bound):
    err = np.abs(eref.f64(Y) - want)
    assert np.all(err <= bound), f"worst {float(np.nanmax(err / bound)):.3g} of the bound at {np.argwhere(~(err <= bound))[:3].tolist()}"


def _dense(T, K, N, both4, act="none", bias=False, glu=False, residual=False, odd=False):
    rng = np.random.default_rng(T * 7919 + K * 31 + N)
    if both4:
        X, x = _mx4(rng, T, K, 125, 129)
    else:
        X = _pitched((T, K), 1)
        x = eref.f64(X)
    W, w = _mx4(rng, N, K)
    V, v = _mx4(rng, N, K) if glu else (None, None)
    bw, bv = (_randn((N,), 4) if bias else None), (_randn((N,), 5) if bias and glu else None)
    R = _pitched((T, N), 6) if residual else None
    out = None
    if odd:
        base = torch.full((T, N + 5), 7.0, dtype=BF16, device=DEV)
        out = base[:, 2:2 + N]
    Y = b.linear_mx4(X, W, bias=bw, act=ACTS[act], W_up=V, bias_up=bv, residual=R, Y=out)
    b.linear_status()
    c = lambda t: None if t is None else eref.f64(t)                   # noqa: E731
    _check(Y, *eref.linear(x, w, c(bw), act, v, c(bv), c(R), BF16))
    if odd:
        assert bool((base[:, :2] == 7).all()) and bool((base[:, 2 + N:] == 7).all())
    return X, W, V, bw, bv, R, Y


OPTIONS = [dict(act="none"), dict(act="none", bias=True, residual=True), dict(act="gelu_tanh", bias=True), dict(act="silu", glu=True),
           dict(act="relu", glu=True, bias=True, residual=True)]
forms = pytest.mark.parametrize("both4", [False, True], ids=["bf16-rows", "4-bit-rows"])
options = pytest.mark.parametrize("options", OPTIONS, ids=lambda o: "-".join([o["act"]] + [k for k in o if k != "act"]))


@forms
@options
@pytest.mark.parametrize("T,K,N", [(1, 8, 1), (1, 1024, 4096), (2, 72, 128), (7, 520, 344), (8, 4096, 256), (9, 31, 33), (16, 256, 688), (17, 264, 130),
                                   (33, 96, 257), (64, 200, 512), (65, 128, 127), (100, 1024, 200), (129, 72, 300), (300, 392, 520), (513, 64, 129)])
def test_dense(T, K, N, both4, options):
    _dense(T, K, N, both4, **options)


def _on_device(X, W, V, bias, bias_up, R, act, rows16):
    """eref.linear on the device, for weights of a realistic size: (value, bound).  Rows that were split into 4-bit ones carry
    2^-24 of the largest value of their block of 32 at every k."""
    v = lambda q: b.mx4_dequantize(q, F32).double()                    # noqa: E731
    x = v(X) if isinstance(X, b.MX4) else X.double()
    K, eps = x.shape[1], eref.EPS24
    lost = torch.zeros_like(x)
    if rows16:
        pad = torch.nn.functional.pad(x.abs(), (0, -K % 32)).view(len(x), -1, 32)
        lost = (2.0 ** -24 * pad.amax(2, keepdim=True)).expand_as(pad).reshape(len(x), -1)[:, :K]

    def product(q, bb):
        w = v(q)
        add = 0.0 if bb is None else bb.double()
        p = x @ w.t() + add
        return p, (K + 1) * 2 * eps * (x.abs() @ w.abs().t() + abs(add)) + lost @ w.abs().t() + (0 if not rows16 else 12 * eps * (x.abs() @ w.abs().t()))

    p, ep = product(W, bias)
    y = {"none": lambda t: t, "silu": lambda t: t * torch.sigmoid(t)}[act](p)
    e = ep if act == "none" else 1.13 * ep + 2.0 ** -19 * p.abs()
    if V is not None:
        u, eu = product(V, bias_up)
        e = e * (u.abs() + eu) + y.abs() * eu + 2 * eps * (y * u).abs()
        y = y * u
    if R is not None:
        y = y + R.double()
        e = e + 2 * eps * y.abs()
    return y, e + eref.HALF_ULP[BF16] * (y.abs() + e) + 1e-37


def _normal_mx4(N, K, seed):
    return b.mx4_quantize(_randn((N, K), seed, 0.02))


@forms
@pytest.mark.parametrize("T,K,N,glu", [(1, 4096, 14336, True), (5, 4096, 14336, True), (12, 4096, 14300, True), (3, 8192, 9001, False), (9, 8200, 8192, False),
                                       (40, 4096, 14336, True), (130, 4096, 14336, True), (300, 4096, 4096, False), (900, 1032, 4001, True)])
def test_weights_that_are_the_time(T, K, N, glu, both4):
    X = _pitched((T, K), 1)
    X[:, 7] *= 300                                                     # a channel that its neighbours' block has to live with
    rows16 = not both4 and b.linear_mx4_workspace_bytes(T, K, N, has_up=glu) > 0
    X = b.mx4_quantize(X) if both4 else X
    W, V = _normal_mx4(N, K, 2), _normal_mx4(N, K, 3) if glu else None
    bias, bias_up, R = _randn((N,), 4), _randn((N,), 5) if glu else None, _randn((T, N + 3), 6)[:, 1:1 + N]
    act = "silu" if glu else "none"
    Y = b.linear_mx4(X, W, bias=bias, act=ACTS[act], W_up=V, bias_up=bias_up, residual=R)
    again = b.linear_mx4(X, W, bias=bias, act=ACTS[act], W_up=V, bias_up=bias_up, residual=R)
    b.linear_status()
    assert torch.equal(Y, again)
    want, bound = _on_device(X, W, V, bias, bias_up, R, act, rows16)
    err = (Y.double() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())


@forms
@pytest.mark.parametrize("counts", [[4, 0, 1, 9, 3, 12, 2, 1], [0, 25, 0, 0, 31, 0, 0, 3], [64, 1, 0, 90, 130, 12, 300, 8]], ids=lambda c: str(sum(c)))
@pytest.mark.parametrize("K,N,glu", [(2048, 7168, True), (7168, 2050, False)])
def test_experts_of_a_size(counts, K, N, glu, both4):
    G, n = len(counts), sum(counts) + 3
    edges = np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(edges, dtype=torch.int32, device=DEV)
    X = _pitched((n, K), 1)
    X[-3:] = float("nan")
    rows16 = not both4 and b.linear_mx4_workspace_bytes(n, K, N, G, True, glu) > 0
    X = b.mx4_quantize(X) if both4 else X
    stack = lambda seed: [_normal_mx4(N, K, seed + g) for g in range(G)]                                            # noqa: E731
    join = lambda q: b.MX4(torch.stack([m.codes for m in q]), torch.stack([m.scales for m in q]), K)                # noqa: E731
    W, V = stack(10), stack(30) if glu else None
    bias, R = _randn((G, N), 4), _randn((n, N), 6)
    act = "silu" if glu else "none"
    Y = b.linear_mx4(X, join(W), bias=bias, act=ACTS[act], W_up=join(V) if glu else None, residual=R, offsets=offsets)
    b.linear_status()
    assert bool((Y[-3:] == 0).all())
    whole = b.mx4_dequantize(X, F32) if both4 else None
    for g in range(G):
        lo, hi = edges[g], edges[g + 1]
        if hi > lo:
            rows = b.mx4_quantize(whole[lo:hi]) if both4 else X[lo:hi]  # values that are in 4 bits stay what they are
            want, bound = _on_device(rows, W[g], V[g] if glu else None, bias[g], None, R[lo:hi], act, rows16)
            err = (Y[lo:hi].double() - want).abs()
            assert bool((err <= bound).all()), (g, float((err / bound).max()))


def test_nan_and_infinity_in_rows_that_are_split():
    X = _randn((3, 4096), 1)
    W = _normal_mx4(14336, 4096, 2)
    assert b.linear_mx4_workspace_bytes(3, 4096, 14336, has_up=True) > 0
    X[1, 100], X[2, 4095] = float("nan"), float("inf")
    Y = b.linear_mx4(X, W, W_up=W)
    assert bool(torch.isfinite(Y[0]).all()) and not bool(torch.isfinite(Y[1:]).any())


def test_values_at_the_end_of_the_range_in_rows_that_are_split():
    X = _randn((2, 4096), 1)
    X[0, 5], X[0, 700], X[1, 33] = 3.38e38, -3.2e38, 2.0 ** -133
    W = b.mx4_quantize(_randn((14336, 4096), 2, 2.0 ** -20))
    assert b.linear_mx4_workspace_bytes(2, 4096, 14336, has_up=True) > 0
    ones = torch.zeros((14336, 4096), dtype=BF16, device=DEV)          # the gate: relu(1 * x[7]) is x[7]
    X[:, 7], ones[:, 7] = 1.0, 1.0
    Y = b.linear_mx4(X, b.mx4_quantize(ones), act=b.ACT_RELU, W_up=W)
    x, w = X.double(), b.mx4_dequantize(W, F32).double()
    want = x @ w.t()
    amax = x.abs().view(2, 128, 32).amax(2, keepdim=True).expand(2, 128, 32).reshape(2, 4096)
    bound = (4097 + 12) * 2 * eref.EPS24 * (x.abs() @ w.abs().t()) + 2.0 ** -22 * (amax @ w.abs().t())      # the range's end costs a bit of the 24
    bound = bound * 1.01 + 2.0 ** -8 * want.abs()
    assert bool(torch.isfinite(Y).all()) and bool(((Y.double() - want).abs() <= bound).all())


@forms
@pytest.mark.parametrize("T,K,N", [(1, 3, 5), (5, 70, 33), (40, 1001, 131), (260, 133, 390)])
def test_odd_lengths_and_an_output_off_alignment(T, K, N, both4):
    _dense(T, K, N, both4, act="silu", glu=True, bias=True, residual=True, odd=True)
    _dense(T, K, N, both4, act="none", bias=True, residual=True, odd=True)


@forms
@pytest.mark.parametrize("T,K,N", [(1, 12800, 264), (40, 12288, 200), (2100, 320, 1100), (1024, 2048, 520)])
def test_long_contractions_and_many_tiles(T, K, N, both4):
    _dense(T, K, N, both4, act="gelu_tanh", bias=True, residual=True)
    _dense(T, K, N, both4, act="silu", glu=True)


COUNTS = [[1], [0], [0, 0, 3], [5, 0, 1, 2], [1] * 9, [0, 40, 0, 7, 0], [130, 1, 0, 64, 3], [300, 0, 17, 260], [16] * 40, [0] * 70 + [2] + [0] * 30,
          [64, 65, 63, 128, 127, 129, 0, 256, 257]]


@forms
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{sum(c)}")
@pytest.mark.parametrize("options", [dict(act="none"), dict(act="gelu_tanh", glu=True, bias=True, residual=True)], ids=["plain", "all"])
@pytest.mark.parametrize("K,N", [(136, 72), (512, 300)])
@pytest.mark.parametrize("head,tail", [(0, 0), (3, 5)])
def test_per_expert(counts, K, N, both4, options, head, tail):
    """Rows of no expert give zeros, whatever they hold; every other row meets its expert's weights alone."""
    G, n = len(counts), head + sum(counts) + tail
    if n == 0:
        n = tail = 1
    act, glu, bias, residual = options["act"], *(options.get(o, False) for o in ("glu", "bias", "residual"))
    rng = np.random.default_rng(G * 100 + n)
    edges = head + np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(edges, dtype=torch.int32, device=DEV)
    X = _pitched((n, K), 1)
    X[:head], X[edges[-1]:] = float("inf"), float("nan")
    if both4:
        X = b.mx4_quantize(X)
        x = ref.values(*ref.quantize(eref.f64(b.mx4_dequantize(X, F32))))[:, :K]
    else:
        x = eref.f64(X)
    W, w = _mx4_stack(rng, G, N, K)
    V, v = _mx4_stack(rng, G, N, K) if glu else (None, [None] * G)
    bw, bv = (_randn((G, N), 4) if bias else None), (_randn((G, N), 5) if bias and glu else None)
    R = _randn((n, N), 6) if residual else None
    Y = b.linear_mx4(X, W, bias=bw, act=ACTS[act], W_up=V, bias_up=bv, residual=R, offsets=offsets)
    b.linear_status()
    y = eref.f64(Y)
    assert np.all(y[:edges[0]] == 0) and np.all(y[edges[-1]:] == 0)
    c = lambda t, g: None if t is None else eref.f64(t[g])             # noqa: E731
    for g in range(G):
        lo, hi = edges[g], edges[g + 1]
        if hi > lo:
            _check(Y[lo:hi], *eref.linear(x[lo:hi], w[g], c(bw, g), act, v[g], c(bv, g), None if R is None else eref.f64(R[lo:hi]), BF16))


@forms
@pytest.mark.parametrize("T,K,N", [(4, 160, 48), (50, 160, 300), (300, 160, 300)])
def test_offsets_are_not_trusted(T, K, N, both4):
    """Offsets that decrease or leave the rows: no row outside is touched, and the call ends."""
    rng = np.random.default_rng(3)
    W, _ = _mx4_stack(rng, 3, N, K)
    X = _mx4(rng, T, K)[0] if both4 else _randn((T, K), 1)
    for edges in ([-5, 2, 1, T + 90], [T, 0, T, 0], [2 ** 31 - 1, -2 ** 31, 0, 3], [0, 2, 2, 2 ** 31 - 1]):
        base = torch.full((T + 2, N), 7.0, dtype=BF16, device=DEV)
        b.linear_mx4(X, W, offsets=torch.tensor(edges, dtype=torch.int32, device=DEV), Y=base[1:-1])
        b.linear_status()
        assert bool((base[0] == 7).all()) and bool((base[-1] == 7).all())


@forms
@pytest.mark.parametrize("T", [3, 40, 300])
def test_scales_far_apart_and_large(T, both4):
    """Scales from 2^-20 to 2^20 in one row, and scales above 2, where the decoded factor takes two products."""
    rng = np.random.default_rng(T)
    K, N = 320, 200
    for low, high in ((107, 148), (127, 160)):
        W, w = _mx4(rng, N, K, low, high)
        if both4:
            X, x = _mx4(rng, T, K, low, high)
        else:
            X = _randn((T, K), 1)
            x = eref.f64(X)
        _check(b.linear_mx4(X, W), *eref.linear(x, w, None, "none", None, None, None, BF16))
    b.linear_status()


@forms
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("glu", [False, True], ids=["plain", "glu"])
def test_nan_scales_and_values_stay_where_they_are(T, both4, glu):
    rng = np.random.default_rng(T)
    K, N = 160, 140
    W, V = _mx4(rng, N, K)[0], _mx4(rng, N, K)[0] if glu else None
    X = _randn((T, K), 1)
    X[1, 3] = float("nan")
    codes, scales = W.codes.clone(), W.scales.clone()
    scales[0, 1, 5 * 16] = 255                                         # row 5, block 4
    Y = b.linear_mx4(b.mx4_quantize(X) if both4 else X, W._replace(scales=scales), act=b.ACT_SILU, W_up=V)
    b.linear_status()
    want = torch.zeros((T, N), dtype=torch.bool, device=DEV)
    want[1], want[:, 5] = True, True
    assert torch.equal(torch.isnan(Y), want)


@forms
def test_in_place_residual_equal_bits_and_rows_alone(both4):
    for T, K, N in ((5, 256, 200), (60, 256, 200), (400, 256, 200)):
        X, W, V, bw, bv, R, Y = _dense(T, K, N, both4, act="silu", glu=True, bias=True, residual=True)
        again = R.clone()
        b.linear_mx4(X, W, bias=bw, act=b.ACT_SILU, W_up=V, bias_up=bv, residual=again, Y=again)
        assert torch.equal(again, Y)


@forms
def test_other_stream_and_captured(both4):
    rng = np.random.default_rng(0)
    for T in (3, 50, 400):
        X = _randn((T, 256), 1)
        W, _ = _mx4(rng, 300, 256)
        rows = b.mx4_quantize(X) if both4 else X
        want = b.linear_mx4(rows, W)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = b.linear_mx4(b.mx4_quantize(X, stream=side) if both4 else X, W, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            Y = b.linear_mx4(b.mx4_quantize(X) if both4 else X, W)
        X.copy_(_randn((T, 256), 2))
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
        assert torch.equal(Y, b.linear_mx4(b.mx4_quantize(X) if both4 else X, W))


def test_every_access_stays_inside():
    with b.library(build.build_bounds_check()):
        b.bounds_report()
        for rows, K in ((1, 1), (5, 70), (131, 257)):
            for dtype in (BF16, F32):
                for X in (_rows(rows, K, dtype), _rows(rows, K + 5, dtype)[:, 3:3 + K]):
                    b.mx4_dequantize(b.mx4_quantize(X), dtype)
        for T, K, N in ((1, 40, 5), (9, 1001, 33), (40, 200, 257), (300, 136, 131)):
            W, V = (b.mx4_quantize(_rows(N, K, BF16, seed=s)) for s in (1, 2))
            X, bias, R = _pitched((T, K), 3), _randn((N,), 4), _randn((T, N + 1), 5)[:, 1:]
            for x in (X, b.mx4_quantize(X)):
                b.linear_mx4(x, W)
                b.linear_mx4(x, W, bias=bias, act=b.ACT_SILU, W_up=V, bias_up=bias, residual=R)
            S = b.mx4_quantize(torch.stack([_rows(N, K, BF16, seed=s) for s in range(3)]))
            for edges in ([0, T // 2, T // 2, T], [-5, 2, 1, T + 90], [1, 1, 1, 1]):
                for x in (X, b.mx4_quantize(X)):
                    b.linear_mx4(x, S, bias=_randn((3, N), 6), offsets=torch.tensor(edges, dtype=torch.int32, device=DEV))
        for T, K, N in ((2, 4096, 14336), (11, 4100, 14001)):          # rows that are split into 4-bit ones
            assert b.linear_mx4_workspace_bytes(T, K, N, has_up=True) > 0
            W, X = _normal_mx4(N, K, 1), _pitched((T, K), 3)
            for x in (X, b.mx4_quantize(X)):
                b.linear_mx4(x, W, W_up=W, residual=_randn((T, N), 5))
            S, edges = b.MX4(W.codes.expand(2, -1, -1).contiguous(), W.scales.expand(2, -1, -1, -1).contiguous(), K), torch.tensor([-5, 1, T + 9], dtype=torch.int32, device=DEV)
            b.linear_mx4(X, S, W_up=S, offsets=edges)
        rep = b.bounds_report()
    assert rep["violations"] == 0, rep
