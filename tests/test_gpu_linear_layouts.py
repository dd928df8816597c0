"""dass_linear per expert with one of the two biases alone, lengths that are no multiple of 8 and rows at a padded pitch: the
epilogue's 16-byte accesses, against 64 bits and in the checked-access build (which counts misaligned accesses too)."""
import numpy as np
import pytest
import torch

import expert_reference as ref
from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200 import build

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
both = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
# rows, K, N, groups: few rows; tens of rows with and without a split of the contraction; many rows
SIZES = pytest.mark.parametrize("T,K,N,G", [(20, 256, 100, 3), (96, 2048, 100, 3), (120, 512, 1028, 2), (400, 512, 1028, 8), (800, 512, 1027, 8), (3000, 128, 100, 2)])
BIASES = pytest.mark.parametrize("gate,up", [(False, True), (True, False), (True, True), (False, False)], ids=["up", "gate", "both", "none"])


def _randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _padded(t, fill=float("nan")):
    """The same matrix at the next pitch that is a multiple of 8 and longer than its rows."""
    base = torch.full((t.shape[0], t.shape[1] // 8 * 8 + 8), fill, dtype=t.dtype, device=DEV)
    view = base[:, :t.shape[1]]
    view.copy_(t)
    return view


def _inputs(T, K, N, G, dtype, gate, up):
    cuts = sorted(int(v) for v in np.random.default_rng(T + N).integers(0, T + 1, G - 1))
    edges = [0] + cuts + [T]
    X, W, V = _randn((T, K), dtype, 1), _randn((G, N, K), dtype, 2, K ** -0.5), _randn((G, N, K), dtype, 3, K ** -0.5)
    return (edges, torch.tensor(edges, dtype=torch.int32, device=DEV), X, W, V, _randn((G, N), dtype, 4) if gate else None,
            _randn((G, N), dtype, 5) if up else None, _randn((T, N), dtype, 6))


@both
@SIZES
@BIASES
def test_one_bias_and_padded_rows(T, K, N, G, gate, up, dtype):
    edges, offsets, X, W, V, bw, bv, R = _inputs(T, K, N, G, dtype, gate, up)
    for residual in (None, _padded(R)):
        out = _padded(torch.zeros((T, N), dtype=dtype, device=DEV), fill=7.0)
        Y = b.linear(X, W, bias=bw, act=b.ACT_SILU, W_up=V, bias_up=bv, residual=residual, offsets=offsets, Y=out)
        b.linear_status()
        for g in range(G):
            lo, hi = edges[g], edges[g + 1]
            f = lambda t: None if t is None else ref.f64(t[g])                     # noqa: E731
            want, bound = ref.linear(ref.f64(X[lo:hi]), f(W), f(bw), "silu", f(V), f(bv), ref.f64(R[lo:hi]) if residual is not None else None, dtype)
            assert np.all(np.abs(ref.f64(Y[lo:hi]) - want) <= bound)
        pad = torch.as_strided(out, (T, out.stride(0) - N), (out.stride(0), 1), N)
        assert bool((pad == 7).all())


@pytest.fixture(scope="module")
def check_lib():
    with b.library(build.build_bounds_check()):
        assert b.bounds_report()["violations"] == 0
        yield
    torch.cuda.synchronize()


@both
@SIZES
@BIASES
def test_no_access_is_outside_or_misaligned(check_lib, T, K, N, G, gate, up, dtype):
    edges, offsets, X, W, V, bw, bv, R = _inputs(T, K, N, G, dtype, gate, up)
    out = _padded(torch.zeros((T, N), dtype=dtype, device=DEV))
    for residual in (None, _padded(R), R):
        b.linear(X, W, bias=bw, act=b.ACT_SILU, W_up=V, bias_up=bv, residual=residual, offsets=offsets, Y=out)
    b.linear_status()
    rep = b.bounds_report()
    assert rep["violations"] == 0, f"access outside the call's buffers or misaligned: {rep}"
