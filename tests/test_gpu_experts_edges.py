"""Mixture-of-experts calls at the edges of their contracts."""
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


def _no_tokens(dtype, rows, d):
    none, X0 = torch.empty((0, 2), dtype=torch.int32, device=DEV), torch.empty((0, d), dtype=dtype, device=DEV)
    Ys, offsets = torch.ones((rows, d), dtype=dtype, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    for given in (True, False):
        out = torch.full((rows, d), 9.0, dtype=dtype, device=DEV) if given else None
        dYs, dw = b.expert_combine_backward(X0, Ys, none, offsets=offsets, dYs=out)
        assert bool((dYs == 0).all()) and dYs.shape == (rows, d) and dw.shape == (0, 2)
        only, _ = b.expert_combine_backward(X0, Ys, none, offsets=offsets, dYs=out, want_weight=False)
        assert bool((only == 0).all())
    used = torch.tensor([0, 2], dtype=torch.int32, device=DEV)            # rows in use are not touched
    dYs, _ = b.expert_combine_backward(X0, Ys, none, offsets=used, dYs=torch.full((rows, d), 9.0, dtype=dtype, device=DEV))
    assert bool((dYs[:2] == 9).all()) and bool((dYs[2:] == 0).all())
    kept, _ = b.expert_combine_backward(X0, Ys, none, dYs=torch.full((rows, d), 9.0, dtype=dtype, device=DEV))
    assert bool((kept == 9).all())                                        # no offsets: no rows are past the last expert's


@both
@pytest.mark.parametrize("rows,d", [(5, 16), (3, 1), (700, 257), (40, 4104)])
def test_gradient_rows_without_tokens(dtype, rows, d):
    """Rows past the last expert's are zeros also where there is no token at all."""
    _no_tokens(dtype, rows, d)


@both
def test_gradient_rows_without_tokens_stay_inside(dtype):
    with b.library(build.build_bounds_check()):
        b.bounds_report()
        _no_tokens(dtype, 33, 72)
        _no_tokens(dtype, 33, 71)
        rep = b.bounds_report()
    assert rep["violations"] == 0, rep


ACTS = {"none": b.ACT_NONE, **b.ACT_BY_NAME}


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("glu", [False, True], ids=["plain", "glu"])
@pytest.mark.parametrize("T,K,N,dtype", [(4, 64, 72, BF16), (64, 2048, 4096, BF16), (1100, 128, 136, BF16), (4, 64, 72, F32), (70, 64, 72, F32)],
                         ids=["few", "mid", "many", "f32-few", "f32"])
def test_nan_stays_nan_through_every_activation(T, K, N, dtype, act, glu):
    """A NaN among the inputs of an output makes that output NaN, and no other one."""
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)                 # noqa: E731
    X, W, V, bias = rand(T, K), rand(N, K), rand(N, K) if glu else None, rand(N)
    Y = b.linear(X, W, bias=bias, act=ACTS[act], W_up=V)
    assert bool(torch.isfinite(Y).all())
    want = torch.zeros((T, N), dtype=torch.bool, device=DEV)
    X, bias = X.clone(), bias.clone()
    X[1, 3], bias[5] = float("nan"), float("nan")
    want[1], want[:, 5] = True, True
    Y2 = b.linear(X, W, bias=bias, act=ACTS[act], W_up=V)
    b.linear_status()
    assert torch.equal(torch.isnan(Y2), want)
    assert torch.equal(Y2[~want], Y[~want])
