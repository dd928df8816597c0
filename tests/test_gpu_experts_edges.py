"""Mixture-of-experts calls at the edges of their contracts."""
import ctypes

import pytest
import torch

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


class _Word:
    """An int32 of device memory at an address, as a tensor's memory."""

    def __init__(self, address):
        self.__cuda_array_interface__ = {"shape": (1,), "typestr": "<i4", "data": (address, False), "version": 2}


def test_a_timeout_is_reported_once_and_none_is_lost():
    """Every bounded wait that runs out is counted on the device; a query reports what no query has reported and leaves the
    count alone, so that what another stream records beside it is there for the next one."""
    address = b.load()._ZN4dass15linear_timeoutsEv
    address.restype, address.argtypes = ctypes.c_void_p, []
    b.linear_status()
    count = torch.as_tensor(_Word(address()), device=DEV)
    start = int(count)
    for times in (1, 3):
        count += times
        with pytest.raises(b.DassError) as e:
            b.linear_status()
        assert e.value.code == 8
        b.linear_status()
    assert int(count) == start + 4
    s = torch.cuda.Stream()                                              # recorded on another stream, after this query's answer
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        count += 1
    b.linear_status(torch.cuda.current_stream())
    s.synchronize()
    with pytest.raises(b.DassError):
        b.linear_status()
    b.linear_status()
    X = torch.ones((70, 2048), dtype=BF16, device=DEV)
    W = torch.ones((4096, 2048), dtype=BF16, device=DEV)
    assert bool((b.linear(X, W) == 2048).all())
    b.linear_status()


def test_a_call_that_was_made_once_can_be_captured():
    """The same call replayed from a graph on new inputs; one size for each of the bf16 kernels."""
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    for T, K, N in ((4, 64, 72), (64, 2048, 4096), (1100, 128, 136)):
        X, W, Y = (torch.randn(s, generator=g, device=DEV).to(BF16) for s in ((T, K), (N, K), (T, N)))
        b.linear(X, W, Y=Y)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.linear(X, W, Y=Y)
        X.copy_(torch.randn((T, K), generator=g, device=DEV).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, b.linear(X, W))
        del graph
    b.linear_status()
