"""The checked-access build over ragged cases of the mixture-of-experts calls and of dass_linear: no load or store falls
outside the buffers a call was given, whatever ids, slots and offsets hold."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200 import build

pytestmark = pytest.mark.gpu
DEV = "cuda"
both = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def check_lib():
    with b.library(build.build_bounds_check()):
        assert b.bounds_report()["violations"] == 0
        yield
    torch.cuda.synchronize()


def _clean():
    rep = b.bounds_report()
    assert rep["violations"] == 0, f"access outside the call's buffers: {rep}"


def _rand(*shape, dtype):
    return torch.randn(shape, device=DEV).to(dtype)


@both
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (33, 7, 3), (100, 60, 8), (65, 257, 9), (9, 1000, 32)])
def test_route(check_lib, dtype, T, E, k):
    for x in (_rand(T, E, dtype=dtype), _rand(T, E + 5, dtype=dtype)[:, 3:3 + E]):
        for renorm in (True, False):
            ids, w = b.route_topk(x, k, renormalise=renorm)
            b.route_topk_backward(x, ids, w, renormalise=renorm)
            wild = torch.randint(-(1 << 31), 1 << 31, (T, k), device=DEV).int()
            b.route_topk_backward(x, wild, w, renormalise=renorm)
            _clean()


@both
@pytest.mark.parametrize("T,E,k,d", [(1, 4, 2, 8), (37, 8, 3, 257), (700, 60, 8, 72), (2100, 300, 2, 40)])
def test_order_and_rows(check_lib, dtype, T, E, k, d):
    ids = torch.randint(-2, E + 2, (T, k), device=DEV, dtype=torch.int32)
    offsets, slot, source = b.expert_sort(ids, E)
    _clean()
    X, w = _rand(T, d, dtype=dtype), torch.rand(T, k, device=DEV)
    wild = torch.where(torch.rand(T, k, device=DEV) < 0.5, slot, torch.randint(-(1 << 31), 1 << 31, (T, k), device=DEV).int())
    for s in (slot, wild):
        Xs = torch.zeros((T * k, d), dtype=dtype, device=DEV)
        b.expert_gather(X, s, offsets, Xs=Xs)
        b.expert_gather(X, s, offsets, weight=w, Xs=Xs)
        b.expert_combine(Xs, s, w, residual=X)
        b.expert_gather_backward(Xs, s)
        b.expert_combine_backward(X, Xs, s, w, offsets, dYs=torch.zeros_like(Xs))
        b.expert_combine_backward(X, Xs, s, want_rows=False)
        _clean()


@both
@pytest.mark.parametrize("T,K,N", [(1, 70, 33), (5, 1000, 131), (20, 520, 2000), (70, 264, 300), (200, 133, 515), (600, 72, 1030), (1, 8, 1)])
def test_linear_dense(check_lib, dtype, T, K, N):
    up8 = (K + 7) // 8 * 8
    X, W, V = _rand(T, up8, dtype=dtype)[:, :K], _rand(N, up8, dtype=dtype)[:, :K], _rand(N, up8, dtype=dtype)[:, :K]
    bias, R = _rand(N, dtype=dtype), _rand(T, N + 3, dtype=dtype)[:, 1:N + 1]
    out = torch.empty((T, N + 3), dtype=dtype, device=DEV)[:, 2:N + 2]
    b.linear(X, W, bias=bias, residual=R)
    b.linear(X, W, act=b.ACT_GELU_TANH, W_up=V, bias=bias, bias_up=bias, residual=R, Y=out)
    b.linear_status()
    _clean()


@both
@pytest.mark.parametrize("T,G", [(3, 5), (40, 4), (300, 3), (900, 40), (1500, 2)])
def test_linear_per_expert(check_lib, dtype, T, G):
    K, N = 104, 331
    X, W, V, bias = _rand(T, K, dtype=dtype), _rand(G, N, K, dtype=dtype), _rand(G, N, K, dtype=dtype), _rand(G, N, dtype=dtype)
    cuts = torch.sort(torch.randint(0, T + 1, (G + 1,), device=DEV)).values.int()
    lies = torch.randint(-(1 << 31), 1 << 31, (G + 1,), device=DEV).int()
    for o in (cuts, torch.flip(cuts, (0,)), lies, torch.full_like(cuts, T), torch.zeros_like(cuts)):
        b.linear(X, W, bias=bias, offsets=o)
        b.linear(X, W, act=b.ACT_SILU, W_up=V, bias=bias, bias_up=bias, offsets=o)
        b.linear_status()
        _clean()


def test_control_a_shortened_range_is_caught(check_lib):
    X, W = _rand(300, 64, dtype=torch.bfloat16), _rand(520, 64, dtype=torch.bfloat16)
    Y = torch.full((300, 520), 7.0, dtype=torch.bfloat16, device=DEV)
    b.bounds_shrink_next(2048)
    b.linear(X, W, Y=Y)
    assert b.bounds_report()["violations"] > 0
    assert bool((Y.view(-1)[-1024:] == 7.0).all())
    b.linear(X, W, Y=Y)
    _clean()
