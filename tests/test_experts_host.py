"""Refusals of the mixture-of-experts calls and of dass_linear that are decided before the device is touched."""
import ctypes

import pytest
import torch

import expert_reference as ref
from paper_2405_01943_b200 import binding, build

NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5, 6
P = 1 << 20                                                            # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_route(lib):
    f = lambda x=P, T=4, E=8, ld=8, dt=1, k=2, norm=0, ids=P, w=P: lib.dass_route_topk(x, T, E, ld, dt, k, norm, ids, w, None)  # noqa: E731
    assert f(x=None) == NULL and f(ids=None) == NULL and f(w=None) == NULL
    assert f(dt=5) == DTYPE and f(norm=2) == DTYPE
    assert f(T=-1) == SHAPE and f(E=0) == SHAPE and f(ld=7) == SHAPE and f(k=0) == SHAPE and f(k=9) == SHAPE
    assert f(E=1025, ld=1025) == UNSUPPORTED and f(E=64, ld=64, k=33) == UNSUPPORTED and f(T=1 << 31) == UNSUPPORTED
    assert f(x=P + 2) == ALIGN and f(ids=P + 1) == ALIGN and f(w=P + 2) == ALIGN
    assert f(T=0) == 0
    g = lambda x=P, T=4, E=8, k=2, ids=P, dw=P, dl=P, ldd=8: lib.dass_route_topk_backward(x, T, E, 8, 1, k, 0, ids, dw, dl, ldd, None)  # noqa: E731
    assert g(x=None) == NULL and g(ids=None) == NULL and g(dw=None) == NULL and g(dl=None) == NULL
    assert g(ldd=7) == SHAPE and g(dl=P + 2) == ALIGN and g(T=0) == 0


def test_sort(lib):
    out = ctypes.c_size_t(7)
    q = lib.dass_expert_sort_workspace_bytes
    assert q(4, 2, 8, None) == NULL and q(-1, 2, 8, ctypes.byref(out)) == SHAPE and q(4, 0, 8, ctypes.byref(out)) == SHAPE
    assert q(4, 2, 1025, ctypes.byref(out)) == UNSUPPORTED and q(4, 33, 8, ctypes.byref(out)) == UNSUPPORTED
    assert q(1 << 31, 1, 8, ctypes.byref(out)) == UNSUPPORTED and q(1 << 62, 32, 8, ctypes.byref(out)) == UNSUPPORTED
    assert q(16, 2, 8, ctypes.byref(out)) == 0 and out.value == 0
    assert q(100000, 8, 64, ctypes.byref(out)) == 0 and out.value > 0
    f = lambda ids=P, T=4, k=2, E=8, off=P, slot=P, src=P, ws=P, n=1 << 20: lib.dass_expert_sort(ids, T, k, E, off, slot, src, ws, n, None)  # noqa: E731
    assert f(ids=None) == NULL and f(off=None) == NULL and f(slot=None) == NULL
    assert f(E=0) == SHAPE and f(off=P + 2) == ALIGN and f(src=P + 1) == ALIGN
    assert f(T=100000, ws=None) == WORKSPACE and f(T=100000, n=8) == WORKSPACE and f(T=100000, ws=P + 4) == ALIGN


def test_rows(lib):
    g = lambda X=P, T=4, d=16, ldx=16, dt=0, slot=P, k=2, Xs=P, rows=8, ldxs=16: lib.dass_expert_gather(  # noqa: E731
        X, T, d, ldx, dt, slot, k, None, None, Xs, rows, ldxs, None)
    assert g(X=None) == NULL and g(slot=None) == NULL and g(Xs=None) == NULL and g(dt=2) == DTYPE
    assert g(ldx=15) == SHAPE and g(ldxs=15) == SHAPE and g(d=0) == SHAPE and g(T=-1) == SHAPE and g(k=0) == SHAPE and g(rows=-1) == SHAPE
    assert g(k=33) == UNSUPPORTED and g(T=1 << 30) == UNSUPPORTED and g(X=P + 1) == ALIGN and g(slot=P + 2) == ALIGN
    assert g(rows=0) == 0 and g(T=0) == 0
    c = lambda Ys=P, d=16, ldys=16, slot=P, T=4, R=None, ldr=0, Y=P, ldy=16: lib.dass_expert_combine(  # noqa: E731
        Ys, 8, d, ldys, 0, slot, T, 2, None, R, ldr, Y, ldy, None)
    assert c(Ys=None) == NULL and c(slot=None) == NULL and c(Y=None) == NULL and c(ldys=8) == SHAPE and c(ldy=8) == SHAPE
    assert c(R=P, ldr=8) == SHAPE and c(R=P + 1, ldr=16) == ALIGN and c(T=0) == 0
    h = lambda dY=P, Ys=P, dYs=P, dw=P, ldd=16: lib.dass_expert_combine_backward(dY, 4, 16, 16, Ys, 8, 16, 0, P, 2, None, None, dYs, ldd, dw, None)  # noqa: E731
    assert h(dYs=None, dw=None) == NULL and h(dY=None) == NULL and h(Ys=None) == NULL and h(ldd=8) == SHAPE and h(dw=P + 2) == ALIGN


def test_linear(lib):
    def f(X=P, T=4, K=64, ldx=64, W=P, V=None, N=32, ldw=64, gs=0, b=None, bu=None, act=3, R=None, ldr=0, Y=P, ldy=32, dt=0, off=None, G=1):
        return lib.dass_linear(X, T, K, ldx, W, V, N, ldw, gs, b, bu, act, R, ldr, Y, ldy, dt, off, G, None)
    assert f(X=None) == NULL and f(W=None) == NULL and f(Y=None) == NULL and f(bu=P) == NULL
    assert f(dt=2) == DTYPE and f(act=4) == DTYPE and f(act=-1) == DTYPE
    assert f(T=-1) == SHAPE and f(K=0) == SHAPE and f(N=0) == SHAPE and f(ldx=63) == SHAPE and f(ldw=56) == SHAPE and f(ldy=31) == SHAPE
    assert f(R=P, ldr=31) == SHAPE and f(G=2) == SHAPE and f(G=0, off=P) == SHAPE and f(G=2, off=P, gs=64) == SHAPE
    assert f(X=P + 8) == ALIGN and f(W=P + 8) == ALIGN and f(V=P + 8) == ALIGN and f(ldx=68) == ALIGN and f(ldw=68) == ALIGN
    assert f(Y=P + 1) == ALIGN and f(b=P + 1) == ALIGN and f(off=P + 2, G=1) == ALIGN and f(off=P, G=2, gs=32 * 64 + 4) == ALIGN
    assert f(T=1 << 31) == UNSUPPORTED and f(G=70000, off=P, gs=32 * 64) == UNSUPPORTED
    assert f(T=0) == 0


def test_the_rounding_unit_of_the_bounds():
    """HALF_ULP is what rounding to nearest can cost and no more: the worst case over a binade, by torch's own cast."""
    x = 1.0 + torch.arange(1 << 16, dtype=torch.float64) / (1 << 16)
    worst = float(((x.to(torch.bfloat16).double() - x).abs() / x).max())
    assert 0.9 * ref.HALF_ULP[torch.bfloat16] < worst <= ref.HALF_ULP[torch.bfloat16]
    x = 1.0 + torch.arange(1 << 16, dtype=torch.float64) * 2.0 ** -30
    worst = float(((x.float().double() - x).abs() / x).max())
    assert 0.9 * ref.HALF_ULP[torch.float32] < worst <= ref.HALF_ULP[torch.float32]
