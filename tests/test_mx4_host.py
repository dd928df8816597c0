"""Refusals of the 4-bit calls and of the balance loss that are decided before the device is touched, and the layout's sizes."""
import ctypes

import numpy as np
import pytest
import torch

import mx4_reference as ref
from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200 import build

OK, NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5, 6
P = 1 << 20                                                            # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return b.load()


def test_sizes(lib):
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    for rows, K, codes, scales in ((0, 1, 0, 0), (1, 1, 16, 512), (128, 128, 128 * 64, 512), (129, 129, 129 * 80, 4 * 512), (3, 32, 48, 512)):
        assert lib.dass_mx4_bytes(rows, K, ctypes.byref(c), ctypes.byref(s)) == OK and (c.value, s.value) == (codes, scales)
        want = b._mx4_shapes((rows,), K)
        assert (int(np.prod(want[0])), int(np.prod(want[1]))) == (codes, scales)
    assert lib.dass_mx4_bytes(1, 1, ctypes.byref(c), None) == OK and lib.dass_mx4_bytes(1, 1, None, None) == NULL
    assert lib.dass_mx4_bytes(-1, 1, ctypes.byref(c), None) == SHAPE and lib.dass_mx4_bytes(1, 0, ctypes.byref(c), None) == SHAPE
    assert lib.dass_mx4_bytes(1 << 31, 1, ctypes.byref(c), None) == UNSUPPORTED


def test_quantize(lib):
    f = lambda x=P, G=1, rows=4, K=40, ld=40, stride=0, dt=0, c=P, s=P: lib.dass_mx4_quantize(x, G, rows, K, ld, stride, dt, c, s, None)  # noqa: E731
    d = lambda x=P, G=1, rows=4, K=40, ld=40, stride=0, dt=0, c=P, s=P: lib.dass_mx4_dequantize(c, s, G, rows, K, x, ld, stride, dt, None)  # noqa: E731
    for g in (f, d):
        assert g(x=None) == NULL and g(c=None) == NULL and g(s=None) == NULL
        assert g(dt=2) == DTYPE
        assert g(G=0) == SHAPE and g(rows=-1) == SHAPE and g(K=0) == SHAPE and g(ld=39) == SHAPE and g(G=2, stride=159) == SHAPE
        assert g(rows=1 << 31) == UNSUPPORTED and g(K=1 << 31, ld=1 << 31) == UNSUPPORTED and g(rows=1 << 30, K=1 << 30, ld=1 << 30) == UNSUPPORTED
        assert g(x=P + 1) == ALIGN and g(c=P + 8) == ALIGN and g(s=P + 4) == ALIGN and g(x=P + 2, dt=1) == ALIGN
        assert g(rows=0) == OK


def test_linear(lib):
    def f(X=P, ldx=64, xc=None, xs=None, T=4, K=64, wc=P, ws=P, uc=None, us=None, N=8, bias=None, bu=None, act=3, R=None, ldr=8, Y=P, ldy=8,
          off=None, groups=1, work=None):
        return lib.dass_linear_mx4(X, ldx, xc, xs, T, K, wc, ws, uc, us, N, bias, bu, act, R, ldr, Y, ldy, off, groups, work, 0, None)

    assert f(act=4) == DTYPE
    assert f(X=None) == NULL and f(wc=None) == NULL and f(ws=None) == NULL and f(uc=P) == NULL and f(us=P) == NULL and f(Y=None) == NULL
    assert f(X=None, xc=P) == NULL and f(X=None, xs=P) == NULL and f(bu=P) == NULL
    assert f(xc=P, xs=P) == UNSUPPORTED
    assert f(T=-1) == SHAPE and f(K=0) == SHAPE and f(N=0, ldy=0) == SHAPE and f(ldx=56) == SHAPE and f(ldy=7) == SHAPE and f(R=P, ldr=7) == SHAPE
    assert f(groups=0) == SHAPE and f(groups=2) == SHAPE
    for name in ("X", "wc", "ws"):
        assert f(**{name: P + 8}) == ALIGN
    assert f(uc=P + 8, us=P) == ALIGN and f(uc=P, us=P + 8) == ALIGN and f(ldx=65) == ALIGN
    assert f(X=None, xc=P + 8, xs=P) == ALIGN and f(X=None, xc=P, xs=P + 8) == ALIGN
    assert f(bias=P + 1) == ALIGN and f(R=P + 1) == ALIGN and f(Y=P + 1) == ALIGN and f(off=P + 2) == ALIGN
    assert f(work=P + 8) == ALIGN
    assert f(T=1 << 29) == UNSUPPORTED and f(N=1 << 31, ldy=1 << 31) == UNSUPPORTED and f(off=P, groups=1025) == UNSUPPORTED
    assert f(T=0) == OK and f(T=0, X=None, Y=None) == OK


def test_workspace_of_the_product(lib):
    q, out = lib.dass_linear_mx4_workspace_bytes, ctypes.c_size_t(9)
    f = lambda T=5, K=4096, N=14336, G=1, off=0, up=1, x4=0: q(T, K, N, G, off, up, x4, ctypes.byref(out))          # noqa: E731
    assert q(1, 1, 1, 1, 0, 0, 0, None) == NULL
    assert f(T=-1) == SHAPE and f(K=0) == SHAPE and f(N=0) == SHAPE and f(G=0) == SHAPE and f(G=2) == SHAPE
    assert f(T=1 << 29) == UNSUPPORTED and f(off=1, G=1025) == UNSUPPORTED
    assert f(T=0) == OK and out.value == 0
    assert f(x4=1) == OK and out.value == 0                            # only bf16 rows are split into others
    assert f(K=64, N=64) == OK and out.value == 0                      # and only where the weights are the time
    assert f() == OK and out.value > 0
    need = out.value
    assert lib.dass_linear_mx4(P, 4096, None, None, 5, 4096, P, P, P, P, 14336, None, None, 3, None, 0, P, 14336, None, 1, P, need - 1, None) == WORKSPACE
    assert lib.dass_linear_mx4(P, 4096, None, None, 5, 4096, P, P, P, P, 14336, None, None, 3, None, 0, P, 14336, None, 1, None, need, None) == WORKSPACE
    assert f(G=8, off=1) == OK and out.value > need
    assert b.linear_mx4_workspace_bytes(5, 4096, 14336, has_up=True) == need


def test_balance(lib):
    out = ctypes.c_size_t(7)
    q = lib.dass_route_balance_workspace_bytes
    assert q(4, 8, None) == NULL and q(-1, 8, ctypes.byref(out)) == SHAPE and q(4, 0, ctypes.byref(out)) == SHAPE
    assert q(4, 1025, ctypes.byref(out)) == UNSUPPORTED and q(1 << 31, 8, ctypes.byref(out)) == UNSUPPORTED
    assert q(4, 8, ctypes.byref(out)) == OK and out.value == 0
    assert q(65536, 128, ctypes.byref(out)) == OK and out.value > 0

    def f(x=P, T=65536, E=128, ld=128, dt=1, ids=P, k=8, loss=P, counts=P, share=P, ws=P, n=out.value):
        return lib.dass_route_balance(x, T, E, ld, dt, ids, k, loss, counts, share, ws, n, None)

    def g(x=P, T=4, E=8, ld=8, dt=1, ids=P, k=2, counts=P, dloss=None, add=None, lda=8, dl=P, ldd=8):
        return lib.dass_route_balance_backward(x, T, E, ld, dt, ids, k, counts, dloss, add, lda, dl, ldd, None)

    for h in (f, g):
        assert h(x=None) == NULL and h(ids=None) == NULL and h(counts=None) == NULL
        assert h(dt=3) == DTYPE
        assert h(T=-1) == SHAPE and h(E=0, ld=0) == SHAPE and h(ld=7) == SHAPE and h(k=0) == SHAPE
        assert h(E=1025, ld=1025) == UNSUPPORTED and h(k=33) == UNSUPPORTED and h(T=1 << 28, k=8) == UNSUPPORTED
        assert h(x=P + 2) == ALIGN and h(ids=P + 2) == ALIGN and h(counts=P + 1) == ALIGN
    assert f(loss=None) == NULL and f(share=None) == NULL and f(loss=P + 2) == ALIGN and f(share=P + 2) == ALIGN
    assert f(ws=None) == WORKSPACE and f(n=out.value - 1) == WORKSPACE and f(ws=P + 4) == ALIGN
    assert g(dl=None) == NULL and g(ldd=7) == SHAPE and g(add=P, lda=7) == SHAPE
    assert g(dl=P + 2) == ALIGN and g(add=P + 2) == ALIGN and g(dloss=P + 1) == ALIGN
    assert g(T=0) == OK


def test_reference_rounds_to_the_nearest_code_and_keeps_the_mask():
    """The definition the GPU tests go by, by hand: ties to the even code, saturation, powers of two, zeros, NaN blocks."""
    x = np.zeros((2, 70))
    x[0, :10] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26, 7.9]       # scale 1: the largest, 7.9, lies in [4, 8)
    x[0, 32] = 2.0 ** -140
    x[1, 64:70] = [np.nan, 1, 2, 3, 4, 5]
    codes, scales = ref.quantize(x)
    assert scales[0].tolist() == [127, 0, 0] and scales[1].tolist() == [0, 0, 255]
    assert ref.values(codes, scales)[0, :10].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, 6.0]
    assert np.isnan(ref.values(codes, scales)[1, 64:]).all() and (codes[0, 10:] == 0).all()
    assert np.array_equal(ref.unpack(ref.pack(codes)), codes)


class _Device(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 0


def test_bindings_refuse_what_does_not_fit(lib, monkeypatch):
    calls = []

    class Library:
        def __getattr__(self, name):
            return getattr(lib, name) if name.endswith("_bytes") else lambda *a: calls.append(name) or b.OK

    monkeypatch.setattr(b, "load", lambda: Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype).as_subclass(_Device)                          # noqa: E731
    u8 = torch.uint8
    W = b.MX4(z(40, 32, dtype=u8), z(1, 1, 512, dtype=u8), 64)
    X, I = z(5, 64), z(6, 2, dtype=torch.int32)
    assert W.shape == (40, 64) and b.linear_mx4(X, W).shape == (5, 40) and len(calls) == 1
    q = b.mx4_quantize(X)
    assert q.shape == (5, 64) and b.linear_mx4(q, W, W_up=W).shape == (5, 40) and b.mx4_dequantize(W).shape == (40, 64)
    bad = [lambda: b.linear_mx4(z(5, 65), W), lambda: b.linear_mx4(X, b.MX4(W.codes[:, :16], W.scales, 64)),
           lambda: b.linear_mx4(X, b.MX4(W.codes, W.scales[:, :, ::2], 64)), lambda: b.linear_mx4(X, b.MX4(W.codes, W.scales.int(), 64)),
           lambda: b.linear_mx4(X, W, W_up=b.MX4(W.codes[:39], W.scales, 64)), lambda: b.linear_mx4(X, W, bias_up=z(40)),
           lambda: b.linear_mx4(X, W, bias=z(39)), lambda: b.linear_mx4(X, W, bias=z(40, dtype=torch.float32)),
           lambda: b.linear_mx4(X, W, residual=z(5, 39)), lambda: b.linear_mx4(X, W, Y=z(4, 40)), lambda: b.linear_mx4(X.t(), W),
           lambda: b.linear_mx4(X, W, offsets=z(2, dtype=torch.int32)), lambda: b.linear_mx4(torch.zeros(5, 64, dtype=torch.bfloat16), W),
           lambda: b.mx4_quantize(X.t()), lambda: b.mx4_quantize(z(5)), lambda: b.mx4_quantize(X, out=q._replace(cols=63)),
           lambda: b.mx4_quantize(torch.zeros(5, 64)), lambda: b.mx4_quantize(z(5, 0)), lambda: b.mx4_dequantize(W, out=z(40, 63)),
           lambda: b.mx4_dequantize(W, torch.float32, out=z(40, 64)),
           lambda: b.route_balance(z(6, 8), I[:5]), lambda: b.route_balance(z(6, 8), I.long()), lambda: b.route_balance(z(6, 8), I, counts=z(8, dtype=torch.int32)),
           lambda: b.route_balance(z(6, 8), I, workspace=z(64)), lambda: b.route_balance_backward(z(6, 8), I, z(8, dtype=torch.int32)),
           lambda: b.route_balance_backward(z(6, 8), I, z(9, dtype=torch.int32), dloss=z(1, dtype=torch.float32)),
           lambda: b.route_balance_backward(z(6, 8), I, z(9, dtype=torch.int32), add=z(6, 7))]
    for i, call in enumerate(bad):
        before = len(calls)
        with pytest.raises(ValueError):
            call()
        assert len(calls) == before, i
    for call in (lambda: b.linear_mx4(z(5, 64, dtype=torch.float32), W), lambda: b.mx4_quantize(z(5, 64, dtype=torch.float16)),
                 lambda: b.mx4_dequantize(W, torch.float16), lambda: b.route_balance(z(6, 8, dtype=torch.float16), I)):
        with pytest.raises(TypeError):
            call()
    assert b.route_balance(z(6, 8), I)[1].shape == (9,) and b.route_balance_backward(z(6, 8), I, z(9, dtype=torch.int32), add=z(6, 8)).shape == (6, 8)
