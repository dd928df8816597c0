"""4-bit weights and the balance loss in the layers that use them: a run of the calls together."""

import numpy as np
import pytest
import torch

import expert_reference as eref
import mx4_reference as ref
from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200.experts import ExpertLayer
from paper_2405_01943_b200.layer import LayerPruner

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _rand(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(BF16)


def _layer(T, E, k, d, I):
    X = _rand((T, d), 0)
    return X, ExpertLayer(_rand((E, d), 1), *(_rand(s, 2 + i, 0.05) for i, s in enumerate(((E, I, d), (E, I, d), (E, d, I)))), k=k)


def _rounded(x):
    return ref.values(*ref.quantize(x))[:, :x.shape[1]]


def _bf16(x):
    return torch.from_numpy(x).to(BF16).double().numpy()


@pytest.mark.parametrize("rows4", [False, True], ids=["bf16-rows", "4-bit-rows"])
@pytest.mark.parametrize("T,E,k,d,I", [(1, 4, 2, 96, 160), (37, 4, 2, 96, 160), (300, 3, 1, 256, 320)])
def test_quantized_experts(T, E, k, d, I, rows4):
    """Every token's output from 64-bit products of the 4-bit values, with the two roundings to bf16 (and to 4 bits) that the
    calls document.  An intermediate value next to a border may round the other way: a bf16 step of it, or in 4 bits a code's."""
    X, layer = _layer(T, E, k, d, I)
    layer.calibrate(X)
    layer.finalize()
    pruned = layer.prune()
    small = pruned.quantize(rows_in_4_bits=rows4)
    for W, Q in ((pruned.Wg, small.Wg), (pruned.Wd, small.Wd)):
        assert Q.shape == tuple(W.shape) and bool((b.mx4_dequantize(Q)[W == 0] == 0).all())       # the mask is kept
    Y, saved = small.forward(X, residual=X, keep=True)
    small.check()
    value = lambda Q, e: eref.f64(b.mx4_dequantize(Q, F32)[e])                                      # noqa: E731
    x, r = eref.f64(X), saved.routed
    ids, weight = r.expert.cpu().numpy(), eref.f64(r.weight)
    want, bound = x.copy(), np.abs(x) * 2 ** -8
    for e in range(E):
        g, u, w = (value(Q, e) for Q in (small.Wg, small.Wu, small.Wd))
        for t, j in zip(*np.nonzero(ids == e)):
            row = _rounded(x[t:t + 1]) if rows4 else x[t:t + 1]
            h, eh = eref.linear(row, g, None, "silu", u, None, None, BF16)
            hb = _bf16(h)
            # a value that the bound lets cross a border of bf16 moves a step (2^-7), and in 4 bits up to a step of its block (2 of 8)
            step = np.where(np.abs(h - hb) + (eh - np.abs(h) * 2 ** -8) > np.abs(h) * 2 ** -9 * 0.99, 2 ** -7 * np.abs(h), 0.0)
            if rows4:
                pad = np.pad(np.abs(hb), ((0, 0), (0, -I % 32))).reshape(-1, 32)
                q = _rounded(hb)
                low, high = _rounded(hb - step - 2 ** -24 * np.abs(hb)), _rounded(hb + step + 2 ** -24 * np.abs(hb))
                step = np.maximum(np.abs(low - q), np.abs(high - q))
                # a block whose largest value may cross a power of two takes another scale: all of its values may move
                top = pad.max(1)
                open_ = np.repeat(np.floor(np.log2(np.maximum(top * (1 + 2 ** -7), 1e-300))) != np.floor(np.log2(np.maximum(top * (1 - 2 ** -7), 1e-300))), 32)[:I]
                step = np.maximum(step, open_[None] * np.repeat(top, 32)[:I][None] / 4)
                hb = q
            y, ey = eref.linear(hb, w, None, "none", None, None, None, BF16)
            want[t] += weight[t, j] * y[0]
            bound[t] += weight[t, j] * (ey[0] + (step @ np.abs(w).T)[0] + 2 ** -8 * np.abs(y[0])) + 2 ** -8 * np.abs(weight[t, j] * y[0])
    bound += 2 ** -8 * np.abs(want)
    err = np.abs(eref.f64(Y) - want)
    assert np.all(err <= bound), float((err / bound).max())


def test_the_experts_form_is_checked():
    X, layer = _layer(8, 4, 2, 64, 96)
    small = layer.quantize()
    for call in (small.quantize, lambda: small.calibrate(X), small.prune):
        with pytest.raises(RuntimeError):
            call()
    with pytest.raises(ValueError):
        ExpertLayer(layer.Wr, small.Wg, layer.Wu, layer.Wd, 2)
    with pytest.raises(ValueError):
        ExpertLayer(layer.Wr, layer.Wg, layer.Wu, layer.Wd, 2, rows_in_4_bits=True)


@pytest.mark.parametrize("T,E,k", [(50, 8, 2), (3000, 40, 4)])
def test_router_gradient_with_balance(T, E, k):
    X, layer = _layer(T, E, k, 64, 96)
    Y, saved = layer.forward(X, keep=True)
    dY = _rand(Y.shape, 9, 0.1)
    plain = layer.router_gradient(dY, saved)
    both = layer.router_gradient(dY, saved, balance=0.5)
    loss, counts, share = layer.balance(saved.routed)
    x, ids = eref.f64(saved.routed.logits), saved.routed.expert.cpu().numpy()
    wl, wc, _, p, counted = ref.balance(x, ids)
    assert np.array_equal(counts.cpu().numpy(), wc) and abs(float(loss) - wl) <= 1e-5 * wl
    want = eref.f64(plain) + ref.balance_gradient(p, counted, wc, k, 0.5)
    err = np.abs(eref.f64(both) - want)
    bound = ref.gradient_bound(x, p, wc, k, 0.5, BF16, eref.f64(plain))
    assert np.all(err <= bound), float((err / bound).max())
    twice = layer.router_gradient(dY, saved, balance=0.5, counts=2 * counts)       # f and 1 / n: half the gradient for twice the tokens
    want = eref.f64(plain) + 0.5 * ref.balance_gradient(p, counted, wc, k, 0.5)
    assert np.all(np.abs(eref.f64(twice) - want) <= bound)


@pytest.mark.parametrize("rows4", [False, True], ids=["bf16-rows", "4-bit-rows"])
@pytest.mark.parametrize("T", [3, 200])
def test_pruned_layer_in_4_bits(T, rows4):
    """LayerPruner's products against the calls they are made of, and the weights against the pruned copies."""
    d, I = 128, 352
    pruner = LayerPruner(T, d, I, BF16)
    X, Wg, Wu, Wd = _rand((T, d), 0), _rand((I, d), 1, 0.1), _rand((I, d), 2, 0.1), _rand((d, I), 3, 0.1)
    out = pruner.prune(X, Wg, Wu, Wd)
    q = pruner.quantize_pruned()
    for name in ("gate", "up", "down"):
        w = eref.f64(out[name]["pruned"])
        assert np.array_equal(eref.f64(b.mx4_dequantize(q[name], F32)), ref.values(*ref.quantize(w))[:, :w.shape[1]])
    Z = pruner.forward_quantized(X, q, rows_in_4_bits=rows4)
    rows = b.mx4_quantize if rows4 else lambda x: x
    H = b.linear_mx4(rows(X), q["gate"], act=b.ACT_SILU, W_up=q["up"])
    x = _rounded(eref.f64(X)) if rows4 else eref.f64(X)
    value = lambda name: eref.f64(b.mx4_dequantize(q[name], F32))                                   # noqa: E731
    want, bound = eref.linear(x, value("gate"), None, "silu", value("up"), None, None, BF16)
    assert np.all(np.abs(eref.f64(H) - want) <= bound)
    h = _rounded(eref.f64(H)) if rows4 else eref.f64(H)
    want, bound = eref.linear(h, value("down"), None, "none", None, None, None, BF16)
    assert np.all(np.abs(eref.f64(Z) - want) <= bound)
    b.linear_status()
