"""Layers with 4-bit weights whose rows are no whole 16 bytes long: the intermediate's pitch is the library's own matter."""
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


def _aligned(x):
    """The same rows at a pitch of whole 16 bytes; the padding is NaN."""
    base = torch.full((*x.shape[:-1], (x.shape[-1] + 7) // 8 * 8), float("nan"), dtype=BF16, device=DEV)
    base[..., :x.shape[-1]] = x
    return base[..., :x.shape[-1]]


def _rounded(x):
    return ref.values(*ref.quantize(x))[:, :x.shape[1]]


@pytest.mark.parametrize("rows4", [False, True], ids=["bf16-rows", "4-bit-rows"])
@pytest.mark.parametrize("T,d,I", [(1, 128, 356), (5, 96, 4), (200, 128, 356)])
def test_pruned_layer(T, d, I, rows4):
    """Pruned in float32, which takes rows of whole 16 bytes (4 values); run on bfloat16 tokens."""
    pruner = LayerPruner(T, d, I, F32)
    X, Wg, Wu, Wd = _rand((T, d), 0), _rand((I, d), 1, 0.1), _rand((I, d), 2, 0.1), _rand((d, I), 3, 0.1)
    pruner.prune(*(t.float() for t in (X, Wg, Wu, Wd)))
    q = pruner.quantize_pruned()
    Z = pruner.forward_quantized(X, q, rows_in_4_bits=rows4)
    rows = b.mx4_quantize if rows4 else lambda x: x
    H = b.linear_mx4(rows(X), q["gate"], act=b.ACT_SILU, W_up=q["up"])
    h = _rounded(eref.f64(H)) if rows4 else eref.f64(H)
    want, bound = eref.linear(h, eref.f64(b.mx4_dequantize(q["down"], F32)), None, "none", None, None, None, BF16)
    assert Z.shape == (T, d) and np.all(np.abs(eref.f64(Z) - want) <= bound)
    b.linear_status()


@pytest.mark.parametrize("rows4", [False, True], ids=["bf16-rows", "4-bit-rows"])
@pytest.mark.parametrize("T,d,I", [(1, 96, 100), (37, 100, 36)])
def test_experts(T, d, I, rows4):
    """A layer against the calls it is made of, with the rows between them in aligned buffers."""
    E, k = 4, 2
    X, Wr = _aligned(_rand((T, d), 0)), _aligned(_rand((E, d), 1))
    Wg, Wu, Wd = (b.mx4_quantize(_rand(s, 2 + i, 0.05)) for i, s in enumerate(((E, I, d), (E, I, d), (E, d, I))))
    small = ExpertLayer(Wr, Wg, Wu, Wd, k, rows_in_4_bits=rows4)
    Y, saved = small.forward(X, residual=X, keep=True)
    r = saved.routed
    rows = b.mx4_quantize if rows4 else _aligned
    H = b.linear_mx4(rows(b.expert_gather(X, r.slot, r.offsets)), Wg, act=b.ACT_SILU, W_up=Wu, offsets=r.offsets)
    Ys = b.linear_mx4(rows(H), Wd, offsets=r.offsets)
    assert torch.equal(saved.Ys, Ys) and torch.equal(Y, b.expert_combine(Ys, r.slot, r.weight, residual=X))
    assert bool(torch.isfinite(Y).all())
    small.check()
