"""What the layers with 4-bit weights refuse and hand on, on the CPU: the library's calls are stood in for."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200.experts import ExpertLayer, Routed
from paper_2405_01943_b200.layer import LayerPruner

BF16, F32 = torch.bfloat16, torch.float32
E, D = 4, 16


def _mx4(shape):
    *lead, cols = shape
    codes, scales = b._mx4_shapes(tuple(lead), cols)[:2]
    return b.MX4(torch.zeros(codes, dtype=torch.uint8), torch.zeros(scales, dtype=torch.uint8), cols)


@pytest.fixture
def calls(monkeypatch):
    """The library's calls as they treat sizes and types; those of linear_mx4 are kept."""
    kept = []

    def linear_mx4(X, W, bias=None, act=b.ACT_NONE, W_up=None, bias_up=None, residual=None, offsets=None, Y=None, workspace=None, stream=None):
        T = X.shape[0]
        kept.append((X, W, Y))
        if not isinstance(X, b.MX4):
            assert X.dtype == BF16 and X.stride(1) == 1 and X.stride(0) % 8 == 0 and X.data_ptr() % 16 == 0     # as the library has it
        return torch.zeros((T, W.shape[-2]), dtype=BF16) if Y is None else Y

    monkeypatch.setattr(b, "linear_mx4", linear_mx4)
    monkeypatch.setattr(b, "mx4_quantize", lambda X, out=None, stream=None: kept.append(("quantize", X)) or _mx4(X.shape))
    monkeypatch.setattr(b, "expert_gather", lambda X, slot, offsets, Xs=None: X.repeat(2, 1) if Xs is None else Xs)
    monkeypatch.setattr(b, "expert_combine", lambda Ys, slot, weight, residual=None: Ys[:len(Ys) // 2])
    return kept


def _layer(dtype, I=32):
    return ExpertLayer(*(torch.zeros(s, dtype=dtype) for s in ((E, D), (E, I, D), (E, I, D), (E, D, I))), 2)


_routed = Routed(*(torch.zeros(0),) * 6)


@pytest.mark.parametrize("rows4", [False, True], ids=["bf16-rows", "4-bit-rows"])
def test_float32_is_refused_before_any_call(calls, rows4):
    with pytest.raises(TypeError):
        _layer(F32).quantize(rows_in_4_bits=rows4)
    assert not calls
    small = _layer(BF16).quantize(rows_in_4_bits=rows4)
    calls.clear()
    with pytest.raises(TypeError):
        small.forward(torch.zeros(5, D), routed=_routed)
    assert not calls
    assert small.forward(torch.zeros(5, D, dtype=BF16), routed=_routed).dtype == BF16
    pruner = LayerPruner(5, D, 32, F32, device="cpu", overlap_projections=False)
    weights = pruner.quantize_pruned()                                        # float32 copies are quantised
    calls.clear()
    with pytest.raises(TypeError):
        pruner.forward_quantized(torch.zeros(5, D), weights, rows_in_4_bits=rows4)
    assert not calls
    assert pruner.forward_quantized(torch.zeros(5, D, dtype=BF16), weights, rows_in_4_bits=rows4).shape == (5, D)


@pytest.mark.parametrize("rows4", [False, True], ids=["bf16-rows", "4-bit-rows"])
@pytest.mark.parametrize("I", [4, 32, 36, 356])
def test_rows_of_any_length_reach_the_second_product(calls, I, rows4):
    pruner = LayerPruner(5, D, I, BF16, device="cpu", overlap_projections=False)
    weights = pruner.quantize_pruned()
    for T in (1, 5):
        assert pruner.forward_quantized(torch.zeros(T, D, dtype=BF16), weights, rows_in_4_bits=rows4).shape == (T, D)
        assert _layer(BF16, I).quantize(rows_in_4_bits=rows4).forward(torch.zeros(T, D, dtype=BF16), routed=_routed).shape == (T, D)
