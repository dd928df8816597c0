"""dass_linear_mx4 in every variant that its choice of kernel can take, against 64-bit products."""
import pytest
import torch

import expert_reference as eref
import mx4_variants as v
import test_gpu_mx4 as t
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F64 = torch.bfloat16, torch.float64
ACTIVATIONS = {"none": lambda x: x, "silu": lambda x: x * torch.sigmoid(x), "relu": lambda x: x.clamp_min(0),
               "gelu_tanh": lambda x: 0.5 * x * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3)))}


def _weights(groups, N, K, seed):
    """Random weights in 4 bits, a matrix or a stack of them; scales differ from block to block."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    shape = (groups, N, K) if groups else (N, K)
    w = torch.randn(shape, generator=g, device=DEV) * 0.02
    w *= torch.exp2(torch.randint(-2, 3, (*shape[:-1], (K + 31) // 32), generator=g, device=DEV).float()).repeat_interleave(32, -1)[..., :K]
    return b.mx4_quantize(w)


def _offsets(T, groups, seed):
    """Uneven groups, some of them empty, and rows before the first and after the last."""
    g = torch.Generator().manual_seed(seed)
    share = torch.rand(groups, generator=g) ** 2 + 0.02
    if groups > 2:
        share[int(torch.randint(0, groups, (1,), generator=g))] = 0
    head, tail = (1, 2) if T > 8 else (0, 0)
    edges = torch.cat((torch.zeros(1), share.cumsum(0) / share.sum())) * (T - head - tail)
    return (edges.round().int() + head).tolist()


def _want(x, lost, w, up, bias, bias_up, residual, act):
    """Value and bound of expert_reference.linear, on the device.  `lost` is what a split row may be off by, element by element."""
    K, eps = x.shape[1], eref.EPS24

    def product(w, add):
        a = 0.0 if add is None else add.to(F64)
        size = x.abs() @ w.abs().t()
        extra = 0.0 if lost is None else lost @ w.abs().t() + 12 * eps * size                  # a sum of 12 parts
        return x @ w.t() + a, (K + 1) * 2 * eps * (size + abs(a)) + extra

    p, ep = product(w, bias)
    y = ACTIVATIONS[act](p)
    e = ep if act == "none" else 1.13 * ep + 2.0 ** -19 * p.abs()
    if up is not None:
        u, eu = product(up, bias_up)
        e = e * (u.abs() + eu) + y.abs() * eu + 2 * eps * (y * u).abs()
        y = y * u
    if residual is not None:
        y = y + residual.to(F64)
        e = e + 2 * eps * y.abs()
    return y, e + eref.HALF_ULP[BF16] * (y.abs() + e) + 1e-37


@pytest.mark.parametrize("case", range(len(v.CASES)), ids=lambda i: "-".join(str(int(x)) for x in v.CASES[i]))
def test_variant(case):
    both4, glu, T, K, N, groups = v.CASES[case]
    kernel = v.plan(T, K, N, groups, both4, glu)[0]
    rows = t._pitched((T, K), case)
    X = b.mx4_quantize(rows) if both4 else rows
    x = b.mx4_dequantize(X, torch.float32).to(F64) if both4 else rows.to(F64)
    lost = None
    if kernel == 1 and not both4:
        pad = torch.nn.functional.pad(x.abs(), (0, -K % 32)).view(T, -1, 32)
        lost = (2.0 ** -24 * pad.amax(2, keepdim=True)).expand_as(pad).reshape(T, -1)[:, :K]
    W, V = _weights(groups, N, K, 2), _weights(groups, N, K, 3) if glu else None
    per = (groups, N) if groups else (N,)
    bias, bias_up, residual = (t._randn(per, 4), t._randn(per, 5) if glu else None, t._pitched((T, N), 6)) if case % 2 else (None, None, None)
    edges = _offsets(T, groups, case) if groups else [0, T]
    offsets = torch.tensor(edges, dtype=torch.int32, device=DEV) if groups else None
    names = list(ACTIVATIONS)
    # the CTA-pair kernels have an instance for each activation
    for act in names if kernel >= 2 else [names[case % 4]]:
        Y = b.linear_mx4(X, W, bias=bias, act=t.ACTS[act], W_up=V, bias_up=bias_up, residual=residual, offsets=offsets)
        assert torch.equal(b.linear_mx4(X, W, bias=bias, act=t.ACTS[act], W_up=V, bias_up=bias_up, residual=residual, offsets=offsets), Y)
        b.linear_status()
        assert bool((Y[:edges[0]] == 0).all()) and bool((Y[edges[-1]:] == 0).all())
        for g in range(max(groups, 1)):
            lo, hi = edges[g], edges[g + 1]
            if lo == hi:
                continue
            one = lambda q: None if q is None else b.mx4_dequantize(b.MX4(q.codes[g], q.scales[g], K) if groups else q, torch.float32).to(F64)  # noqa: E731
            part = lambda z: None if z is None else z[g] if groups else z                                          # noqa: E731
            want, bound = _want(x[lo:hi], None if lost is None else lost[lo:hi], one(W), one(V), part(bias), part(bias_up),
                                None if residual is None else residual[lo:hi], act)
            err = (Y[lo:hi].to(F64) - want).abs()
            assert bool((err <= bound).all()), (act, g, float((err / bound).max()), (err > bound).nonzero()[:3].tolist())
