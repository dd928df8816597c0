"""The operators together: a mixture-of-experts layer calibrated, pruned, run and differentiated (experts.py)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import expert_reference as ref
import oracle
from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200.experts import ExpertLayer

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _layer(T, E, k, d, I, dtype, act="silu", renormalise=True, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)                # noqa: E731
    X = rand(T, d).to(dtype)
    Wr = (rand(E, d) * d ** -0.5).to(dtype)
    Wr[-1] -= 4.0 * (X.float().mean(0) / d).to(dtype)
    return X, ExpertLayer(Wr, (rand(E, I, d) * d ** -0.5).to(dtype), (rand(E, I, d) * d ** -0.5).to(dtype), (rand(E, d, I) * I ** -0.5).to(dtype),
                          k, act, renormalise)


def _reference(layer, X, routed, act, round_to):
    """Y in 64 bits from the choice the layer made, the steps rounded where the layer stores them."""
    r = lambda a: ref.f64(torch.from_numpy(a).to(round_to))                  # noqa: E731
    ids, w = routed.expert.cpu().numpy(), ref.f64(routed.weight)
    Y = np.zeros((X.shape[0], layer.d))
    x = ref.f64(X)
    for e in range(layer.E):
        t, j = np.nonzero(ids == e)
        if len(t):
            h = r(ref.act(act, x[t] @ ref.f64(layer.Wg[e]).T) * (x[t] @ ref.f64(layer.Wu[e]).T))
            np.add.at(Y, t, w[t, j, None] * r(h @ ref.f64(layer.Wd[e]).T))
    return Y


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,E,k,d,I,act,renorm", [(1, 8, 2, 128, 256, "silu", True), (40, 8, 2, 256, 512, "gelu_tanh", False), (700, 6, 3, 136, 264, "relu", True)])
def test_forward(T, E, k, d, I, act, renorm, dtype):
    X, layer = _layer(T, E, k, d, I, dtype, act, renorm)
    R = torch.randn((T, d), device=DEV).to(dtype)
    r = layer.route(X)
    Y = layer.forward(X, residual=R, routed=r)
    want = _reference(layer, X, r, act, dtype) + ref.f64(R)
    layer.check()
    # bf16: a stored h or y that lies at a rounding boundary may fall to the other side, a whole unit (2^-7) of one term
    tol = 2.0 ** -6 if dtype == BF16 else 1e-4
    assert np.abs(ref.f64(Y) - want).max() <= tol * max(1.0, np.abs(want).max())
    assert np.linalg.norm(ref.f64(Y) - want) <= (2.0 ** -7 if dtype == BF16 else 1e-5) * np.linalg.norm(want)


@pytest.mark.parametrize("dtype,tol", [(BF16, 2e-3), (F32, 1e-5)], ids=["bf16", "f32"])
def test_calibration_and_pruning_per_expert(dtype, tol):
    T, E, k, d, I = 600, 5, 2, 128, 256
    X, layer = _layer(T, E, k, d, I, dtype)
    r = layer.route(X)
    r = r._replace(expert=torch.where(r.expert == 3, torch.full_like(r.expert, -1), r.expert))   # an expert that no token reaches
    r = r._replace(**dict(zip(("offsets", "slot", "source"), b.expert_sort(r.expert, E))))
    layer.reset()
    counts = layer.calibrate(X[:200], routed=None)
    layer.reset()
    counts = layer.calibrate(X, routed=r)
    norm = layer.finalize()
    ids = r.expert.cpu().numpy()
    assert counts == [(ids == e).sum() for e in range(E)] and counts[3] == 0
    f32 = lambda t: t.float().cpu().numpy()                                   # noqa: E731
    pruned = layer.prune(alpha=0.5)
    for e in range(E):
        if e == 3:
            assert bool((norm[e] == 0).all())
            use = torch.ones_like(norm[e])
        else:
            rows = X[torch.from_numpy(np.nonzero((ids == e).any(1))[0]).to(DEV)]
            want = oracle.norm_from_sumsq(oracle.calib_sumsq(f32(rows), f32(layer.Wg[e]), f32(layer.Wu[e]), oracle.ACT_SILU))
            assert np.abs(norm[e].cpu().numpy() - want).max() <= tol * want.max()
            use = norm[e]
        for W, P, axis, alpha in ((layer.Wg, pruned.Wg, b.AXIS_ROWS, 0.5), (layer.Wd, pruned.Wd, b.AXIS_COLS, 1.0)):
            assert torch.equal(P[e], b.score_nm(W[e], use, axis, alpha, 2, 4, axis, want_mask=False)[1])
    pruned.check()
    assert float((pruned.Wu == 0).float().mean()) >= 0.5


def test_router_gradient_against_differences():
    T, E, k, d, I = 24, 6, 2, 64, 128
    X, layer = _layer(T, E, k, d, I, F32)
    Y, saved = layer.forward(X, keep=True)
    dY = torch.randn((T, d), device=DEV)
    got = ref.f64(layer.router_gradient(dY, saved))
    r, Ys, g = saved.routed, ref.f64(saved.Ys), ref.f64(dY)
    logits, ids, slot = ref.f64(r.logits), r.expert.cpu().numpy(), r.slot.cpu().numpy()

    def loss(row, t):
        w = ref.route_weights_of(row, ids[t], over_all=False)
        return (w[:, None] * Ys[slot[t]]).sum(0) @ g[t]
    h = 1e-5
    for t in range(T):
        for e in range(E):
            up, dn = logits[t].copy(), logits[t].copy()
            up[e] += h
            dn[e] -= h
            diff = (loss(up, t) - loss(dn, t)) / (2 * h)
            assert abs(got[t, e] - diff) <= 1e-4 * max(1.0, np.abs(got[t]).max())


def test_the_example_runs_and_the_router_helps():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "prune_expert_layer.py")
    spec = importlib.util.spec_from_file_location("prune_expert_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(T=512, E=4, d=256, I=512, steps=8) > 0


def test_shapes_are_checked():
    X, layer = _layer(8, 4, 2, 64, 128, BF16)
    with pytest.raises(ValueError):
        ExpertLayer(layer.Wr, layer.Wg, layer.Wu, layer.Wg, 2)
    with pytest.raises(ValueError):
        ExpertLayer(layer.Wr[:3], layer.Wg, layer.Wu, layer.Wd, 2)
