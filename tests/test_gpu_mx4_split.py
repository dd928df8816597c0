"""What a bf16 row is as a sum of 4-bit ones: products with a single term, so that nothing but the split is in the result."""
import numpy as np
import pytest
import torch

import expert_reference as eref
import mx4_split_reference as s
import mx4_variants as v
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
# sizes whose rows are split, with tiles of 4, 8 and 10 rows: (rows, k, columns, experts), plain and gated
SIZES = [(form[1], *size) for table in (v.SHAPES, v.IN_USE) for form, sizes in table.items() if not form[0] for size in sizes
         if size[1] * size[2] * max(size[3], 1) < 7e7]


def _one_term(N, K, groups, at):
    """Weights of 1 at k = at[n] of row n, and 0 elsewhere."""
    w = torch.zeros((max(groups, 1), N, K), dtype=BF16, device=DEV)
    w[:, torch.arange(N, device=DEV), at] = 1.0
    return b.mx4_quantize(w if groups else w[0])


def _check(T, K, N, groups, glu, X):
    at = torch.arange(N, device=DEV) * 37 % K                          # 37 and K share no factor in these sizes, or columns repeat
    rows = torch.from_numpy(X).to(BF16).to(DEV)
    base = torch.zeros((T, (K + 7) // 8 * 8), dtype=BF16, device=DEV)
    base[:, :K] = rows
    W, options = _one_term(N, K, groups, at), {}
    if glu:                                                            # the gate is the row's 1, the only value of its block
        options = dict(act=b.ACT_RELU, W_up=W)
        W = _one_term(N, K, groups, torch.full((N,), K // 64 * 32, device=DEV))
    if groups:
        options["offsets"] = torch.tensor([T * g // groups for g in range(groups + 1)], dtype=torch.int32, device=DEV)
    Y = eref.f64(b.linear_mx4(base[:, :K], W, **options))
    b.linear_status()
    k = at.cpu().numpy()
    bound = 2.0 ** -24 * s.block_max(X)[:, k] + 2.0 ** -8 * np.abs(X[:, k])
    err = np.abs(Y - X[:, k])
    assert np.all(err <= bound), (float((err / bound).max()), np.argwhere(err > bound)[:3].tolist())
    want = torch.from_numpy(s.together(s.pieces(X))).to(BF16).double().numpy()[:, k]
    assert np.array_equal(Y, want), np.argwhere(Y != want)[:3].tolist()


def _cases():
    out = []
    for glu, T, K, N, groups in SIZES:
        kernel, tile = v.plan(T, K, N, groups, False, glu)[:2]
        if kernel == 1:
            out.append((T, K, N, groups, glu, tile))
    return out


def test_rows_of_many_sizes_come_back():
    """Blocks that hold 30 binades, and small values beside large ones: to 2^-24 of the block's largest, and bit for bit what the
    twelve pieces add up to (each of which tests/test_mx4_split_host.py shows these rows to need)."""
    cases = _cases()
    assert {(c[3] > 0, c[4], c[5]) for c in cases} == {(g, glu, tile) for g in (False, True) for glu in (False, True) for tile in (4, 8, 10)}
    for T, K, N, groups, glu, tile in cases:
        X = s.wide_rows(np.random.default_rng(T), T, K)
        if glu:
            lo = K // 64 * 32
            X[:, lo:lo + 32] = 0.0
            X[:, lo] = 1.0
        _check(T, K, N, groups, glu, X)


@pytest.mark.parametrize("e", [-104, -110, -121, -126])
def test_small_rows_are_held_to_half_the_smallest_step(e):
    T, K, N, groups, glu, _ = _cases()[0]
    X = np.ldexp(np.random.default_rng(-e).normal(size=(T, K)), e)
    X = torch.from_numpy(X).to(BF16).double().numpy()
    base = torch.zeros((T, (K + 7) // 8 * 8), dtype=BF16, device=DEV)
    base[:, :K] = torch.from_numpy(X).to(DEV)
    at = torch.arange(N, device=DEV) * 37 % K
    w = torch.zeros((N, K), dtype=BF16, device=DEV)
    w[torch.arange(N, device=DEV), at] = 2.0 ** 40                     # so that no result is small
    assert not glu and not groups
    Y = eref.f64(b.linear_mx4(base[:, :K], b.mx4_quantize(w))) * 2.0 ** -40
    b.linear_status()
    k = at.cpu().numpy()
    bound = np.maximum(2.0 ** -24 * s.block_max(X)[:, k], 2.0 ** -129)
    bound = bound + 2.0 ** -8 * (np.abs(X[:, k]) + bound)
    assert np.all(np.abs(Y - X[:, k]) <= bound)
