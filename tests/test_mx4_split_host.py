"""The split of bf16 rows into 4-bit ones, by its definition: what 12 pieces hold, and that the test's rows need every one."""
import numpy as np
import pytest
import torch

import mx4_split_reference as s


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def test_twelve_pieces_hold_24_bits_of_a_block():
    rng = np.random.default_rng(0)
    for X in (rng.normal(size=(50, 320)), s.wide_rows(rng, 50, 330), rng.normal(size=(50, 320)) ** 5, np.ldexp(rng.normal(size=(9, 64)), 120), np.ldexp(rng.normal(size=(9, 64)), -100)):
        X = _bf16(X)
        assert np.all(np.abs(s.pieces(X).sum(0) - X) <= 2.0 ** -24 * s.block_max(X))


def test_small_blocks_are_held_to_the_smallest_code():
    """No scale is below 2^-127, so no code's step below 2^-128: half of one is what a value may be off by."""
    rng = np.random.default_rng(1)
    for e in (-110, -120, -126, -131):
        X = _bf16(np.ldexp(rng.normal(size=(20, 64)), e))
        assert np.all(np.abs(s.pieces(X).sum(0) - X) <= np.maximum(2.0 ** -24 * s.block_max(X), 2.0 ** -129))


@pytest.mark.parametrize("T,K", [(8, 1769), (20, 3459)])
def test_the_rows_need_every_piece(T, K):
    """Without any one of the 12 some products differ after their rounding to bf16; without one of the first eight they leave the
    documented bound, which later ones stay below (bf16's own 8 bits are used up before)."""
    X = s.wide_rows(np.random.default_rng(T), T, K)
    assert np.array_equal(_bf16(X), X)
    parts = s.pieces(X)
    want = _bf16(s.together(parts))
    bound = 2.0 ** -24 * s.block_max(X) + 2.0 ** -8 * np.abs(X)
    assert np.all(np.abs(want - X) <= bound)
    for j in range(s.PIECES):
        less = parts.copy()
        less[j] = 0
        got = _bf16(s.together(less))
        assert (got != want).any(), j
        if j < 8:
            assert (np.abs(got - X) > bound).any(), j
    assert (np.abs(_bf16(s.together(parts[:7])) - X) > bound).any()
