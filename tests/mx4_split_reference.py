"""Rows in bf16 as sums of 4-bit rows (numpy): the split as dass_linear_mx4 states it, and rows that need all of it."""
import numpy as np

from mx4_reference import SIZES

PIECES = 12


def pieces(X, count=PIECES):
    """[count x rows x K] float64: of what the pieces before left, the nearest e2m1 values under the scale that takes the largest of
    a block of 32 into (3, 6] (at most 2^125, at least 2^-127); ties to the even code."""
    rows, K = X.shape
    blocks = (K + 31) // 32
    rest = np.zeros((rows, blocks * 32))
    rest[:, :K] = X
    rest = rest.reshape(rows, blocks, 32)
    out = np.zeros((count, rows, blocks * 32))
    for j in range(count):
        m, e = np.frexp(np.abs(rest).max(2))                           # m 2^e, m in [0.5, 1): above 0.75 one more
        s = np.clip(np.where(m > 0.75, e, e - 1) - 2, -127, 125)[:, :, None]
        y = np.minimum(np.ldexp(np.abs(rest), -s), 6.0)
        at = np.searchsorted(SIZES, y, side="right") - 1
        up = np.minimum(at + 1, 7)
        above, below = SIZES[up] - y, y - SIZES[at]
        size = np.where((above < below) | ((above == below) & (at % 2 == 1)), SIZES[up], SIZES[at])
        piece = np.copysign(np.ldexp(size, s), rest)
        rest = rest - piece
        out[j] = piece.reshape(rows, -1)
    return out[:, :, :K]


def together(parts):
    """The pieces added up as the kernel does it: in f32, the smallest first."""
    total = np.zeros(parts.shape[1:], np.float32)
    for p in parts[::-1]:
        total = total + p.astype(np.float32)
    return total.astype(np.float64)


def block_max(X):
    rows, K = X.shape
    pad = np.pad(np.abs(X), ((0, 0), (0, -K % 32))).reshape(rows, -1, 32).max(2)
    return np.repeat(pad, 32, 1)[:, :K]


def wide_rows(rng, rows, K):
    """bf16 numbers whose blocks of 32 hold sizes from 2^20 down to 2^-10, and some a single large value among 1s."""
    x = np.ldexp(1 + rng.integers(0, 128, (rows, K)) / 128, 20 - rng.integers(0, 31, (rows, K))) * rng.choice([-1.0, 1.0], (rows, K))
    one = (np.arange(K) // 32) % 5 == 0                                # 1.99 x 2^20 and 1.37 x 2^10 beside 1.71
    x[:, one] = 219 / 128
    x[:, one & (np.arange(K) % 32 == 7)] = 255 / 128 * 2.0 ** 20
    x[:, one & (np.arange(K) % 32 == 19)] = -175 / 128 * 2.0 ** 10
    return x
