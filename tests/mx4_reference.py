"""Plain 64-bit definitions (numpy) of the microscaled 4-bit values and of the router's balance, and the error bounds that
follow from the kernels' documented arithmetic."""
import numpy as np
import torch

from expert_reference import EPS24, HALF_ULP

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ------------------------------------------------------------------ 4-bit values
def quantize(X):
    """(codes [rows x up32(K)], one a value, and scale bytes [rows x blocks]) of float64 rows that hold f32 values."""
    rows, K = X.shape
    blocks = (K + 31) // 32
    x = np.zeros((rows, blocks * 32))
    x[:, :K] = X
    x = x.reshape(rows, blocks, 32)
    bad = ~np.isfinite(x).all(2)
    size = np.where(bad[:, :, None], 0.0, np.abs(x))
    most = size.max(2)
    _, e = np.frexp(most)                                              # most = m 2^e, m in [0.5, 1)
    s = np.where(most > 0, np.maximum(0, e - 1 - 2 + 127), 0)
    y = np.minimum(np.ldexp(size, (127 - s)[:, :, None]), 6.0)
    at = np.searchsorted(SIZES, y, side="right") - 1                   # the size at or below y
    up = np.minimum(at + 1, 7)
    to_up, to_down = SIZES[up] - y, y - SIZES[at]
    code = np.where((to_up < to_down) | ((to_up == to_down) & (at % 2 == 1)), up, at)
    code = np.where(np.signbit(np.where(bad[:, :, None], 0.0, x)), code + 8, code)
    return code.reshape(rows, -1).astype(np.uint8), np.where(bad, 255, s).astype(np.uint8)


def values(codes, scales):
    """float64 values of codes [rows x 32 blocks] under scale bytes [rows x blocks]."""
    v = np.where(codes >= 8, -1.0, 1.0) * SIZES[codes & 7]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v.reshape(*scales.shape, 32) * s[:, :, None]).reshape(codes.shape)


def pack(codes):
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def unpack(packed):
    out = np.empty((packed.shape[0], packed.shape[1] * 2), np.uint8)
    out[:, 0::2], out[:, 1::2] = packed & 15, packed >> 4
    return out


def tile(scales, fill=0):
    """Scale bytes [rows x blocks] in the stored order, byte by byte as the format is stated."""
    rows, blocks = scales.shape
    R, B = (rows + 127) // 128, (blocks + 3) // 4
    out = np.full((R, B, 512), fill, np.uint8)
    for r in range(rows):
        for b in range(blocks):
            out[r // 128, b // 4, r % 32 * 16 + r % 128 // 32 * 4 + b % 4] = scales[r, b]
    return out


def random_mx4(rng, rows, K, low=118, high=124):
    """A random matrix in 4 bits: (packed codes, tiled scales, its float64 values [rows x K])."""
    blocks = (K + 31) // 32
    codes = rng.integers(0, 16, (rows, blocks * 32), dtype=np.uint8)
    codes[:, K:] = 0
    scales = rng.integers(low, high, (rows, blocks), dtype=np.uint8)
    return pack(codes), tile(scales), values(codes, scales)[:, :K]


# ------------------------------------------------------------------ balance
def balance(logits, expert):
    """(loss, counts [E + 1], share [E], p [T x E], counted [T])."""
    T, E = logits.shape
    k = expert.shape[1]
    x = np.minimum(np.where(np.isnan(logits), -np.inf, logits), float(np.finfo(np.float32).max))
    p = np.zeros((T, E))
    for t in range(T):
        on = x[t] > -np.inf
        if on.any():
            e = np.exp(x[t, on] - x[t, on].max())
            p[t, on] = e / e.sum()
    inside = (expert >= 0) & (expert < E)
    counted = inside.any(1)
    counts = np.zeros(E + 1, np.int64)
    for e in range(E):
        counts[e] = (expert == e).sum()
    n = counts[E] = int(counted.sum())
    if n == 0:
        return 0.0, counts, np.zeros(E), p, counted
    share = p[counted].sum(0) / n
    return E * float((counts[:E] / (n * k)) @ share), counts, share, p, counted


def balance_gradient(p, counted, counts, k, dloss):
    E, n = len(counts) - 1, int(counts[-1])
    if n == 0:
        return np.zeros(p.shape)
    f = counts[:E] / (n * k)
    return dloss * E / n * p * (f - (p @ f)[:, None]) * counted[:, None]


def softmax_bound(logits, E):
    """Relative, of a probability: the subtraction from the row's maximum (range R of the finite logits; below -104 the
    exponential is 0 or subnormal), expf (2 units) in numerator and sum, a sum of E terms, the reciprocal and a product."""
    finite = logits[np.isfinite(logits)]
    R = float(finite.max() - finite.min()) if finite.size else 0.0
    return 2 * (min(R, 104.0) * EPS24 + 4 * EPS24) + (E + 4) * EPS24


def share_bound(logits, share, T, E):
    """A sum of T positive terms (a unit a term, any order), the quotient, the terms' own error; subnormal terms."""
    return share * (softmax_bound(logits, E) + (T + 3) * EPS24) + 1e-37


def gradient_bound(logits, p, counts, k, dloss, dtype, add=None):
    """f_e: two roundings; the dot product of E terms; the difference; four products.  One rounding to dtype."""
    E, n = len(counts) - 1, max(1, int(counts[-1]))
    f = counts[:E] / (n * k)
    rel = softmax_bound(logits, E)
    dot = (p @ f)[:, None]
    inner = f * 3 * EPS24 + dot * (rel + (E + 5) * EPS24) + EPS24 * np.abs(f - dot)
    c = abs(dloss) * E / n
    e = c * p * (inner + (np.abs(f - dot) + inner) * (rel + 6 * EPS24))
    y = c * p * np.abs(f - dot)
    a = 0.0 if add is None else np.abs(add)
    e = e + EPS24 * (y + a + e) * (add is not None)
    return e + HALF_ULP[dtype] * (y + a + e) + (1e-40 if dtype == torch.bfloat16 else 1e-44) * 16
