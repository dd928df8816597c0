"""Plain 64-bit definitions of the mixture-of-experts operators and of the matrix product with an epilogue (numpy, loops
over tokens and experts), and the error bounds that follow from the kernels' documented arithmetic."""
import numpy as np
import torch

EPS24 = 2.0 ** -24                                    # half a unit in the last place of an f32, relative
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float32: EPS24}   # significands of 8 and 24 bits, rounded to nearest


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


# ------------------------------------------------------------------ router
def route_order(row):
    """The unmasked experts of a row, highest logit first, ties by index; and the row with +inf taken as the largest f32."""
    x = np.minimum(np.where(np.isnan(row), -np.inf, row), float(np.finfo(np.float32).max))
    alive = [e for e in range(len(x)) if x[e] > -np.inf]
    return sorted(alive, key=lambda e: (-x[e], e)), x


def route(logits, k, over_all):
    T, E = logits.shape
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        order, x = route_order(logits[t])
        if not order:
            continue
        chosen = order[:k]
        part = order if over_all else chosen
        e = np.exp(x - x[order[0]])
        ids[t, :len(chosen)] = chosen
        w[t, :len(chosen)] = e[chosen] / e[part].sum()
    return ids, w


def route_weights_of(x, chosen, over_all):
    """The weights of fixed choices as a function of one row of logits (for differences)."""
    part = np.arange(len(x)) if over_all else np.array(chosen)
    e = np.exp(x - x.max())
    return e[chosen] / e[part].sum()


def route_gradient(logits, k, over_all, dweight):
    ids, w = route(logits, k, over_all)
    out = np.zeros(logits.shape)
    for t in range(len(logits)):
        order, x = route_order(logits[t])
        chosen = [e for e in ids[t] if e >= 0]
        if not chosen:
            continue
        part = order if over_all else chosen
        p = np.zeros(len(x))
        e = np.exp(x[part] - x[order[0]])
        p[part] = e / e.sum()
        up = np.zeros(len(x))
        up[chosen] = dweight[t, :len(chosen)]
        out[t] = p * (up - (p * up).sum())
    return out


def route_weight_bound(logits, E):
    """Relative: the subtraction from the maximum (range R of the finite logits), expf (2 units), numerator and sum alike,
    a sum of E terms and the division."""
    finite = logits[np.isfinite(logits)]
    R = float(finite.max() - finite.min()) if finite.size else 0.0
    return 2 * (min(R, 104.0) * EPS24 + 4 * EPS24) + (E + 2) * EPS24


# ------------------------------------------------------------------ order
def sort(ids, E):
    T, k = ids.shape
    flat = ids.reshape(-1)
    order = [f for e in range(E) for f in np.flatnonzero(flat == e)]
    offsets = np.array([int(((flat >= 0) & (flat < e)).sum()) for e in range(E + 1)], np.int32)
    slot, source = np.full(T * k, -1, np.int32), np.full(T * k, -1, np.int32)
    slot[order] = np.arange(len(order))
    source[:len(order)] = order
    return offsets, slot.reshape(T, k), source


# ------------------------------------------------------------------ rows
def combine(Ys, slot, weight, residual):
    """(value, sum of magnitudes) of the weighted sum."""
    T, k = slot.shape
    y = np.zeros((T, Ys.shape[1])) if residual is None else residual.copy()
    mag = np.abs(y)
    for t in range(T):
        for j in range(k):
            if 0 <= slot[t, j] < len(Ys):
                term = (1.0 if weight is None else weight[t, j]) * Ys[slot[t, j]]
                y[t] += term
                mag[t] += np.abs(term)
    return y, mag


def combine_gradient(dY, Ys, slot, weight):
    """(dYs, dweight, sum of magnitudes of dweight's terms)."""
    T, k = slot.shape
    dYs, dw, mag = np.zeros(Ys.shape), np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            s = slot[t, j]
            if 0 <= s < len(Ys):
                dYs[s] = (1.0 if weight is None else weight[t, j]) * dY[t]
                dw[t, j] = (dY[t] * Ys[s]).sum()
                mag[t, j] = np.abs(dY[t] * Ys[s]).sum()
    return dYs, dw, mag


# ------------------------------------------------------------------ matrix product
def act(name, x):
    if name == "silu":
        return x / (1.0 + np.exp(-x))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)))
    return np.maximum(x, 0.0) if name == "relu" else x


def linear(X, W, bias, act_name, W_up, bias_up, residual, dtype):
    """(value, bound) for one group of rows.  Bound: f32 sums of K + 1 terms (a unit of 2^-23 a term, which also covers an
    accumulator that truncates), the activation's slope (at most 1.13) and its own error (2^-19 relative, of its argument's
    size: fast exponentials), two products and one addition in f32, one rounding to dtype."""
    with np.errstate(over="ignore"):
        K = X.shape[1]
        p = X @ W.T + (0.0 if bias is None else bias)
        ep = (K + 1) * 2 * EPS24 * (np.abs(X) @ np.abs(W).T + (0.0 if bias is None else np.abs(bias)))
        y = act(act_name, p)
        e = ep if act_name == "none" else 1.13 * ep + 2.0 ** -19 * np.abs(p)
        if W_up is not None:
            u = X @ W_up.T + (0.0 if bias_up is None else bias_up)
            eu = (K + 1) * 2 * EPS24 * (np.abs(X) @ np.abs(W_up).T + (0.0 if bias_up is None else np.abs(bias_up)))
            e = e * (np.abs(u) + eu) + np.abs(y) * eu + 2 * EPS24 * np.abs(y * u)
            y = y * u
        if residual is not None:
            y = y + residual
            e = e + 2 * EPS24 * np.abs(y)
        return y, e + HALF_ULP[dtype] * (np.abs(y) + e) + 1e-37
