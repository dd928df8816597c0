"""The mixture-of-experts operators and the matrix product with an epilogue, as measured cases.

A case is one call (or the calls of one direction) of an operator at one size.  ``run`` computes it in its plain form
(elementary torch operations in 32 bits, rounded once) or, where ``own`` is set, through this repository's package.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
LARGEST = float(torch.finfo(torch.float32).max)


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the router of a decode step: 32 sequences, many small experts, softmax over all of them; latency
        {"name": "route_decode", "op": "route", "T": 32, "E": 64, "k": 6, "dtype": "bf16", "renorm": False, "backward": False},
        # the router while it is tuned: a large batch, f32 logits, forward and gradient
        {"name": "route_train", "op": "route", "T": 65536, "E": 128, "k": 8, "dtype": "f32", "renorm": True, "backward": True},
        # the way in of a decode step: 16 sequences, 8 large experts; latency
        {"name": "dispatch_decode", "op": "dispatch", "T": 16, "E": 8, "k": 2, "d": 4096, "dtype": "bf16", "drop": 0.0, "backward": False},
        # odd sizes, f32, padding tokens that no expert gets, with the gradient
        {"name": "dispatch_ragged", "op": "dispatch", "T": 3001, "E": 60, "k": 3, "d": 1001, "dtype": "f32", "drop": 0.1, "backward": True},
        # a prefill or calibration batch over many small experts, with the gradient
        {"name": "dispatch_train", "op": "dispatch", "T": 16384, "E": 64, "k": 6, "d": 2048, "dtype": "bf16", "drop": 0.0, "backward": True},
        # the way back of a decode step, added to the residual stream; latency
        {"name": "combine_decode", "op": "combine", "T": 16, "E": 8, "k": 2, "d": 4096, "dtype": "bf16", "drop": 0.0, "residual": True, "backward": False},
        # the way back of a training batch, with the gradients of rows and weights
        {"name": "combine_train", "op": "combine", "T": 16384, "E": 64, "k": 6, "d": 2048, "dtype": "bf16", "drop": 0.0, "residual": True, "backward": True},
        # one token's output projection (4096 wide, as the 7B-shaped layers), with bias and residual; bound by the weights
        {"name": "linear_token", "op": "linear", "T": 1, "K": 4096, "N": 4096, "dtype": "bf16", "act": "none", "glu": False, "bias": True, "residual": True},
        # the tiny f32 layer's sizes, biased GeLU projection
        {"name": "linear_tiny_f32", "op": "linear", "T": 128, "K": 256, "N": 688, "dtype": "f32", "act": "gelu_tanh", "glu": False, "bias": True, "residual": False},
        # a batch's output projection at the 70B-shaped width, with bias and residual; bound by the tensor cores
        {"name": "linear_prefill", "op": "linear", "T": 8192, "K": 8192, "N": 8192, "dtype": "bf16", "act": "none", "glu": False, "bias": True, "residual": True},
        # the experts of a decode step: Mistral-7B-shaped GLU experts, a few rows each; bound by the weights
        {"name": "experts_decode", "op": "experts", "T": 16, "E": 8, "k": 2, "d": 4096, "I": 14336, "dtype": "bf16", "act": "silu", "drop": 0.0},
        # the same experts on a prefill or calibration batch, with padding tokens; bound by the tensor cores
        {"name": "experts_prefill", "op": "experts", "T": 8192, "E": 8, "k": 2, "d": 4096, "I": 14336, "dtype": "bf16", "act": "silu", "drop": 0.02},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step))


def draw(rng):
    op = rng.choice(("route", "dispatch", "combine", "linear", "experts"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    act = rng.choice(("none", "silu", "gelu_tanh", "relu"))
    if op == "route":
        E = _log(rng, 4, 512)
        return {"op": op, "T": _log(rng, 1, 65536 if E <= 128 else 16384), "E": E, "k": rng.randint(1, min(8, E)), "dtype": dtype,
                "renorm": rng.random() < 0.5, "backward": rng.random() < 0.5}
    if op in ("dispatch", "combine"):
        T, E = _log(rng, 1, 16384), _log(rng, 4, 256)
        k = rng.randint(1, min(8, E))
        d = _log(rng, 64, max(64, min(8192, 6 * 16384 * 2048 // (T * k))), rng.choice((1, 8, 64)) if dtype == "bf16" else 1)
        c = {"op": op, "T": T, "E": E, "k": k, "d": max(64, d), "dtype": dtype, "drop": rng.choice((0.0, 0.0, 0.1, 0.9)), "backward": rng.random() < 0.5}
        if op == "combine":
            c["residual"] = rng.random() < 0.5
        return c
    if op == "linear":
        K, N = _log(rng, 64, 8192, 8), _log(rng, 33, 14336)
        glu = act != "none" and rng.random() < 0.5
        top = 2.0e12 if dtype == "bf16" else 4.0e10          # flops
        return {"op": op, "T": _log(rng, 1, max(1, min(16384, int(top / (2.0 * K * N * (1 + glu)))))), "K": K, "N": N, "dtype": dtype,
                "act": act, "glu": glu, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5}
    E = _log(rng, 4, 64)
    d = _log(rng, 256, 4096, 8)
    I = _log(rng, 256, max(256, min(14336, 8 * 4096 * 14336 // (E * d))), 8)
    k = rng.randint(1, min(6, E))
    most = int(4.0e12 / (6.0 * d * I * k))
    return {"op": op, "T": _log(rng, 1, max(1, min(8192, most))), "E": E, "k": k, "d": d, "I": I, "dtype": "bf16",
            "act": rng.choice(("silu", "gelu_tanh", "relu")), "drop": rng.choice((0.0, 0.0, 0.1))}


def _active(c):
    """How many of the experts get a row, on average, were every choice alike."""
    return c["E"] * (1.0 - (1.0 - 1.0 / c["E"]) ** (c["T"] * c["k"] * (1.0 - c["drop"])))


def work(case):
    c, z = case, SIZE[case["dtype"]]
    T = c["T"]
    if c["op"] == "route":
        one = T * c["E"] * z
        back = (1 if c["renorm"] else 2) * one + 8 * T * c["k"]      # over the chosen alone, only their logits are read again
        return {"bytes": one + 8 * T * c["k"] + (back if c["backward"] else 0), "flops": 4.0 * T * c["E"] * (2 if c["backward"] else 1)}
    if c["op"] == "dispatch":
        n, kept = T * c["k"], T * c["k"] * (1.0 - c["drop"])
        one = T * c["d"] * z + n * c["d"] * z + 12 * n
        return {"bytes": one + (c["backward"] and kept * c["d"] * z + T * c["d"] * z + 4 * n), "flops": kept * c["d"] if c["backward"] else 1.0 * n}
    if c["op"] == "combine":
        n, kept, row = T * c["k"], T * c["k"] * (1.0 - c["drop"]), c["d"] * z
        one = kept * row + T * row * (2 if c["residual"] else 1) + 8 * n
        return {"bytes": one + (c["backward"] and T * row + kept * row + n * row + 12 * n), "flops": (2.0 + 3.0 * c["backward"]) * kept * c["d"]}
    if c["op"] == "linear":
        m = 1 + c["glu"]
        return {"bytes": z * (T * c["K"] + m * c["N"] * c["K"] + (1 + c["residual"]) * T * c["N"] + m * c["bias"] * c["N"]),
                "flops": 2.0 * m * T * c["K"] * c["N"]}
    kept = T * c["k"] * (1.0 - c["drop"])
    return {"bytes": z * (3.0 * _active(c) * c["d"] * c["I"] + 2.0 * kept * c["d"]), "flops": 6.0 * kept * c["d"] * c["I"]}


# ------------------------------------------------------------------------------------------------ inputs

def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def _weights(gen, shape, dtype):
    """Projections of several matrices are made in their own type: the f32 values of all of them would not fit beside each other."""
    return torch.randn(shape, generator=gen, device=DEV, dtype=dtype).mul_(0.02)


def _logits(gen, T, E, dtype):
    """Router logits: a token's own part and an expert's popularity, which makes the loads uneven."""
    return (torch.randn((T, E), generator=gen, device=DEV) * 1.5 + torch.randn(E, generator=gen, device=DEV) * 0.5).to(dtype)


def _choice(gen, c):
    """Expert ids [T x k] as a router gives them, with -1 for all of a padding token's."""
    ids = torch.topk(_logits(gen, c["T"], c["E"], torch.float32), c["k"], dim=1).indices.to(torch.int32)
    return torch.where(torch.rand((c["T"], 1), generator=gen, device=DEV) < c["drop"], torch.full_like(ids, -1), ids)


def _order(ids, E):
    """(offsets, slot, source) of ids by elementary operations: the stable order by expert, what was dropped last."""
    n = ids.numel()
    key = torch.where((ids >= 0) & (ids < E), ids, torch.full_like(ids, E)).reshape(-1)
    _, order = torch.sort(key, stable=True)
    offsets = (key[:, None] < torch.arange(E + 1, device=DEV)).sum(0)
    rank = torch.empty(n, dtype=torch.int64, device=DEV).scatter_(0, order, torch.arange(n, device=DEV))
    slot = torch.where(key < E, rank, torch.full_like(rank, -1))
    source = torch.where(torch.arange(n, device=DEV) < offsets[E], order, torch.full_like(order, -1))
    return offsets.to(torch.int32), slot.to(torch.int32).view(ids.shape), source.to(torch.int32)


def prepare(case, seed):
    c, dtype = case, TYPES[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = dict(c)
    if c["op"] == "route":
        s["logits"] = _logits(gen, c["T"], c["E"], dtype)
        s["dweight"] = _normal(gen, (c["T"], c["k"]), torch.float32)
    elif c["op"] == "dispatch":
        s["ids"] = _choice(gen, c)
        s["X"] = _normal(gen, (c["T"], c["d"]), dtype)
        s["dXs"] = _normal(gen, (c["T"] * c["k"], c["d"]), dtype) if c["backward"] else None
    elif c["op"] == "combine":
        s["offsets"], s["slot"], _ = _order(_choice(gen, c), c["E"])
        s["weight"] = torch.softmax(_normal(gen, (c["T"], c["k"]), torch.float32), 1)
        s["Ys"] = _normal(gen, (c["T"] * c["k"], c["d"]), dtype)
        s["R"] = _normal(gen, (c["T"], c["d"]), dtype) if c["residual"] else None
        s["dY"] = _normal(gen, (c["T"], c["d"]), dtype, 0.1) if c["backward"] else None
    elif c["op"] == "linear":
        s["X"] = _normal(gen, (c["T"], c["K"]), dtype)
        s["W"] = _weights(gen, (c["N"], c["K"]), dtype)
        s["V"] = _weights(gen, (c["N"], c["K"]), dtype) if c["glu"] else None
        s["b"] = _normal(gen, (c["N"],), dtype, 0.1) if c["bias"] else None
        s["bv"] = _normal(gen, (c["N"],), dtype, 0.1) if c["bias"] and c["glu"] else None
        s["R"] = _normal(gen, (c["T"], c["N"]), dtype) if c["residual"] else None
    else:
        s["offsets"], _, source = _order(_choice(gen, c), c["E"])
        s["X"] = _normal(gen, (c["T"] * c["k"], c["d"]), dtype) * (source >= 0)[:, None]
        s["Wg"] = _weights(gen, (c["E"], c["I"], c["d"]), dtype)
        s["Wu"] = _weights(gen, (c["E"], c["I"], c["d"]), dtype)
        s["Wd"] = _weights(gen, (c["E"], c["d"], c["I"]), dtype)
        s["most"] = max(1, int((s["offsets"][1:] - s["offsets"][:-1]).max()))   # rows of the fullest expert: the plan of a padded product
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _act(name, x):
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x.clamp_min(0.0) if name == "relu" else x


def _plain_route(s):
    T, E, k = s["T"], s["E"], s["k"]
    l = s["logits"].float()
    l = torch.where(l.isnan(), torch.full_like(l, -math.inf), l).clamp_max(LARGEST)
    top, at = torch.sort(l, dim=1, descending=True, stable=True)
    ids = torch.where(top[:, :k] > -math.inf, at[:, :k], torch.full_like(at[:, :k], -1))
    e = torch.where(l > -math.inf, torch.exp(l - top[:, :1]), torch.zeros_like(l))
    chosen = torch.where(ids >= 0, e.gather(1, at[:, :k]), torch.zeros_like(top[:, :k]))
    total = (chosen if s["renorm"] else e).sum(1, keepdim=True)
    share = torch.where(total > 0, 1.0 / total, torch.zeros_like(total))
    w = chosen * share
    out = {"expert": ids.to(torch.int32), "weight": w}
    if s["backward"]:
        dw = torch.where(ids >= 0, s["dweight"], torch.zeros_like(w))
        dot = (w * dw).sum(1, keepdim=True)
        if s["renorm"]:
            g = torch.zeros_like(l).scatter_add_(1, at[:, :k], w * (dw - dot))
        else:
            g = e * share * (torch.zeros_like(l).scatter_add_(1, at[:, :k], dw) - dot)
        out["dlogits"] = g.to(s["logits"].dtype)
    return out


def _rows_of(M, slot):
    """M[slot] in f32, zero where slot is -1: [T x k x d]."""
    return M[slot.long().clamp_min(0)].float() * (slot >= 0)[:, :, None]


def _plain_dispatch(s):
    offsets, slot, source = _order(s["ids"], s["E"])
    X = s["X"].float()
    rows = X[torch.div(source.long().clamp_min(0), s["k"], rounding_mode="floor")] * (source >= 0)[:, None]
    out = {"offsets": offsets, "slot": slot, "source": source, "Xs": rows.to(s["X"].dtype)}
    if s["backward"]:
        out["dX"] = _rows_of(s["dXs"], slot).sum(1).to(s["X"].dtype)
    return out


def _plain_combine(s):
    rows = _rows_of(s["Ys"], s["slot"])
    y = (rows * s["weight"][:, :, None]).sum(1)
    out = {"Y": (y + s["R"].float() if s["residual"] else y).to(s["Ys"].dtype)}
    if s["backward"]:
        dY = s["dY"].float()
        kept = (s["slot"] >= 0)
        to = torch.where(kept, s["slot"].long(), torch.full_like(s["slot"].long(), s["Ys"].shape[0])).reshape(-1)   # one row more, for what was dropped
        dYs = torch.zeros((s["Ys"].shape[0] + 1, s["d"]), dtype=torch.float32, device=DEV)
        dYs[to] = (s["weight"][:, :, None] * dY[:, None, :]).reshape(-1, s["d"])
        out["dYs"] = dYs[:-1].to(s["Ys"].dtype)
        out["dweight"] = (rows * dY[:, None, :]).sum(2)
    return out


def _plain_linear(s):
    X = s["X"].float()
    y = X @ s["W"].float().t()
    y = _act(s["act"], y + s["b"].float() if s["bias"] else y)
    if s["glu"]:
        v = X @ s["V"].float().t()
        y = y * (v + s["bv"].float() if s["bias"] else v)
    return {"Y": (y + s["R"].float() if s["residual"] else y).to(s["X"].dtype)}


def _plain_experts(s):
    n, E, most = s["X"].shape[0], s["E"], s["most"]
    start = s["offsets"].long()
    at = start[:-1, None] + torch.arange(most, device=DEV)                                   # [E x most]: every expert's rows, padded
    X = s["X"].float()[at.clamp_max(n - 1)]
    H = _act(s["act"], X @ s["Wg"].float().transpose(1, 2)) * (X @ s["Wu"].float().transpose(1, 2))
    Y = H @ s["Wd"].float().transpose(1, 2)
    row = torch.arange(n, device=DEV)
    of = (row[:, None] >= start[None, 1:-1]).sum(1)                                          # a row's expert
    inside = row < start[-1]
    back = (of * most + row - start[of]).clamp(0, E * most - 1)
    return {"Y": (Y.reshape(E * most, -1)[back] * inside[:, None]).to(s["X"].dtype)}


def _own(s):
    from paper_2405_01943_b200 import binding as b

    if s["op"] == "route":
        expert, weight = b.route_topk(s["logits"], s["k"], renormalise=s["renorm"])
        out = {"expert": expert, "weight": weight}
        if s["backward"]:
            out["dlogits"] = b.route_topk_backward(s["logits"], expert, s["dweight"], renormalise=s["renorm"])
        return out
    if s["op"] == "dispatch":
        offsets, slot, source = b.expert_sort(s["ids"], s["E"])
        out = {"offsets": offsets, "slot": slot, "source": source, "Xs": b.expert_gather(s["X"], slot, offsets)}
        if s["backward"]:
            out["dX"] = b.expert_gather_backward(s["dXs"], slot)
        return out
    if s["op"] == "combine":
        out = {"Y": b.expert_combine(s["Ys"], s["slot"], s["weight"], residual=s["R"])}
        if s["backward"]:
            out["dYs"], out["dweight"] = b.expert_combine_backward(s["dY"], s["Ys"], s["slot"], s["weight"], s["offsets"])
        return out
    act = {"none": b.ACT_NONE, **b.ACT_BY_NAME}[s["act"]]
    if s["op"] == "linear":
        return {"Y": b.linear(s["X"], s["W"], bias=s["b"], act=act, W_up=s["V"], bias_up=s["bv"], residual=s["R"])}
    H = b.linear(s["X"], s["Wg"], act=act, W_up=s["Wu"], offsets=s["offsets"])
    return {"Y": b.linear(H, s["Wd"], offsets=s["offsets"])}


_PLAIN = {"route": _plain_route, "dispatch": _plain_dispatch, "combine": _plain_combine, "linear": _plain_linear, "experts": _plain_experts}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op, f64 = s["op"], torch.float64
    if op == "route":
        l = torch.nan_to_num(s["logits"].to(f64), nan=-math.inf, posinf=LARGEST, neginf=-math.inf)
        at = l.argsort(dim=1, descending=True, stable=True)[:, :s["k"]]
        p = l.softmax(1) if not s["renorm"] else torch.zeros_like(l).scatter_(1, at, l.gather(1, at).softmax(1))
        w = p.gather(1, at)
        out = {"expert": None, "weight": w}
        if s["backward"]:
            up = torch.zeros_like(l).scatter_(1, at, s["dweight"].to(f64))
            out["dlogits"] = p * (up - (p * up).sum(1, keepdim=True))
        return out
    if op == "dispatch":
        offsets, slot, source = (v.cpu() for v in _order(s["ids"], s["E"]))
        Xs = torch.zeros((s["T"] * s["k"], s["d"]), dtype=f64, device=DEV)
        end = int(offsets[-1])
        Xs[:end] = s["X"].to(f64)[(source[:end].long() // s["k"]).to(DEV)]
        out = {"offsets": None, "slot": None, "source": None, "Xs": Xs}
        if s["backward"]:
            token = (source[:end].long() // s["k"]).to(DEV)
            out["dX"] = torch.zeros((s["T"], s["d"]), dtype=f64, device=DEV).index_add_(0, token, s["dXs"][:end].to(f64))
        return out
    if op == "combine":
        Y = s["R"].to(f64).clone() if s["residual"] else torch.zeros((s["T"], s["d"]), dtype=f64, device=DEV)
        Ys, w = s["Ys"].to(f64), s["weight"].to(f64)
        dYs, dw = torch.zeros_like(Ys), torch.zeros_like(w)
        for j in range(s["k"]):
            t = (s["slot"][:, j] >= 0).nonzero().reshape(-1)
            r = s["slot"][t, j].long()
            Y[t] += w[t, j, None] * Ys[r]
            if s["backward"]:
                dYs[r] = w[t, j, None] * s["dY"][t].to(f64)
                dw[t, j] = (s["dY"][t].to(f64) * Ys[r]).sum(1)
        return {"Y": Y, "dYs": dYs, "dweight": dw} if s["backward"] else {"Y": Y}
    fn = {"silu": lambda x: x * torch.sigmoid(x), "gelu_tanh": lambda x: x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)),
          "relu": lambda x: torch.relu(x), "none": lambda x: x}[s["act"]]
    if op == "linear":
        X = s["X"].to(f64)
        zero = torch.zeros(s["N"], dtype=f64, device=DEV)
        Y = fn(torch.addmm(s["b"].to(f64) if s["bias"] else zero, X, s["W"].to(f64).t()))
        if s["glu"]:
            Y = Y * torch.addmm(s["bv"].to(f64) if s["bias"] else zero, X, s["V"].to(f64).t())
        return {"Y": Y + s["R"].to(f64) if s["residual"] else Y}
    Y = torch.zeros(s["X"].shape, dtype=f64, device=DEV)
    edge = s["offsets"].tolist()
    for e in range(s["E"]):
        x = s["X"][edge[e]:edge[e + 1]].to(f64)
        if len(x):
            Y[edge[e]:edge[e + 1]] = (fn(x @ s["Wg"][e].to(f64).t()) * (x @ s["Wu"][e].to(f64).t())) @ s["Wd"][e].to(f64).t()
    return {"Y": Y}
