"""A mixture-of-experts layer through the DaSS path: every expert is a GLU MLP that is calibrated, pruned and run on the
tokens the router sends it.

    layer = ExpertLayer(Wr, Wg, Wu, Wd, k=2, act="silu")      # router [E x d], Wg / Wu [E x I x d], Wd [E x d x I]
    Y = layer.forward(X, residual=X)                            # nothing waits for the device
    layer.calibrate(X); norm = layer.finalize()                 # per expert: the neuron norms over its own tokens
    pruned = layer.prune(alpha=0.5)                             # an ExpertLayer with N:M-pruned experts, same router
    Yp, saved = pruned.forward(X, keep=True)
    dlogits = pruned.router_gradient(dY, saved, balance=0.01)   # what tuning the router around the pruned experts needs
    small = pruned.quantize()                                   # the same experts in 4 bits a weight

All work runs in the CUDA library; the sequence of its calls is what this file adds.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Union

import torch

from . import binding as b


class Routed(NamedTuple):
    """Where the tokens of one batch went: the router's choice and the order by expert."""
    logits: torch.Tensor
    expert: torch.Tensor
    weight: torch.Tensor
    offsets: torch.Tensor
    slot: torch.Tensor
    source: torch.Tensor


class Saved(NamedTuple):
    """What the gradient of a forward pass needs."""
    routed: Routed
    Ys: torch.Tensor


class ExpertLayer:
    """Weights of E experts stacked in one tensor (or one MX4) per projection, and their router.

    With ``rows_in_4_bits`` the rows that meet 4-bit weights are quantised too."""

    def __init__(self, Wr: torch.Tensor, Wg: Union[torch.Tensor, b.MX4], Wu: Union[torch.Tensor, b.MX4], Wd: Union[torch.Tensor, b.MX4], k: int,
                 act: str = "silu", renormalise: bool = True, router_bias: Optional[torch.Tensor] = None, rows_in_4_bits: bool = False):
        E, I, d = Wg.shape
        if Wu.shape != (E, I, d) or Wd.shape != (E, d, I) or Wr.shape != (E, d):
            raise ValueError("Wr [E x d], Wg and Wu [E x I x d] and Wd [E x d x I] must agree in E, I and d")
        self.E, self.I, self.d, self.k = E, I, d, int(k)
        self.Wr, self.Wg, self.Wu, self.Wd, self.router_bias = Wr, Wg, Wu, Wd, router_bias
        self.act, self.renormalise = b.ACT_BY_NAME[act], bool(renormalise)
        self.quantized, self.rows_in_4_bits = isinstance(Wg, b.MX4), bool(rows_in_4_bits)
        if not self.quantized == isinstance(Wu, b.MX4) == isinstance(Wd, b.MX4):
            raise ValueError("all three projections must be in 4 bits, or none")
        if self.rows_in_4_bits and not self.quantized:
            raise ValueError("rows in 4 bits go with weights in 4 bits")
        self.sumsq = torch.zeros((E, I), dtype=torch.float64, device=Wg.device)
        self.norm = torch.zeros((E, I), dtype=torch.float32, device=Wg.device)
        self._finalized = False
        self._calib_ws: Optional[torch.Tensor] = None
        self._calib_status = torch.zeros(1, dtype=torch.int32, device=Wg.device)     # the worst of all calibration calls since reset()

    # ------------------------------------------------------------------ forward
    def route(self, X: torch.Tensor, among: Optional[torch.Tensor] = None) -> Routed:
        """The router's choice; with ``among`` (truth values [T x E]) only among the experts it names.

        The logits are stored in X's dtype, as a projection's output is: for a bf16 layer two experts closer than one part in
        256 can tie, and then the lower index is chosen."""
        logits = b.linear(X, self.Wr, bias=self.router_bias)
        if among is not None:
            logits = logits.masked_fill(~among, float("-inf"))
        expert, weight = b.route_topk(logits, self.k, renormalise=self.renormalise)
        return Routed(logits, expert, weight, *b.expert_sort(expert, self.E))

    def forward(self, X: torch.Tensor, residual: Optional[torch.Tensor] = None, routed: Optional[Routed] = None, keep: bool = False):
        """Y[t] = residual[t] + sum_j weight[t,j] * expert_j(X[t]).  With ``keep`` also what router_gradient needs.

        An expert's intermediate H and its output are rounded to X's dtype between the calls, as a dense layer's are: in bf16
        an expert's output is 2.3e-3 off the exact one, of which the last rounding alone is 1.7e-3.  Experts in 4 bits take
        bfloat16 tokens alone, also where rows_in_4_bits quantises them."""
        if self.quantized and X.dtype != torch.bfloat16:
            raise TypeError(f"experts in 4 bits take bfloat16 tokens, not {X.dtype}")
        r = routed if routed is not None else self.route(X)
        Xs = b.expert_gather(X, r.slot, r.offsets, Xs=b.mx4_rows(r.slot.numel(), self.d, X.device) if self.quantized else None)
        H = b.mx4_rows(Xs.shape[0], self.I, X.device) if self.quantized else None
        H = self._product(Xs, self.Wg, r.offsets, act=self.act, W_up=self.Wu, Y=H)
        Ys = self._product(H, self.Wd, r.offsets)
        Y = b.expert_combine(Ys, r.slot, r.weight, residual=residual)
        return (Y, Saved(r, Ys)) if keep else Y

    def _product(self, X: torch.Tensor, W: Union[torch.Tensor, b.MX4], offsets: torch.Tensor, **options) -> torch.Tensor:
        if not self.quantized:
            return b.linear(X, W, offsets=offsets, **options)
        return b.linear_mx4(b.mx4_quantize(X) if self.rows_in_4_bits else X, W, offsets=offsets, **options)

    # ------------------------------------------------------------------ the router's balance and gradient
    def balance(self, routed: Routed):
        """(loss, counts, share): the balance loss of a batch's choices (1 for even loads, E for one expert alone), the choices
        per expert and, last, the tokens that have any, and the mean probability of each expert."""
        return b.route_balance(routed.logits, routed.expert)

    def router_gradient(self, dY: torch.Tensor, saved: Saved, balance: float = 0.0, counts: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Gradient of the router's logits [T x E] from that of the layer's output, the experts held fixed, plus ``balance``
        times that of the balance loss.  ``counts`` are the batch's own unless given (summed over several batches or ranks).
        For bfloat16 logits the two are each rounded to bfloat16, as every gradient of them is: the first before the second is
        added, the sum once more.
        (Through the router's product it is dWr = dlogits^T X, and dlogits Wr for the layer's input.)"""
        r = saved.routed
        _, dweight = b.expert_combine_backward(dY, saved.Ys, r.slot, r.weight, want_rows=False)
        dlogits = b.route_topk_backward(r.logits, r.expert, dweight, renormalise=self.renormalise)
        if balance:
            if counts is None:
                _, counts, _ = self.balance(r)
            factor = torch.full((), float(balance), dtype=torch.float32, device=dlogits.device)
            b.route_balance_backward(r.logits, r.expert, counts, dloss=factor, add=dlogits, dlogits=dlogits)
        return dlogits

    # ------------------------------------------------------------------ 4-bit weights
    def quantize(self, rows_in_4_bits: bool = False) -> "ExpertLayer":
        """The layer with its experts in microscaled 4-bit values (a quarter of the bytes; what pruning set to zero stays zero).
        With ``rows_in_4_bits`` tokens and intermediate rows are quantised as well, which the 4-bit tensor pipe needs.
        For bfloat16 layers: the products with 4-bit weights take bfloat16 rows and give bfloat16."""
        if self.quantized:
            raise RuntimeError("the experts are in 4 bits already")
        if self.Wg.dtype != torch.bfloat16:
            raise TypeError(f"a layer of {self.Wg.dtype} cannot be quantised: products with 4-bit weights take bfloat16 rows")
        out = ExpertLayer(self.Wr, *(b.mx4_quantize(W) for W in (self.Wg, self.Wu, self.Wd)), self.k, renormalise=self.renormalise,
                          router_bias=self.router_bias, rows_in_4_bits=rows_in_4_bits)
        out.act = self.act
        return out

    # ------------------------------------------------------------------ calibration and pruning
    def reset(self) -> None:
        self.sumsq.zero_()
        self._calib_status.zero_()

    def calibrate(self, X: torch.Tensor, routed: Optional[Routed] = None) -> list:
        """Adds a batch of tokens to every expert's neuron sums: the tokens routed to an expert are its calibration set.
        Returns the tokens per expert.  (Waits for the device once: the calibration calls take their sizes on the host.)"""
        if self.quantized:
            raise RuntimeError("calibrate the layer before its experts are quantised")
        r = routed if routed is not None else self.route(X)
        Xs = b.expert_gather(X, r.slot, r.offsets)
        edges = r.offsets.tolist()
        most = max(hi - lo for lo, hi in zip(edges, edges[1:]))
        if most and (self._calib_ws is None or self._calib_ws.numel() < b.calib_workspace_bytes(most, self.d, self.I, X.dtype)):
            self._calib_ws = b.calib_workspace(most, self.d, self.I, X.dtype, X.device)
        for e, (lo, hi) in enumerate(zip(edges, edges[1:])):
            if hi > lo:
                b.calib_accumulate(Xs[lo:hi], self.Wg[e], self.Wu[e], self.act, self.sumsq[e], self._calib_ws)
                # the next call clears the workspace's status word, and a larger workspace may replace it
                torch.maximum(self._calib_status, self._calib_ws[:4].view(torch.int32), out=self._calib_status)
        return [hi - lo for lo, hi in zip(edges, edges[1:])]

    def finalize(self) -> torch.Tensor:
        """norm[e, i]: neuron i's norm over expert e's tokens (0 for an expert that none reached)."""
        b.norm_finalize(self.sumsq.view(-1), self.norm.view(-1))
        self._finalized = True
        return self.norm

    def prune(self, alpha: float = 0.5, n_keep: int = 2, m: int = 4) -> "ExpertLayer":
        """A layer with every expert's projections pruned N:M by the norms of the last finalize(): Eq. 4 with ``alpha`` on
        gate and up, Eq. 5 on down.  An expert that had no tokens then has no norms: it is pruned by magnitude alone."""
        if self.quantized:
            raise RuntimeError("prune the layer before its experts are quantised")
        if not self._finalized:
            raise RuntimeError("prune() needs the norms of a finalize()")
        out = ExpertLayer(self.Wr, torch.empty_like(self.Wg), torch.empty_like(self.Wu), torch.empty_like(self.Wd), self.k,
                          renormalise=self.renormalise, router_bias=self.router_bias)
        out.act = self.act
        seen = (self.norm > 0).any(dim=1, keepdim=True)
        norm = torch.where(seen, self.norm, torch.ones_like(self.norm))
        for e in range(self.E):
            for W, P, axis, power in ((self.Wg, out.Wg, b.AXIS_ROWS, alpha), (self.Wu, out.Wu, b.AXIS_ROWS, alpha), (self.Wd, out.Wd, b.AXIS_COLS, 1.0)):
                b.prune_nm(W[e], norm[e], axis, power, n_keep, m, axis, W_pruned=P[e], want_mask=False, want_compressed=False)
        return out

    def check(self) -> None:
        """Raises if a bounded device-side wait gave up in any calibration call since reset(), or in any pruning or product
        that has not been reported yet (synchronises the stream)."""
        b.calib_status(self._calib_status)
        b.prune_status()
        b.linear_status()
