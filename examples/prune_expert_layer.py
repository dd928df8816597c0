"""Prunes the experts of a mixture-of-experts layer 2:4 by the norms over each expert's own tokens, then tunes the router
around the pruned experts towards the dense layer's output.  Synthetic weights and tokens.

    python examples/prune_expert_layer.py [tokens] [experts] [d] [d_int]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2405_01943_b200.experts import ExpertLayer  # noqa: E402


def main(T: int = 4096, E: int = 8, d: int = 1024, I: int = 2816, k: int = 2, steps: int = 20) -> float:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    X = rand(T, d)
    X[:, :8] *= 10.0                                                        # a few outlier channels
    X = X.bfloat16()
    weights = [(rand(*s) * 0.02).bfloat16() for s in ((E, I, d), (E, I, d), (E, d, I))]
    router = rand(E, d) * 0.02

    dense = ExpertLayer(router.bfloat16(), *weights, k=k)
    target = dense.forward(X)
    dense.reset()
    tokens = dense.calibrate(X)
    dense.finalize()
    pruned = dense.prune(alpha=0.5)

    # Gradient descent on the router, each token held to the experts that the dense layer sends it to, with backtracking.
    among = torch.zeros((T, E), dtype=torch.bool, device="cuda").scatter_(1, dense.route(X).expert.long(), True)
    size, before, best, direction = 1e-2, None, None, None
    for step in range(steps + 1):
        Y, saved = pruned.forward(X, routed=pruned.route(X, among), keep=True)
        error = Y.float() - target.float()
        loss = float(error.square().mean() / target.float().square().mean())
        before = loss if before is None else before
        if best is None or loss < best[0]:
            best = (loss, router)
            dlogits = pruned.router_gradient((error * (2.0 / T)).bfloat16(), saved)
            grad = dlogits.float().t() @ X.float()
            direction = grad * (router.norm() / grad.norm().clamp_min(1e-20))
        else:
            size *= 0.5
        router = best[1] - size * direction
        pruned.Wr = router.bfloat16()
    loss, router = best
    pruned.Wr = router.bfloat16()
    pruned.check()
    print(f"{E} experts of {d} x {I}, top-{k}; tokens per expert {min(tokens)} .. {max(tokens)} of {T * k}")
    print(f"2:4 pruned, relative squared error of the layer's output: {before:.4f}; after {steps} steps on the router: {loss:.4f}")
    return before - loss


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:]))
