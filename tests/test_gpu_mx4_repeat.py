"""Large products with 4-bit weights, again and again with the caches in another state: the rings go round many times, and
every run has the same bits, which are right."""
import pytest
import torch

import test_gpu_mx4 as t
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
RUNS = 40


def _stir(i):
    torch.empty((1 + 13 * (i % 5)) << 22, dtype=torch.uint8, device=DEV).fill_(i)
    if i % 3 == 0:
        torch.cuda._sleep(1000 * i)


@t.forms
@pytest.mark.parametrize("T,K,N,glu,residual", [(2048, 4096, 11008, False, True), (1024, 2048, 14336, True, False), (512, 14336, 4096, False, True),
                                                (300, 8200, 9000, False, False), (130, 4096, 14336, True, True), (8, 4096, 14336, True, True),
                                                (3, 14336, 4096, False, True)])
def test_every_run_has_the_right_bits(T, K, N, glu, residual, both4):
    X = t._randn((T, K), 1)
    rows16 = not both4 and b.linear_mx4_workspace_bytes(T, K, N, has_up=glu) > 0
    X = b.mx4_quantize(X) if both4 else X
    W, V = t._normal_mx4(N, K, 2), t._normal_mx4(N, K, 3) if glu else None
    R = t._randn((T, N), 4) if residual else None
    act = "silu" if glu else "none"
    run = lambda: b.linear_mx4(X, W, act=t.ACTS[act], W_up=V, residual=R)                             # noqa: E731
    first = run()
    want, bound = t._on_device(X, W, V, None, None, R, act, rows16)
    assert bool(((first.double() - want).abs() <= bound).all())
    for i in range(RUNS):
        _stir(i)
        Y = run()
        assert torch.equal(Y, first), f"run {i}: {int((Y != first).sum())} values differ"
    b.linear_status()


@t.forms
def test_every_run_over_experts_has_the_right_bits(both4):
    G, K, N = 8, 2048, 7168
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    ids = torch.topk(torch.randn((1500, G), generator=g, device=DEV), 2, dim=1).indices.int()
    offsets, _, _ = b.expert_sort(ids, G)
    X = t._randn((3000, K), 1)
    X = b.mx4_quantize(X) if both4 else X
    stack = lambda s: [t._normal_mx4(N, K, s + e) for e in range(G)]                                  # noqa: E731
    W, V = stack(10), stack(30)
    join = lambda q: b.MX4(torch.stack([m.codes for m in q]), torch.stack([m.scales for m in q]), K)  # noqa: E731
    Wj, Vj = join(W), join(V)
    run = lambda: b.linear_mx4(X, Wj, act=b.ACT_SILU, W_up=Vj, offsets=offsets)                       # noqa: E731
    first = run()
    edges = offsets.tolist()
    whole = b.mx4_dequantize(X, torch.float32) if both4 else X
    for e in range(G):
        lo, hi = edges[e], edges[e + 1]
        rows = b.mx4_quantize(whole[lo:hi]) if both4 else whole[lo:hi]
        want, bound = t._on_device(rows, W[e], V[e], None, None, None, "silu", False)
        assert bool(((first[lo:hi].double() - want).abs() <= bound).all()), e
    for i in range(RUNS):
        _stir(i)
        Y = run()
        assert torch.equal(Y, first), f"run {i}: {int((Y != first).sum())} values differ"
    b.linear_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_every_run_of_the_balance_loss_has_the_same_bits(dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    logits = torch.randn((65536, 128), generator=g, device=DEV).to(dtype)
    ids = torch.topk(logits.float(), 8, dim=1).indices.int()
    first = b.route_balance(logits, ids)
    d = b.route_balance_backward(logits, ids, first[1])
    p = torch.softmax(logits.double(), 1)
    f = torch.bincount(ids.reshape(-1).long(), minlength=128).double() / (65536 * 8)
    assert abs(float(first[0]) - 128 * float((f * p.mean(0)).sum())) < 1e-5 and bool((first[2].double() - p.mean(0)).abs().max() < 1e-7)
    for i in range(RUNS):
        _stir(i)
        again = b.route_balance(logits, ids)
        assert all(torch.equal(x, y) for x, y in zip(again, first)) and torch.equal(b.route_balance_backward(logits, ids, again[1]), d)
