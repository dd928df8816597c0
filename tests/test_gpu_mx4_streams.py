"""Calls with 4-bit values and the balance loss on other streams, captured, and side by side."""
import pytest
import torch

import test_gpu_streams as streams
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


def _rand(shape, seed, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(BF16)


T, K, N, E = 5, 4096, 14336, 96
CALLS = {
    "mx4_quantize": lambda z, s: b.mx4_quantize(z["X"], stream=s)[:2],
    "mx4_dequantize": lambda z, s: b.mx4_dequantize(b.MX4(z["codes"], z["scales"], K), stream=s),
    "linear_mx4": lambda z, s: b.linear_mx4(z["X"], b.MX4(z["codes"], z["scales"], K), W_up=b.MX4(z["codes"], z["scales"], K), stream=s),
    "route_balance": lambda z, s: b.route_balance(z["logits"], z["ids"], stream=s),
    "route_balance_backward": lambda z, s: b.route_balance_backward(z["logits"], z["ids"], z["counts"], stream=s),
}


@pytest.fixture(scope="module")
def inputs():
    W = b.mx4_quantize(_rand((N, K), 1, 0.02))
    z = {"X": _rand((T, K), 0), "codes": W.codes, "scales": W.scales, "logits": _rand((20000, E), 2),
         "ids": torch.randint(-1, E, (20000, 4), device=DEV, dtype=torch.int32), "counts": torch.ones(E + 1, dtype=torch.int32, device=DEV)}
    assert b.linear_mx4_workspace_bytes(T, K, N, has_up=True) > 0 and b.route_balance_workspace_bytes(20000, E) > 0
    torch.cuda.synchronize()
    return z


@pytest.mark.parametrize("name", CALLS)
def test_released_memory_stays_with_the_calls_stream(monkeypatch, inputs, name):
    outs, made = streams._recorded(monkeypatch, inputs, CALLS[name], torch.cuda.Stream())
    assert made, "the call allocated nothing"
    sizes = sorted({n for _, n in streams._spans(outs)} | {1 << 9, 1 << 12, 1 << 16, 278528})
    outs.clear()
    kept, now = streams._allocated_now(sizes)
    for a in made:
        assert not any(lo <= a < lo + n for lo, n in now), "memory of a call on another stream was handed to the current stream"


@pytest.mark.parametrize("name", CALLS)
def test_a_call_behind_other_work_of_its_stream(inputs, name):
    want = streams._tensors(CALLS[name](inputs, None))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
    got = streams._tensors(CALLS[name](inputs, s))
    junk = [torch.full((278528,), 0x7f, dtype=torch.uint8, device=DEV) for _ in range(100)]
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and len(junk) == 100


def test_two_streams_at_once(inputs):
    """Calls that split rows and calls that add up partial sums, many of each side by side: every one as it is alone."""
    other = dict(inputs, X=_rand((T, K), 7), logits=_rand((20000, E), 8))
    cases = [(name, z) for name in ("linear_mx4", "route_balance", "mx4_quantize") for z in (inputs, other)]
    want = [streams._tensors(CALLS[n](z, None)) for n, z in cases]
    side = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for i, (n, z) in enumerate(cases):
            got.append((i, streams._tensors(CALLS[n](z, side[(i + len(got)) % 3]))))
    torch.cuda.synchronize()
    for i, outs in got:
        assert all(torch.equal(p, q) for p, q in zip(outs, want[i])), cases[i][0]
    b.linear_status()


def test_two_captured_graphs_that_share_a_workspace(inputs):
    """Calls that are ordered may share a workspace, captured or not: replays in turn, on changed inputs."""
    W = b.MX4(inputs["codes"], inputs["scales"], K)
    X1, X2 = _rand((T, K), 3), _rand((T, K), 4)
    l1, l2 = _rand((20000, E), 5), _rand((20000, E), 6)
    ws = torch.empty(max(b.linear_mx4_workspace_bytes(T, K, N, has_up=True), b.route_balance_workspace_bytes(20000, E)), dtype=torch.uint8, device=DEV)
    run = lambda X, l: (b.linear_mx4(X, W, W_up=W, workspace=ws), *b.route_balance(l, inputs["ids"], workspace=ws))       # noqa: E731
    run(X1, l1)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for X, l in ((X1, l1), (X2, l2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(X, l))
        graphs.append(g)
    for seed in (11, 12):
        X1.copy_(_rand((T, K), seed)), X2.copy_(_rand((T, K), seed + 20)), l1.copy_(_rand((20000, E), seed + 40)), l2.copy_(_rand((20000, E), seed + 60))
        for g in graphs + graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for (X, l), out in zip(((X1, l1), (X2, l2)), outs):
            want = (b.linear_mx4(X, W, W_up=W), *b.route_balance(l, inputs["ids"]))
            assert all(torch.equal(p, q) for p, q in zip(out, want))
    b.linear_status()


def test_another_devices_tensors_are_refused(inputs, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in CALLS.values():
        with pytest.raises(ValueError):
            call(inputs, None)
