"""The mean probabilities of the balance loss where they are counts: every token is seen exactly once."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS24 = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 3], ids=["dense", "odd-pitch"])
@pytest.mark.parametrize("T", [1, 63, 1025, 20011, 65537])
@pytest.mark.parametrize("E", [1, 8, 13, 32, 60, 128, 256, 300, 512, 1000])
def test_every_token_counts_once(T, E, pad, dtype):
    """One finite logit a token: its probability is 1, the others 0, and the sums are whole numbers below 2^24, exact in f32 in any
    order.  share = sum x (1 / n): two roundings.  A token more or less would move a share by 1 / n, far above that."""
    g = torch.Generator(device=DEV)
    g.manual_seed(T * 7 + E)
    base = torch.full((T, E + pad), 5.0, dtype=dtype, device=DEV)
    logits = base[:, pad:]
    logits.fill_(float("-inf"))
    at = torch.randint(0, E, (T,), generator=g, device=DEV)
    at[T // 2:] = (at[T // 2:] * at[T // 2:]) % E                      # uneven loads
    logits[torch.arange(T, device=DEV), at] = torch.randn(T, generator=g, device=DEV).to(dtype)
    ids = torch.stack((at, torch.full_like(at, -1)), 1).int()
    ids[torch.rand(T, generator=g, device=DEV) < 0.1] = -1             # padding
    used = ids[:, 0] >= 0
    n = int(used.sum())
    want = torch.bincount(at[used], minlength=E)
    loss, counts, share = b.route_balance(logits, ids)
    assert torch.equal(counts[:E].long(), want) and int(counts[E]) == n
    exact = want.double() / max(n, 1)
    assert bool(((share.double() - exact).abs() <= 2.01 * EPS24 * exact).all())
    # loss = E sum_e f_e P_e: two roundings more a term, a sum of E terms, the last factor's two
    true = E * float((exact * exact / 2).sum())
    assert abs(float(loss) - true) <= (E + 10) * EPS24 * true
