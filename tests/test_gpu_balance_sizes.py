"""The balance loss at every number of experts around which its kernel's layout or memory changes."""
import pytest
import torch

import expert_reference as eref
import mx4_reference as ref
import test_gpu_balance as t
from paper_2405_01943_b200 import binding as b

pytestmark = pytest.mark.gpu
EDGES = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 679, 680, 681, 682, 683, 684, 1021, 1022, 1023, 1024]


@t.both
@pytest.mark.parametrize("E", EDGES)
def test_numbers_of_experts(E, dtype):
    for T, k in ((3, 1), (40, 5), (420 if E > 256 else 100, 2)):
        logits, ids = t._inputs(T, E, k, dtype, seed=E)
        t._both_ways(logits, ids, dtype)


def test_every_number_of_experts_runs():
    """Loss and counts of one token and of a batch that takes the second kernel, for all E that the call allows."""
    for E in range(1, 1025):
        for T in (1, 20000):
            ids = (torch.arange(T, device="cuda", dtype=torch.int32) % E)[:, None].contiguous()
            loss, counts, share = b.route_balance(torch.zeros((T, E), device="cuda"), ids)
            n = torch.bincount(ids[:, 0].long(), minlength=E)
            assert torch.equal(counts[:E].long(), n) and int(counts[E]) == T
            # even probabilities: the loss is 1 for any loads; each is 1 / E to expf's and the sums' rounding
            assert abs(float(loss) - 1.0) <= 1e-4 and bool(((share * E - 1.0).abs() <= 1e-4).all()), (E, T)
