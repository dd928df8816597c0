"""What ExpertLayer keeps between its calls, on the CPU: the library's calls are stood in for."""
import pytest
import torch

from paper_2405_01943_b200 import binding as b
from paper_2405_01943_b200.experts import ExpertLayer, Routed

E, I, D = 4, 8, 8


def _layer():
    return ExpertLayer(torch.zeros(E, D), torch.zeros(E, I, D), torch.zeros(E, I, D), torch.zeros(E, D, I), 2)


def _routed(counts):
    offsets = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32)
    return Routed(*(torch.zeros(0),) * 3, offsets, torch.zeros(0), torch.zeros(0))


@pytest.fixture
def calibration(monkeypatch):
    """calib_accumulate as it treats the workspace: cleared at the start, then the status of this call."""
    statuses = []

    def accumulate(X, Wg, Wu, act, sumsq, workspace):
        workspace[:4].view(torch.int32).fill_(statuses.pop(0) if statuses else 0)
        sumsq += 1.0

    def status(workspace):
        if int(workspace.view(torch.uint8)[:4].view(torch.int32)):
            raise b.DassError(8, "dass_calib_status")
    monkeypatch.setattr(b, "calib_accumulate", accumulate)
    monkeypatch.setattr(b, "calib_status", status)
    monkeypatch.setattr(b, "calib_workspace_bytes", lambda T, d, I, dtype: 256 * T)
    monkeypatch.setattr(b, "calib_workspace", lambda T, d, I, dtype, device: torch.zeros(256 * T, dtype=torch.uint8))
    monkeypatch.setattr(b, "expert_gather", lambda X, slot, offsets: torch.zeros(64, D))
    monkeypatch.setattr(b, "prune_status", lambda: None)
    monkeypatch.setattr(b, "linear_status", lambda: None)
    return statuses


def test_check_sees_a_timeout_in_any_calibration_call(calibration):
    X = torch.zeros(16, D)
    for batches in ([[8, 0, 0, 0]], [[0, 8, 0, 0], [0, 0, 8, 0]], [[0, 8, 0, 0], [0, 0, 0, 0]], [[0, 0, 0, 8]], [[0, 0, 0, 0], [8, 0, 0, 0], [0, 0, 0, 0], [0, 0, 0, 0]]):
        layer = _layer()
        layer.check()
        for n, batch in enumerate(batches):
            calibration[:] = batch
            layer.calibrate(X, routed=_routed([2 + 4 * n] * E))               # later batches need a larger workspace
        with pytest.raises(b.DassError):
            layer.check()
        with pytest.raises(b.DassError):
            layer.check()                                                     # the sums stay wrong until reset()
        layer.reset()
        layer.check()
        layer.calibrate(X, routed=_routed([1, 0, 2, 0]))
        layer.check()


def test_prune_goes_by_the_last_finalize_alone(calibration, monkeypatch):
    used = []
    monkeypatch.setattr(b, "norm_finalize", lambda sumsq, norm: norm.copy_(sumsq.sqrt()))
    monkeypatch.setattr(b, "prune_nm", lambda W, norm, *a, **k: used.append(norm.clone()))
    X, layer = torch.zeros(16, D), _layer()
    with pytest.raises(RuntimeError):
        layer.prune()                                                         # no norms yet
    layer.calibrate(X, routed=_routed([2, 0, 3, 0]))
    with pytest.raises(RuntimeError):
        layer.prune()                                                         # sums, but still no norms
    assert not used
    norm = layer.finalize()
    assert norm.shape == (E, I) and bool((norm[0] == 1).all()) and bool((norm[1] == 0).all())

    def norms_of_prune():
        used.clear()
        layer.prune()
        assert len(used) == 3 * E
        return torch.stack(used[::3])
    one = torch.ones(E, I)                                                    # experts 1 and 3 had no tokens: magnitude alone
    layer.norm[0], one[0] = 0.5, 0.5
    assert torch.equal(norms_of_prune(), one)
    layer.calibrate(X, routed=_routed([0, 4, 0, 0]))                          # sums of a later batch are not the last finalize's norms
    assert torch.equal(norms_of_prune(), one)
    layer.reset()                                                             # nor does clearing them change those
    assert torch.equal(norms_of_prune(), one)
