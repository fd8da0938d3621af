"""The training device's step when a kernel gave up a wait, without a GPU: it
raises before a parameter changes, so that nothing void is kept or uploaded."""
import pytest
import torch

from paper_2504_13850_gb300 import api, sequence


def device(monkeypatch):
    d = sequence.SequenceDevice.__new__(sequence.SequenceDevice)
    d.head = torch.randn(2, 8, generator=torch.Generator().manual_seed(1)).requires_grad_()
    d.params, d.steps = [d.head], 0
    d.opt = torch.optim.SGD(d.params, lr=0.1)
    x = torch.randn(3, 4, 8, generator=torch.Generator().manual_seed(2))
    monkeypatch.setattr(d, "forward", lambda tokens, lengths: x, raising=False)
    return d, (torch.zeros(3, 4, dtype=torch.int64), torch.tensor([4, 2, 3]), torch.tensor([0, 1, 0]))


def test_a_step_whose_kernels_gave_up_changes_nothing(monkeypatch):
    d, batch = device(monkeypatch)
    before = d.head.detach().clone()

    def gave_up():
        raise api.FedOptimaError("attention_error: FO_ERR_TIMEOUT")

    monkeypatch.setattr(api, "attention_error", gave_up)
    with pytest.raises(api.FedOptimaError):
        d.step(*batch)
    assert torch.equal(d.head.detach(), before) and d.steps == 0
    monkeypatch.setattr(api, "attention_error", lambda: None)
    x, loss = d.step(*batch)
    assert d.steps == 1 and not torch.equal(d.head.detach(), before) and x.shape == (3, 4, 8)
