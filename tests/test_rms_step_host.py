"""A step of a device with orthogonalised updates that ends with an error leaves the
device as it was; the operators are plain stand-ins, without a GPU."""
import pytest
import torch

from paper_2504_13850_gb300 import api, sequence


def test_a_step_whose_update_gave_up_changes_nothing(monkeypatch):
    d = sequence.RmsDevice.__new__(sequence.RmsDevice)
    d.head, other = torch.randn(2, 8).requires_grad_(), torch.randn(8).requires_grad_()
    d.matrices, d.momenta, d.matrix_lr, d.momentum, d.weight_decay = [torch.randn(8, 8).requires_grad_()], [torch.randn(8, 8)], 0.1, 0.9, 0.0
    d.opt = torch.optim.SGD([d.head, other], lr=0.1, momentum=0.9)
    x = torch.randn(3, 4, 8)

    def forward(tokens, lengths):
        y = (x * other) @ d.matrices[0].t()
        return y, x.byte(), x.byte()

    def muon_step(params, grads, momenta, lr, momentum, weight_decay):
        with torch.no_grad():
            for p, g, m in zip(params, grads, momenta):
                m.mul_(momentum).add_(g)
                p.sub_(lr * m)

    def gave_up():
        raise api.FedOptimaError("orthogonalize_error: FO_ERR_TIMEOUT")

    monkeypatch.setattr(d, "forward", forward, raising=False)
    monkeypatch.setattr(api, "attention_error", lambda: None)
    monkeypatch.setattr(api, "muon_step", muon_step)
    batch = torch.zeros(3, 4, dtype=torch.int64), torch.tensor([4, 2, 3]), torch.tensor([0, 1, 0])
    held = [*d.matrices, *d.momenta, d.head, other]
    monkeypatch.setattr(api, "orthogonalize_error", gave_up)
    before = [t.detach().clone() for t in held]
    with pytest.raises(api.FedOptimaError, match="TIMEOUT"):
        d.step(*batch)
    assert all(torch.equal(t, b) for t, b in zip(held, before)) and not d.opt.state
    monkeypatch.setattr(api, "orthogonalize_error", lambda: None)
    d.step(*batch)
    assert not any(torch.equal(t, b) for t, b in zip(held, before))
