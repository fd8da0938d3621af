"""The autograd functions of devices with root-mean-square norms, without a GPU:
the operators are plain stand-ins.  A second derivative is refused, and a step
whose attention kernels gave up a wait changes nothing."""
import pytest
import torch

from paper_2504_13850_gb300 import api, sequence


@pytest.fixture
def operators(monkeypatch):
    """Linear stand-ins: lookup, and norms that only scale."""
    def norm(x, residual, weight):
        with torch.no_grad():
            s = x if residual is None else x + residual
            return s * weight, s, s.sum(-1)

    def grad(dy, ds, s, weight, r):
        with torch.no_grad():
            dx = dy * weight if ds is None else dy * weight + ds
            return dx, (dy * s).reshape(-1, s.shape[-1]).sum(0)

    monkeypatch.setattr(api, "embedding", lambda ids, table, scale, dtype: (table.detach()[ids] * scale))
    monkeypatch.setattr(api, "embedding_grad",
                        lambda dout, ids, vocab, scale, dtype: torch.zeros(vocab, dout.shape[-1]).index_add_(0, ids, dout * scale))
    monkeypatch.setattr(api, "rms_norm", norm)
    monkeypatch.setattr(api, "rms_norm_grad", grad)
    monkeypatch.setattr(api, "rms_norm_8bit", lambda x, r, w, with_y: (x.byte(), x.byte()[..., :1], *norm(x, r, w)))


def test_gradients_reach_every_input(operators):
    table, ids = torch.randn(6, 4, requires_grad=True), torch.tensor([1, 5, 1])
    x, res, w = torch.randn(3, 4, requires_grad=True), torch.randn(3, 4, requires_grad=True), torch.randn(4, requires_grad=True)
    e = sequence.TokenEmbedding.apply(table, ids, 2.0)
    y, s = sequence.AddNorm.apply(x, e, w)
    z, q, scales = sequence.UploadNorm.apply(sequence.Norm.apply(y, w), s + res, w)
    assert not q.requires_grad and not scales.requires_grad
    z.pow(2).sum().backward()
    E = (table.detach()[ids] * 2.0).requires_grad_()
    X, R, Wt = (t.detach().clone().requires_grad_() for t in (x, res, w))
    S = X + E
    ((S * Wt * Wt + S + R) * Wt).pow(2).sum().backward()
    assert torch.allclose(x.grad, X.grad) and torch.allclose(res.grad, R.grad) and torch.allclose(w.grad, Wt.grad)
    assert torch.allclose(table.grad, torch.zeros(6, 4).index_add_(0, ids, E.grad * 2.0))


def test_second_derivatives_are_refused(operators):
    ids = torch.tensor([1, 0])
    table, x, w = torch.randn(3, 4, requires_grad=True), torch.randn(2, 4, requires_grad=True), torch.randn(4, requires_grad=True)
    for f in (lambda: (sequence.TokenEmbedding.apply(table, ids, 1.0), table), lambda: (sequence.Norm.apply(x, w), x),
              lambda: (sequence.AddNorm.apply(x, x, w)[0], x), lambda: (sequence.UploadNorm.apply(x, x, w)[0], x)):
        y, leaf = f()
        g, = torch.autograd.grad((y ** 2).sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (g + leaf).sum().backward()


def test_a_step_whose_kernels_gave_up_changes_nothing(monkeypatch):
    d = sequence.RmsDevice.__new__(sequence.RmsDevice)
    d.head = torch.randn(2, 8).requires_grad_()
    d.matrices, d.momenta, d.matrix_lr, d.momentum, d.weight_decay = [d.head], [torch.zeros(2, 8)], 0.1, 0.9, 0.0
    d.opt = torch.optim.SGD([torch.zeros(1, requires_grad=True)], lr=0.1)
    x, calls = torch.randn(3, 4, 8), []
    monkeypatch.setattr(d, "forward", lambda tokens, lengths: (x, x.byte(), x.byte()), raising=False)
    monkeypatch.setattr(api, "muon_step", lambda *a, **kw: calls.append("muon_step"))
    monkeypatch.setattr(api, "orthogonalize_error", lambda: calls.append("orthogonalize_error"))

    def gave_up():
        raise api.FedOptimaError("attention_error: FO_ERR_TIMEOUT")

    monkeypatch.setattr(api, "attention_error", gave_up)
    batch = torch.zeros(3, 4, dtype=torch.int64), torch.tensor([4, 2, 3]), torch.tensor([0, 1, 0])
    with pytest.raises(api.FedOptimaError):
        d.step(*batch)
    assert calls == []
    monkeypatch.setattr(api, "attention_error", lambda: None)
    upload, loss = d.step(*batch)
    assert calls == ["muon_step", "orthogonalize_error"] and len(upload) == 2 and bool(torch.isfinite(loss))
