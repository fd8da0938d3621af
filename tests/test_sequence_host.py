"""The training device's autograd functions, without a GPU: the operators are
stand-ins.  A second derivative is refused; it would be zero, unnoticed beside
other terms."""
import numpy as np
import pytest
import torch

from paper_2504_13850_gb300 import api, sequence


@pytest.fixture
def operators(monkeypatch):
    """Linear stand-ins: o = v, and dropout that keeps everything."""
    monkeypatch.setattr(api, "attention_forward", lambda q, k, v, **how: (v.clone(), q.sum(3).permute(0, 2, 1)))

    def backward(do, q, k, v, o, lse, grads=None, **how):
        with torch.no_grad():             # the library writes through pointers
            grads[0].zero_(), grads[1].zero_(), grads[2].copy_(do)
        return *grads, torch.zeros_like(how["table"])

    monkeypatch.setattr(api, "attention_backward", backward)
    monkeypatch.setattr(api, "dropout_add", lambda x, r, p, seed, call: x + r)
    monkeypatch.setattr(api, "dropout_grad", lambda dy, p, seed, call: dy.clone())


def test_second_derivatives_are_refused(operators):
    qkv = torch.randn(1, 4, 3, 2, 8, requires_grad=True)
    table = torch.randn(2, 4, requires_grad=True)
    o = sequence.PackedAttention.apply(qkv, table, np.zeros(3, np.uint8), torch.zeros(1, 4, dtype=torch.int32))
    g, = torch.autograd.grad((o ** 2).sum(), qkv, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g + qkv).sum().backward()
    x, r = (torch.randn(3, 8, requires_grad=True) for _ in range(2))
    y = sequence.ResidualDropout.apply(x, r, 0.5, 1, 1)
    g, = torch.autograd.grad((y ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g + x).sum().backward()
