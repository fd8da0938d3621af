"""How attention_backward lays out the gradient that autograd hands it, without a
GPU: what the tensor cores cannot read is copied, nothing else is."""
import pytest
import torch

from paper_2504_13850_gb300 import api

BF, F32 = torch.bfloat16, torch.float32


def wide(t):
    return t.data_ptr() % 16 == 0 and t.stride(3) == 1 and all(
        n == 1 or s >= 8 and s % 8 == 0 for n, s in zip(t.shape[:3], t.stride()[:3]))


def given(name, dtype=BF, D=64):
    x = torch.randn(2, 6, 4, D).to(dtype)
    return {
        "a sum over everything": lambda: torch.ones((), dtype=dtype).expand(2, 6, 4, D),
        "a mean over tokens": lambda: x[:, :1].expand(2, 6, 4, D),
        "a mean over the batch": lambda: x[:1].expand(2, 6, 4, D),
        "one gradient for every head": lambda: x[:, :, :1].expand(2, 6, 4, D),
        "a transposed last dimension": lambda: torch.randn(2, 6, D, 4).to(dtype).transpose(2, 3),
        "an odd offset": lambda: torch.randn(2 * 6 * 4 * D + 1).to(dtype)[1:].view(2, 6, 4, D),
        "odd strides": lambda: torch.randn(2, 6, 4, D + 3).to(dtype)[..., :D],
        "contiguous": lambda: x,
        "heads before tokens": lambda: torch.randn(2, 4, 6, D).to(dtype).transpose(1, 2),
        "part of a projection": lambda: torch.randn(2, 6, 8, D).to(dtype)[:, :, 2:6],
        "a batch of one": lambda: torch.randn(1, 6, 4, D).to(dtype).as_strided((1, 6, 4, D), (3, 4 * D, D, 1)),
    }[name]()


COPIED = ["a sum over everything", "a mean over tokens", "a mean over the batch", "one gradient for every head",
          "a transposed last dimension", "an odd offset", "odd strides"]
KEPT = ["contiguous", "heads before tokens", "part of a projection", "a batch of one"]


@pytest.mark.parametrize("name", COPIED)
def test_what_the_tensor_cores_cannot_read_is_copied(name):
    g = given(name)
    d = api._dense_gradient(torch, g)
    assert not wide(g) and wide(d) and torch.equal(d, g)


@pytest.mark.parametrize("name", KEPT)
def test_what_they_can_read_is_not(name):
    g = given(name)
    assert api._dense_gradient(torch, g) is g


def test_other_types_and_widths_keep_what_the_kernels_take():
    for name in COPIED + KEPT:
        for dtype, D in ((F32, 64), (BF, 20)):
            g = given(name, dtype, D)
            d = api._dense_gradient(torch, g)
            assert d.stride(3) == 1 and torch.equal(d, g)
            assert (d is g) == (g.stride(3) == 1)
    odd = torch.zeros(3, 4)
    assert api._dense_gradient(torch, odd) is odd           # refused further on
