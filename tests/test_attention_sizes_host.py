"""Sizes beyond 32 bits are refused by the binding, without a GPU: the library's
fields hold 32, and a size that wraps would name another problem."""
import pytest
import torch

from paper_2504_13850_gb300 import api


class Shape:
    """A device tensor as far as the checks before the call look at it."""
    is_cuda, dtype = True, torch.bfloat16

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)


def spec(q, k):
    return api._attention_spec(torch, q, k, False, 0.0, None, None, None, None, None, None)


@pytest.mark.parametrize("dim", range(4))
def test_sizes_that_wrap(dim):
    for n in (1 << 31, (1 << 32) + 1):
        size = [1, 1, 1, 8]
        size[dim] = n
        with pytest.raises(ValueError, match="2\\^31"):
            spec(Shape(*size), Shape(*size))
    with pytest.raises(ValueError, match="2\\^31"):
        spec(Shape(1, 1, 1, 8), Shape(1, 1, (1 << 32) + 1, 8))
    s = spec(Shape(2, 3, 4, 8), Shape(2, 3, 1, 8))
    assert (s.batch, s.len, s.heads, s.kv_heads, s.head_dim) == (2, 3, 4, 1, 8)
