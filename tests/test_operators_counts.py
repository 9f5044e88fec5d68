"""Rows and columns are counted in 32 bits below the binding: a tensor with more is refused there,
before it is copied, and does not come out as a call of few rows."""
import math

import pytest
import torch

from paper_2608_06291_gb300 import operators


class Shape:
    """A CUDA tensor's shape without its memory."""

    dtype = torch.bfloat16

    def __init__(self, *shape):
        self.shape = shape

    def get_device(self):
        return 0

    def numel(self):
        return math.prod(self.shape)

    def is_contiguous(self):
        return True


@pytest.mark.parametrize("shape", [(2 ** 32, 1), (2 ** 32 + 3, 2), (2, 2 ** 31), (2 ** 16, 2 ** 15, 1), (2 ** 33,)])
def test_too_many(shape):
    with pytest.raises(ValueError):
        operators._rows(Shape(*shape), "x", (torch.bfloat16,), 0)


@pytest.mark.parametrize("shape,rows", [((2 ** 31 - 1, 2), 2 ** 31 - 1), ((2 ** 16, 2 ** 14, 64), 2 ** 30),
                                        ((2 ** 31 - 1,), 1), ((0, 5), 0), ((2 ** 40, 0), 0)])
def test_as_many_as_fit(shape, rows):
    t = Shape(*shape)
    assert operators._rows(t, "x", (torch.bfloat16,), 0) == (t, rows, shape[-1])


@pytest.mark.gpu
def test_the_operators_refuse():
    import paper_2608_06291_gb300 as P
    P.build()
    one = torch.ones(1, 1, device="cuda")
    many = one.expand(2 ** 32, 1)       # without its memory
    w = P.bakron_pack_weight(torch.ones(1, 1, dtype=torch.uint8, device="cuda"), one, one * 0, 1)
    for call in (lambda: P.bakron_linear(one.bfloat16().expand(2 ** 32, 1), w),
                 lambda: P.bakron_rmsnorm(many, one[0]), lambda: P.bakron_rmsnorm_backward(many, many, one[0]),
                 lambda: P.bakron_token_logprobs(many), lambda: P.bakron_token_logprobs_backward(many, None, one, None)):
        with pytest.raises(ValueError):
            call()
