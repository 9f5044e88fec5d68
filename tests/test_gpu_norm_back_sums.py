"""The sum over the rows in the gradient of the norm's weight: pairwise over the CTAs' parts, so that small
terms beside a large one are not lost one by one.

h = 1 and eps = 0 make rho 1, so dw is the sum of dy over the rows, each row a part of its own.  32
parts join in 5 levels and a part has at most ceil(rows / 32) terms: (5 + ceil(rows / 32)) 2^-24 of the
terms' sizes.  A term of 0.9 * 2^-24 beside 1 vanishes each time it is added alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2, 31, 32, 37, 64, 100])
@pytest.mark.parametrize("d", [1, 33, 1000, 4096, 11003])
@pytest.mark.parametrize("first", [0, 5, -1])
def test_small_terms_beside_a_large_one(rows, d, first):
    import paper_2608_06291_gb300 as P
    P.build()
    h, w = torch.ones(rows, d, device="cuda"), torch.ones(d, device="cuda")
    dy = torch.full((rows, d), 0.9 * 2.0 ** -24, device="cuda")
    dy[first % rows] = 1.0
    dw = P.bakron_rmsnorm_backward(dy, h, w, 0.0)[1].double()
    want = dy.double().sum(0)
    assert torch.all((dw - want).abs() <= (5 + -(-rows // 32)) * 2.0 ** -24 * want)
