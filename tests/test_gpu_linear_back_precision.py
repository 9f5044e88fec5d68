"""bakron_linear_backward errs by its result's rounding: what its operands lose is far below.

Up to 8 tokens c - z is exact and dy s is kept to 2^-15 of itself.  Above, s (c - z) is rounded to the 11 bits
of fp16 (2^-11; the result to 8 bits, 2^-8) and dy is exact.  Independent roundings add in squares: over
results of many terms the norm of the error is sqrt(1 + 2^-6), 1.008, of the norm of the
exact result's rounding, where operands in bf16 made it 1.35.  Of 4000 and more values both norms are within 4 / sqrt(2 4000) = 4.5% of
what they are on average: 1.06.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P


@pytest.mark.parametrize("m,n,qmax,group", [(1000, 4096, 15, 0), (1000, 4096, 15, 128), (777, 4128, 7, 32), (1000, 4096, 255, 0),
                                            (1000, 4224, 200, 96)])
@pytest.mark.parametrize("t", [1, 3, 4, 5, 8, 9, 17, 64, 200, 384, 520])
def test_error_is_the_results(t, m, n, qmax, group):
    g = torch.Generator(device="cuda").manual_seed(t + m + n + qmax)
    G = n // group if group else 1
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g, device="cuda").float()
    scales = torch.exp(torch.randn(m, G, generator=g, device="cuda")) * 1e-2
    W = ((codes.double().view(m, G, -1) - zeros.double()[:, :, None]) * scales.double()[:, :, None]).view(m, n)
    dy = (torch.randn(t, m, generator=g, device="cuda") * torch.exp(2 * torch.randn(t, 1, generator=g, device="cuda"))).bfloat16()
    dx = P.bakron_linear_backward(dy, P.bakron_pack_weight(codes, scales, zeros, qmax, group), sync=True)
    want = dy.double() @ W
    rounding = (want.bfloat16().double() - want).norm(dim=1)
    assert torch.linalg.norm((dx.double() - want)) <= 1.06 * torch.linalg.norm(rounding)
    # and of each token by itself
    assert torch.all((dx.double() - want).norm(dim=1) <= 1.06 * rounding)


@pytest.mark.parametrize("qmax", [15, 255])
@pytest.mark.parametrize("t", [1, 8, 40, 400])
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1.0, 1e12, 1e30])
def test_any_magnitude(t, qmax, size):
    """Gradients and scales of any size, tokens and rows of different sizes in one call."""
    m, n = 300, 512
    g = torch.Generator(device="cuda").manual_seed(t + qmax)
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    zeros = torch.randint(0, qmax + 1, (m, 1), generator=g, device="cuda").float()
    scales = torch.exp(2 * torch.randn(m, 1, generator=g, device="cuda")) * min(size, 1e15)
    W = (codes.double() - zeros.double()) * scales.double()
    dy = torch.randn(t, m, generator=g, device="cuda") * torch.exp(3 * torch.randn(t, 1, generator=g, device="cuda"))
    dy = (dy / max(size, 1e-15)).bfloat16()
    dy[0, ::3] *= 2.0 ** -12
    dx = P.bakron_linear_backward(dy, P.bakron_pack_weight(codes, scales, zeros, qmax, 0), sync=True)
    want, terms = dy.double() @ W, dy.double().abs() @ W.abs()
    slack = (1.01 * 2.0 ** -11 + (m / 16 + 128) * 2.0 ** -23) * terms + 1.01 * 2.0 ** -8 * want.abs() + 1e-37
    assert torch.all((dx.double() - want).abs() <= slack)
