"""Rows of the layer norm at the end of what fp32 holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

E4M3 = torch.float8_e4m3fn


@pytest.mark.parametrize("rows,d", [(2, 40), (2, 300), (3, 520), (700, 40), (400, 2056), (400, 4104), (320, 8208), (2, 20000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_constant_rows_in_8_bits(rows, d, dtype):
    """Nothing is left of a constant row of 2^e (d 2^e is a multiple of 2^(e - 0) below 2^128, and exact), so it is its
    bias: also where 2^e / sqrt(eps) overflows, which no element of the row has to do with."""
    e = 127 - (d - 1).bit_length()
    x = torch.full((rows, d), 2.0 ** e, device="cuda").to(dtype)
    w = torch.linspace(0.5, 2, d, device="cuda").to(dtype)
    b = torch.linspace(-3, 2, d, device="cuda").to(dtype)
    y, scales, _ = P.bakron_layernorm(x, w, b, 1e-30, out_dtype=E4M3)
    s = b.float().abs().max() / 448
    assert torch.all((scales - s).abs() <= 2.0 ** -23 * s)
    # 8 bits: half a step, 2^-4 of the value, or of the least normal one (2^-6)
    back = y.float() * scales[:, None]
    assert torch.all((back - b.float()).abs() <= 1.01 * 2.0 ** -4 * torch.maximum(b.float().abs(), 2.0 ** -6 * s))


@pytest.mark.parametrize("rows,d", [(3, 40), (3, 1000), (3, 11003), (700, 1000), (700, 1001), (640, 11000), (650, 17000), (2, 65535)])
@pytest.mark.parametrize("value", [1000.0, 96.0])
def test_gradient_of_constant_rows(rows, d, value):
    """The mean of a constant row whose sums are exact is the row, so nothing is left of it: dw is 0, and dx is
    rho (g - mean(g)), rho = 1 / sqrt(eps); also beside rows that are not constant."""
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    h = torch.full((rows, d), value, device="cuda")
    dy = torch.randn(rows, d, generator=g, device="cuda")
    w = torch.rand(d, generator=g, device="cuda") + 0.5
    dx, dw, db = P.bakron_layernorm_backward(dy, h, w, 1e-6)
    assert torch.all(dw == 0)
    q = dy.double() * w.double()
    want = 1e3 * (q - q.mean(1, keepdim=True))
    # the mean of g: 75 additions of 2^-24 of its absolute terms; a few roundings
    slack = 1e3 * (2.0 ** -17 * q.abs().mean(1, keepdim=True) + 2.0 ** -21 * q.abs())
    assert torch.all((dx.double() - want).abs() <= slack)
