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
