"""bakron_linear's SiLU and GELU in fp32 results keep fp32's accuracy, relative to the result,
for few tokens, for tiles split by columns and for many, on whole and ragged rows.

The value arrives as the bias, in fp32.  silu: CUDA's expf has 2 ulp, the sum and the quotient a
rounding each: 4 * 2^-23.  gelu: erfc's argument x = |v| / sqrt(2) is within 2^-23 of itself, which
moves erfc by at most 2 x^2 + 2 times that; CUDA's erfcf has 4 ulp and the product a rounding:
(v^2 + 7) 2^-23.  1e-36 covers results whose parts leave the normal numbers."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,m", [(1, 8003), (16, 8000), (20, 8000), (20, 8003), (400, 40000), (400, 40003)])
def test_activation(act, rows, m):
    import paper_2608_06291_gb300 as P
    P.build()
    v = torch.cat([torch.linspace(-90, 90, m // 4), torch.linspace(-13, 13, m // 4),
                   torch.linspace(-4, 4, m - 2 * (m // 4))]).float().cuda()
    w = P.bakron_pack_weight(torch.ones(m, 1, dtype=torch.uint8, device="cuda"), torch.ones(m, 1, device="cuda"),
                             torch.zeros(m, 1, device="cuda"), 1)
    x = torch.zeros(rows, 1, dtype=torch.bfloat16, device="cuda")
    y = P.bakron_linear(x, w, bias=v, activation=act, out_dtype=torch.float32, sync=True).double()
    v = v.double()
    if act == "silu":
        want, rel = v / (1 + torch.exp(-v)), 4 * torch.ones_like(v)
    else:
        want, rel = 0.5 * v * torch.special.erfc(-v / 2 ** 0.5), v.square() + 7
    assert torch.all((y - want[None]).abs() <= (rel * 2.0 ** -23 * want.abs())[None] + 1e-36)
