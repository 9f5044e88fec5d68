"""bakron_linear where a CTA takes several tiles, for every width of a token tile (32 to 192)
and every kind of operand, with whole and half stages, and grids that end inside one.

Exact: integer tokens, power-of-two scales and fp32 results, every sum an integer below 2^24
times the scale's unit, so the result has no rounding at all."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# tokens, rows of the weight: tiles of 32, 64, 128 and 192 tokens, more of them than SMs (152)
TILES = [(20, 28600), (60, 28600), (500, 9700), (760, 9700)]


@pytest.mark.parametrize("rows,m", TILES)
@pytest.mark.parametrize("n,group", [(640, 0), (1050, 0), (640, 128), (1056, 32), (1152, 96), (768, 384)])
@pytest.mark.parametrize("qmax,xtype", [(15, "bf16"), (15, "e4m3"), (255, "bf16")])
def test_exact_sums_over_many_tiles(rows, m, n, group, qmax, xtype):
    import paper_2608_06291_gb300 as P
    P.build()
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    G = n // group if group else 1
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.exp2(-torch.randint(3, 6, (m, G), generator=g, device="cuda").float())     # units of 2^-5
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g, device="cuda").float()
    lim = 4 if qmax < 16 else 1
    assert n * lim * qmax * 4 < 2 ** 24
    x = torch.randint(-lim, lim + 1, (rows, n), generator=g, device="cuda")
    w = P.bakron_pack_weight(codes, scales, zeros, qmax, group)
    xt = x.to(torch.bfloat16 if xtype == "bf16" else torch.float8_e4m3fn)
    y = P.bakron_linear(xt, w, out_dtype=torch.float32, sync=True)
    k = n // G
    W = scales.repeat_interleave(k, 1) * (codes.float() - zeros.repeat_interleave(k, 1))
    want = x.double() @ W.double().T
    assert torch.equal(y.double(), want)
    again = P.bakron_linear(xt, w, out_dtype=torch.bfloat16, sync=True)
    assert torch.equal(again, want.float().bfloat16())
