"""bakron_linear on e4m3 tokens where a part ends in half a stage (an odd number of 128-column
blocks), down to weights of one block, of which every stage is a half one, and with more
tiles a CTA than there are slots for expanded codes; each call several times.

Exact: integer tokens, power-of-two scales and fp32 results, every sum an integer below 2^24
times the scale's unit, so the result has no rounding at all."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# tokens, rows of the weight: tiles of 32, 64, 128 and 192 tokens, at least 4 a CTA, and
# two calls whose few tiles are split by columns
TILES = [(20, 78000), (60, 80000), (500, 22000), (760, 19400), (40, 300), (200, 700)]


@pytest.mark.parametrize("rows,m", TILES)
@pytest.mark.parametrize("n,group", [(32, 0), (32, 32), (96, 32), (128, 0), (128, 64), (129, 0), (300, 0), (384, 128),
                                     (640, 32), (1664, 0)])
@pytest.mark.parametrize("qmax", [3, 15])
def test_exact_sums(rows, m, n, group, qmax):
    import paper_2608_06291_gb300 as P
    P.build()
    g = torch.Generator(device="cuda").manual_seed(rows + n + qmax)
    G = n // group if group else 1
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.exp2(-torch.randint(3, 6, (m, G), generator=g, device="cuda").float())     # units of 2^-5
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g, device="cuda").float()
    lim = 4
    assert n * lim * qmax * 4 < 2 ** 24
    x = torch.randint(-lim, lim + 1, (rows, n), generator=g, device="cuda")
    w = P.bakron_pack_weight(codes, scales, zeros, qmax, group)
    k = n // G
    W = scales.repeat_interleave(k, 1) * (codes.float() - zeros.repeat_interleave(k, 1))
    want = (x.double() @ W.double().T).float()
    xt = x.to(torch.float8_e4m3fn)
    for _ in range(3):
        assert torch.equal(P.bakron_linear(xt, w, out_dtype=torch.float32, sync=True), want)
