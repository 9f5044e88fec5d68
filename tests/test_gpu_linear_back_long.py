"""bakron_linear_backward where every CTA goes through many blocks: rings that wrap several times, chunks that follow
one another in a warp, sums that pass 4096 products, many tokens by both kernels.  (test_linear_back_cover.py
holds that these sizes are such.)  Bounds as in test_gpu_linear_back_precision.py: an operand's 2^-11, a sum's
additions, one per 16 products and part, and the result's rounding.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

WEIGHTS = [(4099, 11003, 255, 0), (4096, 11008, 15, 0), (11008, 4096, 15, 32), (11008, 4096, 15, 128), (28672, 2176, 7, 128), (28672, 2176, 200, 64)]
TOKENS = [1, 4, 5, 8, 9, 17, 64, 200, 384, 700, 2100]


def _weight(m, n, qmax, group, seed, pow2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    G = n // group if group else 1
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g, device="cuda").float()
    scales = torch.rand(m, G, generator=g, device="cuda") + 0.5
    if pow2:
        scales = torch.exp2(torch.randint(-2, 2, (m, G), generator=g, device="cuda").float())
    W = ((codes.double().view(m, G, -1) - zeros.double()[:, :, None]) * scales.double()[:, :, None]).view(m, n)
    return P.bakron_pack_weight(codes, scales, zeros, qmax, group), W


@pytest.mark.parametrize("m,n,qmax,group", WEIGHTS)
def test_backward(m, n, qmax, group):
    w, W = _weight(m, n, qmax, group, m, False)
    for t in TOKENS:
        dy = torch.randn(t, m, generator=torch.Generator(device="cuda").manual_seed(t), device="cuda").bfloat16()
        dx = P.bakron_linear_backward(dy, w, sync=True)
        want, terms = dy.double() @ W, dy.double().abs() @ W.abs()
        slack = (1.01 * 2.0 ** -11 + (m / 16 + 128) * 2.0 ** -23) * terms + 1.01 * 2.0 ** -8 * want.abs()
        assert torch.all((dx.double() - want).abs() <= slack), t
        assert torch.linalg.norm(dx.double() - want) <= 1.06 * torch.linalg.norm(want.bfloat16().double() - want), t


@pytest.mark.parametrize("m,n,qmax,group", WEIGHTS)
def test_exact(m, n, qmax, group):
    w, W = _weight(m, n, qmax, group, m + 1, True)
    for t in TOKENS:
        dy = torch.randint(-1, 2, (t, m), generator=torch.Generator(device="cuda").manual_seed(t), device="cuda").bfloat16()
        dy[torch.rand(t, m, generator=torch.Generator(device="cuda").manual_seed(t + 1), device="cuda") < 0.5] = 0
        want = dy.double() @ W
        assert float((dy.double().abs() @ W.abs()).max()) < 2 ** 21      # quarters: exact in fp32 in any order
        assert torch.equal(P.bakron_linear_backward(dy, w), want.float().bfloat16()), t


@pytest.mark.parametrize("t", [2, 7, 20, 400, 2100])
def test_offsets_past_32_bits(t):
    """131072 x 16512 codes in 8 bits, 2.16e9 bytes: rows before and behind the 2^31st byte."""
    m, n = 131072, 16512
    g = torch.Generator(device="cuda").manual_seed(t)
    codes = torch.randint(0, 256, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    scales, zeros = torch.rand(m, 1, generator=g, device="cuda") + 0.5, torch.full((m, 1), 128.0, device="cuda")
    w = P.bakron_pack_weight(codes, scales, zeros, 255)
    rows = torch.tensor([0, 1, 127, 128, 65536, 130047, 130048, 131070, 131071], device="cuda")
    dy = torch.zeros(t, m, dtype=torch.bfloat16, device="cuda")
    dy[:, rows] = torch.randn(t, len(rows), generator=g, device="cuda").bfloat16()
    dx = P.bakron_linear_backward(dy, w, sync=True)
    W = (codes[rows].double() - 128) * scales[rows].double()
    want, terms = dy[:, rows].double() @ W, dy[:, rows].double().abs() @ W.abs()
    slack = (1.01 * 2.0 ** -11 + 256 * 2.0 ** -23) * terms + 1.01 * 2.0 ** -8 * want.abs()
    assert torch.all((dx.double() - want).abs() <= slack)
