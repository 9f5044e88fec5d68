"""bakron_linear's operands are the integers c - z themselves, however many tokens there are: what
the codes hold beside their zero is summed, and nothing that would have to cancel.

Tolerances: products of exact operands; a tensor core adds 16 (or 32) of them to a running sum
and cuts at about 2^-23 of the largest term, so n / 16 steps and the fp32 sums over groups
and parts stay within (n / 16 + 64) 2^-22 A, A = sum |s (c - z) x|."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS = [1, 16, 17, 64, 300]


def _tokens(rows, n, sign, seed):
    """e4m3 over its whole range, so that no sum of a token's values fits 24 bits; of one sign or both."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.exp2(torch.rand(rows, n, generator=g, device="cuda") * 17 - 9).clamp(max=448)
    if not sign:
        x *= torch.randint(0, 2, (rows, n), generator=g, device="cuda") * 2 - 1
    return x.to(torch.float8_e4m3fn)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("qmax", [1, 3, 6, 15])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("sign", [False, True])
def test_codes_at_their_zero_give_zero(rows, qmax, group, sign):
    import paper_2608_06291_gb300 as P
    P.build()
    m, n = 200, 2048
    G = n // group if group else 1
    g = torch.Generator(device="cuda").manual_seed(rows + qmax)
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g, device="cuda").float()
    codes = zeros.repeat_interleave(n // G, 1).to(torch.uint8)
    w = P.bakron_pack_weight(codes, torch.rand(m, G, generator=g, device="cuda") + 0.5, zeros, qmax, group)
    y = P.bakron_linear(_tokens(rows, n, sign, 1), w, out_dtype=torch.float32, sync=True)
    assert torch.all(y == 0)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("qmax", [1, 3, 15])
@pytest.mark.parametrize("group", [0, 96, 128])
@pytest.mark.parametrize("sign", [False, True])
@pytest.mark.parametrize("zero", ["low", "high", "any"])
def test_few_codes_beside_their_zero(rows, qmax, group, sign, zero):
    import paper_2608_06291_gb300 as P
    P.build()
    m, n = 130, 1920
    G = n // group if group else 1
    g = torch.Generator(device="cuda").manual_seed(rows + qmax + G)
    zeros = {"low": torch.zeros(m, G), "high": torch.full((m, G), float(qmax)),
             "any": torch.randint(0, qmax + 1, (m, G), generator=torch.Generator().manual_seed(G)).float()}[zero].cuda()
    zz = zeros.repeat_interleave(n // G, 1).to(torch.uint8)
    other = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    codes = torch.where(torch.rand(m, n, generator=g, device="cuda") < 1 / 300, other, zz)
    scales = (0.5 + torch.rand(m, G, generator=g, device="cuda")) * 0.1
    x = _tokens(rows, n, sign, 2)
    y = P.bakron_linear(x, P.bakron_pack_weight(codes, scales, zeros, qmax, group), out_dtype=torch.float32, sync=True)
    W = scales.double().repeat_interleave(n // G, 1) * (codes.double() - zz.double())
    x64 = x.to(torch.float32).double()
    assert torch.all((y.double() - x64 @ W.T).abs() <= (n / 16 + 64) * 2.0 ** -22 * (x64.abs() @ W.abs().T))
