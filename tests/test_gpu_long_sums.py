"""Sums over a hundred thousand terms of one sign and more: the tensor cores cut a sum at each addition, so
in place all the way the results lean toward zero by 2^-24 an addition and more.  They leave the tensor cores every 4096
products (256 additions of up to 2^-23 of the sum so far: 2^-15 at most); after that additions are rounded.  The results' own
roundings (2^-8) have no direction: over N of them the mean is below 4 * 2^-8 / sqrt(3 N).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P


def _lean(got, want):
    rel = (got.double() - want) / want
    return float(rel.mean()), 2.0 ** -15 + 4 * 2.0 ** -8 / (3 * rel.numel()) ** 0.5


@pytest.mark.parametrize("t,m,n", [(400, 131072, 256), (64, 65536, 19456), (8, 65536, 2048), (200, 131072, 128)])
def test_quantised_product(t, m, n):
    g = torch.Generator(device="cuda").manual_seed(t)
    codes = torch.randint(0, 16, (m, n), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.rand(m, 1, generator=g, device="cuda") + 0.5
    w = P.bakron_pack_weight(codes, scales, torch.zeros_like(scales), 15, 0)
    dy = (torch.rand(t, m, generator=g, device="cuda") + 0.5).bfloat16()
    dx = P.bakron_linear_backward(dy, w, sync=True)
    want = torch.zeros(t, n, dtype=torch.float64, device="cuda")
    for i in range(0, m, 8192):
        want += dy[:, i:i + 8192].double() @ (codes[i:i + 8192].double() * scales[i:i + 8192].double())
    lean, most = _lean(dx, want)
    assert abs(lean) <= most


def test_weight_gradient_of_a_million_tokens():
    t, v, d = 1 << 20, 250, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    h = (torch.rand(t, d, generator=g, device="cuda") + 0.5).bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") / 8).bfloat16()
    at = torch.randint(0, 50, (t,), generator=g, device="cuda")      # the others' gradients are of one sign
    c = torch.rand(t, generator=g, device="cuda") + 0.5
    _, _, lse = P.bakron_head_logprobs(h, w, at)
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, c, sync=True)
    want = torch.zeros(v, d, dtype=torch.float64, device="cuda")
    for i in range(0, t, 1 << 17):
        s = slice(i, i + (1 << 17))
        p = torch.softmax(h[s].double() @ w.double().t(), 1)
        want -= (c[s].double()[:, None] * p).t() @ h[s].double()
    lean, most = _lean(dw[50:], want[50:])
    assert abs(lean) <= most


def test_hidden_states_gradient_over_a_large_vocabulary():
    """All other entries of a row of the weight's gradient sum are of one sign where the weight is positive."""
    t, v, d = 300, 1 << 19, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(t, d, generator=g, device="cuda").bfloat16() / 16
    w = (torch.rand(v, d, generator=g, device="cuda") + 0.5).bfloat16()
    at = torch.full((t,), -100, device="cuda")
    _, ent, lse = P.bakron_head_logprobs(h, w, at)
    x = h.double() @ w.double().t()
    p = torch.softmax(x, 1)
    # the entropy's gradient alone, with an entropy so large that all entries are of one sign
    big = torch.full_like(ent, 1e4)
    dh, _ = P.bakron_head_logprobs_backward(h, w, at, lse, None, entropy=big, dentropy=torch.ones_like(ent), weight_grad=False,
                                            sync=True)
    want = -(p * (x - lse.double()[:, None] + 1e4)) @ w.double()
    lean, most = _lean(dh, want)
    assert abs(lean) <= most
