"""bakron_head_logprobs_backward of up to 128 tokens errs by its results' rounding: G is kept in two bf16 parts (to 2^-15),
where one alone, a rounding as large as the result's, made the error up to 1.6 times that.

The norm of the error is that of the exact result's rounding, with what the logits (fp32 sums), the exponential and the fp32
sums lose beside it: 2^-13 of the result at most here (logits of some 20, within 50 2^-23 of their absolute terms).  Two norms of
2000 values and more are within 4 / sqrt(2 2000) = 6% of each other.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P


def _data(t, v, d, spread, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(t, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") * (spread / d ** 0.5)).bfloat16()
    at = torch.randint(0, v, (t,), generator=g, device="cuda")
    at[::3] = -100
    return h, w, at, torch.randn(t, generator=g, device="cuda"), torch.randn(t, generator=g, device="cuda")


@pytest.mark.parametrize("t", [1, 2, 7, 31, 32, 33, 64, 100, 128])
@pytest.mark.parametrize("v,d", [(1692, 2000), (4100, 2048), (70001, 2064)])
@pytest.mark.parametrize("spread", [2.5, 6.0])
def test_error_is_the_results(t, v, d, spread):
    h, w, at, g, u = _data(t, v, d, spread, t + v)
    _, ent, lse = P.bakron_head_logprobs(h, w, at)
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u, sync=True)
    lp = h.double() @ w.double().t() - lse.double()[:, None]
    p = lp.exp()
    ok = at >= 0
    gg = torch.where(ok, g, 0.0).double()
    G = -p * (u.double()[:, None] * (lp + ent.double()[:, None]) + gg[:, None])
    G[torch.arange(t, device="cuda")[ok], at[ok]] += gg[ok]
    for got, want in ((dh, G @ w.double()), (dw, G.t() @ h.double())):
        rounding, off = (want.bfloat16().double() - want).norm(), (got.double() - want).norm()
        assert off <= 1.06 * rounding + 2.0 ** -13 * want.norm()
    # a row of dw by itself, of those that matter
    rows = (G.abs().amax(0) > 1e-3 * G.abs().max()).nonzero()[:, 0]
    want = G.t()[rows] @ h.double()
    rounding, off = (want.bfloat16().double() - want).norm(dim=1), (dw[rows].double() - want).norm(dim=1)
    assert torch.all(off <= 1.06 * rounding + 2.0 ** -10 * want.norm(dim=1) * (t > 1) + 2.0 ** -13 * want.norm(dim=1))


@pytest.mark.parametrize("t", [1, 40, 128])
@pytest.mark.parametrize("shift", [0, 1])
def test_strides_and_repeats(t, shift):
    """Unaligned rows, one target for all, either result alone: the same numbers."""
    h, w, at, g, u = _data(t, 1500, 136, 2.5, t)
    at[:] = 7
    _, ent, lse = P.bakron_head_logprobs(h, w, at)
    a = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u, sync=True)
    hb, wb = torch.zeros(t, 137, device="cuda").bfloat16(), torch.zeros(1500, 137, device="cuda").bfloat16()
    hb[:, shift:shift + 136], wb[:, shift:shift + 136] = h, w
    b = P.bakron_head_logprobs_backward(hb[:, shift:shift + 136], wb[:, shift:shift + 136], at, lse, g, entropy=ent, dentropy=u)
    c, _ = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u, weight_grad=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[0], c)
