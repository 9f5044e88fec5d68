"""Infinite logits at the head: as bakron_token_logprobs has them from the logits themselves."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P


def _data(t, v, d):
    g = torch.Generator(device="cuda").manual_seed(t + v)
    h = torch.randn(t, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") * (2.5 / d ** 0.5)).bfloat16()
    return h, w, torch.arange(t, device="cuda") % v


def _same(a, b, slack=1e-4):
    """Equal where either is no finite number, else near (fp32 results of order 10 from the same logits)."""
    fin = torch.isfinite(b)
    assert torch.equal(torch.isfinite(a), fin)
    assert torch.equal(torch.nan_to_num(a[~fin]), torch.nan_to_num(b[~fin])) and torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.all((a[fin] - b[fin]).abs() <= slack)


@pytest.mark.parametrize("t,v", [(5, 300), (70, 3000), (300, 1000)])
def test_logits_of_minus_infinity(t, v):
    h, w, at = _data(t, v, 64)
    w[:, 7] = w[:, 7].abs() + 0.01
    h[2, 7] = -float("inf")             # every logit of this row
    w[v - 1, 9] = -float("inf")         # one logit of each row: -inf, +inf or (row 2: -inf too) by its sign
    h[:, 9] = h[:, 9].abs() + 0.01
    at[1], at[2], at[3] = v - 1, 4, -100
    logits = h.float() @ w.float().t()
    assert torch.isneginf(logits[2]).all() and torch.isneginf(logits[:, v - 1]).all()
    got, want = P.bakron_head_logprobs(h, w, at, sync=True), P.bakron_token_logprobs(logits, at)
    for a, b in zip(got, want):
        _same(a, b)
    assert torch.isneginf(got[0][1]) and torch.isneginf(got[0][2]) and got[1][2] == 0 and torch.isneginf(got[2][2])


def test_logits_of_infinity_and_far_below():
    """+inf gives NaNs; logits below -1e38 are as good as any others."""
    h, w, at = _data(20, 500, 64)
    h[1, 3] = float("inf")
    w[:, 3] = w[:, 3].abs() + 0.01
    h[4] = 0
    h[4, 5], w[:, 5] = -2.0 ** 120, 1
    w[::2, 5] = 1.5      # logits of -1.3e36 and -2e36
    h[5] = 0
    h[5, 5] = -2.0 ** 127      # -1.7e38 and -2.55e38
    logits = h.float() @ w.float().t()
    got = P.bakron_head_logprobs(h, w, at, sync=True)
    logp, entropy, lse = got
    assert torch.isnan(lse[1]) and torch.isnan(entropy[1]) and torch.isnan(logp[1])
    for r in (4, 5):      # 250 equal logits: their logarithm is lost beside them
        assert lse[r] == logits[r].max() and abs(float(entropy[r]) - float(torch.log(torch.tensor(250.0)))) < 1e-4
    assert logp[5] == 0      # (an odd target)


@pytest.mark.parametrize("t", [5, 300])
def test_backward_of_a_row_without_a_logit(t):
    """A row of lse = -inf gets zeros, as from bakron_token_logprobs_backward; the other rows are their own."""
    h, w, at = _data(t, 700, 64)
    w[:, 7] = w[:, 7].abs() + 0.01
    c, u = torch.ones(t, device="cuda"), torch.full((t,), 0.5, device="cuda")
    _, ent, lse = P.bakron_head_logprobs(h, w, at)
    want, _ = P.bakron_head_logprobs_backward(h, w, at, lse, c, entropy=ent, dentropy=u, weight_grad=False)
    h[2, 7] = -float("inf")
    _, ent, lse = P.bakron_head_logprobs(h, w, at)
    assert torch.isneginf(lse[2])
    got, _ = P.bakron_head_logprobs_backward(h, w, at, lse, c, entropy=ent, dentropy=u, weight_grad=False, sync=True)
    assert torch.all(got[2] == 0)
    keep = torch.arange(t, device="cuda") != 2
    assert torch.equal(got[keep], want[keep])
