"""bakron_head_logprobs_backward where the model is sure of the target: 1 - p from 1e-2 to 1e-5.

The target's entry of G is g (1 - p), with all of p from the 64-bit logits.  What the call gets is lse, and
lse = l_t + log(1 + sum of the others' exponentials over the target's) is nearly l_t itself: the target's logit cancels
where the gradient forms it as the forward pass did.  What is left of l_t - lse is lse's rounding (2^-24 |lse|), the
logarithm's and its argument's (2^-23 and 2^-24) and, for the others, the difference of two
logits' errors.  A logit's sums leave the tensor cores every 512 products (32 additions that may lose 2^-23 of the group's
absolute terms a each, and 16 for what a step's terms lose; d / 512 additions outside): 64 2^-23 a.  So 1 - p is off by 2^-23 |lse| + 2^-21,
and by twice 64 2^-23 a of itself.  Other entries are rounded to bf16 (2^-8, with the exponential 1.01 times that); sums and
the result as in the general test: (v / 16 + 96) 2^-23 of the absolute terms, and one rounding.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P


def _data(t, v, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(v, d, generator=g, device="cuda") / d ** 0.5).bfloat16()
    at = torch.randint(0, v, (t,), generator=g, device="cuda")
    rest = 10.0 ** -torch.linspace(2, 5, t, device="cuda")      # 1 - p, about
    logit = math.log(v) + 0.5 + torch.log((1 - rest) / rest)
    own = w[at].float()
    h = torch.randn(t, d, generator=g, device="cuda") + own * (logit / own.square().sum(1))[:, None]
    return h.bfloat16(), w, at


@pytest.mark.parametrize("t,v,d", [(40, 2000, 4096), (300, 1000, 4160), (64, 5021, 8192)])
@pytest.mark.parametrize("entropy", [False, True])
def test_confident_targets(t, v, d, entropy):
    h, w, at = _data(t, v, d, t + v)
    x = h.double() @ w.double().t()
    lse64 = torch.logsumexp(x, 1)
    lp = x - lse64[:, None]
    p = lp.exp()
    here = torch.arange(t, device="cuda")
    others = p.clone()
    others[here, at] = 0
    rest = others.sum(1)      # 1 - p without a cancellation
    assert rest.min() < 3e-5 and rest.max() > 3e-3
    logp, ent, lse = P.bakron_head_logprobs(h, w, at, sync=True)
    ent64 = -torch.special.xlogy(p, p).sum(1)
    g = 0.5 + torch.rand(t, generator=torch.Generator().manual_seed(1)).cuda()
    u = g / 4 if entropy else None
    dh, _ = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u, weight_grad=False, sync=True)
    g = g.double()
    G = -g[:, None] * others
    G[here, at] = g * rest
    a = (h.double().abs() @ w.double().abs().t()).amax(1)
    lg = 64 * 2.0 ** -23 * a
    one = 2.0 ** -23 * lse64.abs() + 2.0 ** -21      # of l - lse
    err = g[:, None] * others * (1.01 * 2.0 ** -8 + 2 * (lg + one))[:, None]
    err[here, at] = g * (one + 2 * lg * rest)
    if entropy:
        # p (log p + H): each of the two is off by `one` and the logits' errors on the others' part; the forward pass's H
        # sums v exponentials (2^-20 of what is beside the target, whose logarithms reach 32) and s = 1 + ... (2^-21)
        u = u.double()
        z = u[:, None] * p * (lp + ent64[:, None])
        G -= z
        off = (2 * one + 2.0 ** -21 + 2 * lg * (ent64 + rest) + 2.0 ** -15 * ent64)[:, None] + 2 * (lg + one)[:, None] * (lp.abs() + ent64[:, None])
        err += u[:, None] * p * off + 1.01 * 2.0 ** -8 * z.abs()
        err[here, at] -= 1.01 * 2.0 ** -8 * z.abs()[here, at]
        own = u * p[here, at] * (2 * one + 2.0 ** -21 + (2 * lg + 2.0 ** -15) * (ent64 + rest))
        err[here, at] = g * (one + 2 * lg * rest) + own
    W = w.double()
    want = G @ W
    slack = err @ W.abs() + (v / 16 + 96) * 2.0 ** -23 * (G.abs() @ W.abs()) + 1.01 * 2.0 ** -8 * want.abs() + 1e-37
    assert torch.all((dh.double() - want).abs() <= slack)
    # along the target's own row of the weight: the entry itself, within what l - lse leaves of it
    along = (dh.double() * W[at]).sum(1), (want * W[at]).sum(1)
    size = 2.0 ** -8 * (want.abs() * W[at].abs()).sum(1) / d ** 0.5 * 8      # d independent roundings, 8 deviations
    slack = (err.unsqueeze(1) @ (W @ W[at].t()).abs().t().unsqueeze(2))[:, 0, 0] + size + 2.0 ** -17 * (G.abs().unsqueeze(1) @ (W @ W[at].t()).abs().t().unsqueeze(2))[:, 0, 0]
    assert torch.all((along[0] - along[1]).abs() <= slack)
