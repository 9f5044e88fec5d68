"""bakron_head_logprobs and bakron_head_logprobs_backward against their formulas in 64 bits.

Forward: the products are exact and their sums fp32; a sum of d terms errs by at most its
additions, one per 16 terms in the tensor cores (each may lose a whole unit in the last
place, 2^-23, of the running sum, which is at most the sum of absolute terms a), and the
terms of a step are cut to 2^-23 of the largest: (d / 16 + 16) 2^-23 a per logit.  lse takes the
largest logit error and a few roundings of itself, logp twice that; the sum of v exponentials
(2^-22 each) has at most 128 / 4 + 1100 additions, which 2^-19 of slack holds: as an absolute error
of lse, and 32 times that (the spread of the logits) of the entropy.

Backward: an entry of G has its own error of the logits and one rounding to bf16 (2^-8 of the
entry at most with the exponential's 2^-20), except the target's; results have fp32 sums
(at most v / 16 + splits + 64 additions of up to 2^-23 of the absolute terms) and one rounding.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

SHAPES = [(1, 1, 1), (1, 32000, 512), (3, 7, 5), (2, 255, 64), (5, 257, 72), (37, 1000, 136), (128, 513, 64),
          (129, 512, 200), (255, 300, 1000), (256, 2048, 128), (300, 700, 1028), (77, 5021, 1000), (513, 129, 33)]


def _data(t, v, d, seed=0, spread=2.5):
    g = torch.Generator(device="cuda").manual_seed(t + 7 * v + 31 * d + seed)
    h = torch.randn(t, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(v, d, generator=g, device="cuda") * (spread / d ** 0.5)).bfloat16()
    at = torch.randint(0, v, (t,), generator=g, device="cuda")
    at[torch.rand(t, generator=g, device="cuda") < 0.2] = -100
    return h, w, at


def _logit_slack(h, w):
    d = h.shape[1]
    return (d / 16 + 16) * 2.0 ** -23 * (h.double().abs() @ w.double().abs().t())


def _check_forward(h, w, at, got):
    logp, entropy, lse = got
    x = h.double() @ w.double().t()
    want = torch.logsumexp(x, 1)
    p = torch.softmax(x, 1)
    ent = -torch.special.xlogy(p, p).sum(1)
    slack = _logit_slack(h, w).amax(1) + 2.0 ** -19 + 2.0 ** -22 * want.abs()
    assert torch.all((lse.double() - want).abs() <= slack)
    assert torch.all((entropy.double() - ent).abs() <= 32 * slack)
    if at is not None:
        v = w.shape[0]
        ok = (at >= 0) & (at < v)
        exp = x.gather(1, at.clamp(0, v - 1)[:, None])[:, 0] - want
        assert torch.all((logp.double() - exp).abs()[ok] <= 2 * slack[ok])
        assert torch.all(logp[~ok] == 0)


@pytest.mark.parametrize("t,v,d", SHAPES)
def test_forward(t, v, d):
    h, w, at = _data(t, v, d)
    _check_forward(h, w, at, P.bakron_head_logprobs(h, w, at, sync=True))
    none, entropy, lse = P.bakron_head_logprobs(h, w)
    assert none is None
    _check_forward(h, w, None, (None, entropy, lse))


def _back(h, w, at, lse, g, ent, u):
    x = h.double() @ w.double().t()
    lp = x - lse.double()[:, None]
    p = lp.exp()
    v = w.shape[0]
    ok = (at >= 0) & (at < v) if at is not None else torch.zeros(h.shape[0], dtype=torch.bool, device=h.device)
    gg = torch.where(ok, g.double(), 0.0) if g is not None else torch.zeros(h.shape[0], dtype=torch.float64, device=h.device)
    G = -gg[:, None] * p
    if u is not None:
        G -= u.double()[:, None] * p * (lp + ent.double()[:, None])
    size = G.abs()
    if at is not None and g is not None:
        own = torch.zeros_like(G).scatter_(1, at.clamp(0, v - 1)[:, None], gg[:, None])
        G, size = G + own, size + own.abs()
    return G, size


def _check_backward(h, w, at, lse, g, ent, u, dh, dw):
    t, v, d = h.shape[0], w.shape[0], h.shape[1]
    G, size = _back(h, w, at, lse, g, ent, u)
    # entries but the target's: a rounding (half a step, 2^-9 at most 2^-8 of the entry), the logits' error
    cut = G.abs().clone()
    if at is not None and g is not None:
        ok = (at >= 0) & (at < v)
        cut[torch.arange(t, device=h.device)[ok], at[ok]] = 0
    lg = _logit_slack(h, w) + 2.0 ** -19
    factor = 1 + 2 * ((u.abs() / (g.abs() + u.abs()).clamp(min=1e-30)).double()[:, None] if u is not None and g is not None else 1)
    err = cut * 2.0 ** -8 + size * lg * factor * 2 + (size * 32 * 2.0 ** -19)
    if u is not None:      # the two terms of p (lp + H) may cancel
        x = (h.double() @ w.double().t()) - lse.double()[:, None]
        p = x.exp()
        err = err + u.double().abs()[:, None] * p * (x.abs() + ent.double().abs()[:, None] + 1) * (2.0 ** -18 + 2 * lg)
    for got, a, b, e, n in ((dh, G, w.double(), err, v), (dw, G.t(), h.double(), err.t(), t)):
        if got is None:
            continue
        want = a @ b
        slack = e @ b.abs() + (n / 16 + 96) * 2.0 ** -23 * (a.abs() @ b.abs()) + 1.01 * 2.0 ** -8 * want.abs() + 1e-37
        assert torch.all((got.double() - want).abs() <= slack)


@pytest.mark.parametrize("t,v,d", SHAPES)
@pytest.mark.parametrize("kind", ["logp", "entropy", "both"])
def test_backward(t, v, d, kind):
    h, w, at = _data(t, v, d, 1)
    _, ent, lse = P.bakron_head_logprobs(h, w)
    g = torch.randn(t, device="cuda") if kind != "entropy" else None
    u = torch.randn(t, device="cuda") if kind != "logp" else None
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u, sync=True)
    _check_backward(h, w, at, lse, g, ent, u, dh, dw)
    again, none = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u, weight_grad=False)
    assert none is None and torch.equal(again, dh)
    again, dw2 = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u)
    assert torch.equal(again, dh) and torch.equal(dw2, dw)
