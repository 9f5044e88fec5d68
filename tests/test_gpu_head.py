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


@pytest.mark.parametrize("t,v,d", [(2048, 66000, 64), (16500, 300, 64)])
def test_in_pieces(t, v, d):
    """More than one piece of the vocabulary in the backward pass; more than one of the tokens in the forward one."""
    h, w, at = _data(t, v, d, 3)
    got = P.bakron_head_logprobs(h, w, at, sync=True)
    for i in range(0, t, 2048):
        s = slice(i, i + 2048)
        _check_forward(h[s], w, at[s], [g[s] for g in got])
    g = torch.randn(t, device="cuda")
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, got[2], g)
    if t <= 2048:
        _check_backward(h, w, at, got[2], g, None, None, dh, dw)
    else:
        _check_backward(h[-2048:], w, at[-2048:], got[2][-2048:], g[-2048:], None, None, dh[-2048:], None)


def test_repeated_targets():
    """Many tokens of one target, few of others: their rows of dW are sums over tokens."""
    t, v, d = 700, 300, 136
    h, w, at = _data(t, v, d, 4)
    at[:] = 7
    at[::5] = torch.arange(140, device="cuda") % 11
    at[3::50] = -1
    at[4::50] = v      # neither is scored
    _, _, lse = P.bakron_head_logprobs(h, w, at)
    g = torch.randn(t, device="cuda")
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, g)
    _check_backward(h, w, at, lse, g, None, None, dh, dw)


@pytest.mark.parametrize("t", [3, 300])
@pytest.mark.parametrize("shift,extra", [(0, 8), (1, 3), (8, 5)])
def test_strides(t, shift, extra):
    v, d = 500, 264
    h, w, at = _data(t, v, d, 5)
    hb, wb = torch.zeros(t, shift + d + extra, device="cuda").bfloat16(), torch.zeros(v, shift + d + extra, device="cuda").bfloat16()
    hb[:, shift:shift + d], wb[:, shift:shift + d] = h, w
    hs, ws = hb[:, shift:shift + d], wb[:, shift:shift + d]
    a, b = P.bakron_head_logprobs(h, w, at), P.bakron_head_logprobs(hs, ws, at)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    g = torch.randn(t, device="cuda")
    a = P.bakron_head_logprobs_backward(h, w, at, a[2], g)
    b = P.bakron_head_logprobs_backward(hs, ws, at, b[2], g)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    c = P.bakron_head_logprobs(hs.reshape(1, t, d), ws, at.reshape(1, t))
    assert c[0].shape == (1, t) and torch.equal(c[2][0], P.bakron_head_logprobs(h, w, at)[2])


def test_with_the_logits():
    """What bakron_token_logprobs gives for the fp32 logits: both have fp32 sums of exact products."""
    h, w, at = _data(130, 777, 320, 6)
    logits = (h.double() @ w.double().t()).float()
    a, b = P.bakron_head_logprobs(h, w, at), P.bakron_token_logprobs(logits, at)
    slack = _logit_slack(h, w).amax(1) + 2.0 ** -18
    for x, y, k in zip(a, b[:3], (2, 32, 1)):
        assert torch.all((x.double() - y.double()).abs() <= 2 * k * slack)


def test_special_values():
    """A row with a NaN or an infinity keeps to itself; large logits; one token in the vocabulary; no tokens."""
    t, v, d = 40, 300, 64
    h, w, at = _data(t, v, d, 7)
    h[5] *= 1e4      # logits in the tens of thousands
    want = P.bakron_head_logprobs(h, w, at)
    _check_forward(h, w, at, want)
    bad = h.clone()
    bad[1, 3], bad[2, 9] = float("nan"), float("inf")
    got = P.bakron_head_logprobs(bad, w, at)
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[1] = keep[2] = False
    for x, y in zip(want, got):
        assert torch.equal(x[keep], y[keep])
    assert not torch.isfinite(got[2][1:3]).any()
    g = torch.randn(t, device="cuda")
    a, _ = P.bakron_head_logprobs_backward(h, w, at, want[2], g, weight_grad=False)
    b, _ = P.bakron_head_logprobs_backward(bad, w, at, got[2], g, weight_grad=False)
    assert torch.equal(a[keep], b[keep])
    logp, entropy, lse = P.bakron_head_logprobs(h, w[:1], torch.zeros_like(at))
    assert torch.all(logp == 0) and torch.all(entropy == 0)
    none = P.bakron_head_logprobs(h[:0], w, at[:0])
    assert all(x.shape == (0,) for x in none)
    dh, dw = P.bakron_head_logprobs_backward(h[:0], w, at[:0], none[2], none[0])
    assert dh.shape == (0, d) and torch.all(dw == 0)


def test_no_token_is_scored():
    h, w, at = _data(33, 100, 72, 8)
    at[:] = -100
    logp, _, lse = P.bakron_head_logprobs(h, w, at)
    assert torch.all(logp == 0)
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, torch.randn(33, device="cuda"))
    assert torch.all(dh == 0) and torch.all(dw == 0)


def test_against_differences():
    """Along random directions, central differences of the 64-bit function at bf16 points: truncation
    1e-6 relative; the gradient's roundings (2^-8 of each entry of G and of each result) are independent of
    the direction, so their sum stays below 2^-8 of the norms' product."""
    t, v, d = 20, 150, 48
    h, w, at = _data(t, v, d, 9)
    logp, ent, lse = P.bakron_head_logprobs(h, w, at)
    g, u = torch.randn(t, device="cuda"), torch.randn(t, device="cuda")
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, g, entropy=ent, dentropy=u)
    ok = (at >= 0).double()

    def f(hh, ww):
        x = hh @ ww.t()
        lp = torch.log_softmax(x, 1)
        e = -(lp.exp() * lp).sum(1)
        return (g.double() * ok * lp.gather(1, at.clamp(min=0)[:, None])[:, 0] + u.double() * e).sum()

    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        a = torch.randn(t, d, generator=gen, device="cuda", dtype=torch.float64)
        b = torch.randn(v, d, generator=gen, device="cuda", dtype=torch.float64) / d ** 0.5
        e = 1e-4
        num = (f(h.double() + e * a, w.double() + e * b) - f(h.double() - e * a, w.double() - e * b)) / (2 * e)
        got = (dh.double() * a).sum() + (dw.double() * b).sum()
        size = dh.double().norm() * a.norm() + dw.double().norm() * b.norm()
        assert abs(float(num - got)) <= 2.0 ** -8 * float(size)


def test_streams_and_graphs():
    """On a side stream; captured, with two graphs that share a workspace, one after another."""
    h, w, at = _data(70, 900, 128, 10)
    want = P.bakron_head_logprobs(h, w, at)
    g = torch.randn(70, device="cuda")
    back = P.bakron_head_logprobs_backward(h, w, at, want[2], g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = P.bakron_head_logprobs(h, w, at, stream=s)
    gback = P.bakron_head_logprobs_backward(h, w, at, got[2], g, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + back, got + gback))
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    static = torch.zeros_like(h)
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            f = P.bakron_head_logprobs(static, w, at, workspace=ws)
            b = P.bakron_head_logprobs_backward(static, w, at, f[2], g, workspace=ws)
        graphs.append((gr, f + b))
    for x in (h, 2 * h):
        static.copy_(x)
        for gr, _ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        f = P.bakron_head_logprobs(x, w, at)
        b = P.bakron_head_logprobs_backward(x, w, at, f[2], g)
        for _, out in graphs:
            assert all(torch.equal(p, q) for p, q in zip(f + b, out))


def test_timeout_is_reported(monkeypatch):
    h, w, at = _data(300, 2000, 512, 11)
    want = P.bakron_head_logprobs(h, w, at)
    g = torch.randn(300, device="cuda")
    monkeypatch.setenv("BAKRON_SPIN_CYCLES", "0")
    for call in (lambda: P.bakron_head_logprobs(h, w, at, sync=True),
                 lambda: P.bakron_head_logprobs_backward(h, w, at, want[2], g, sync=True)):
        with pytest.raises(P.BakronError) as e:
            call()
        assert e.value.status == 4
    monkeypatch.delenv("BAKRON_SPIN_CYCLES")
    again = P.bakron_head_logprobs(h, w, at, sync=True)
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_refusals():
    h, w, at = _data(8, 50, 64, 12)
    lse = torch.zeros(8, device="cuda")
    for bad in (lambda: P.bakron_head_logprobs(h.float(), w, at), lambda: P.bakron_head_logprobs(h, w.float(), at),
                lambda: P.bakron_head_logprobs(h, w[:, :63], at), lambda: P.bakron_head_logprobs(h, w, at[:7]),
                lambda: P.bakron_head_logprobs(h, w, at.int()), lambda: P.bakron_head_logprobs(h, w.cpu(), at),
                lambda: P.bakron_head_logprobs(h, w.reshape(2, 25, 64), at),
                lambda: P.bakron_head_logprobs_backward(h, w, at, lse.double(), lse),
                lambda: P.bakron_head_logprobs_backward(h, w, at, lse, lse[:3])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: P.bakron_head_logprobs(h, w[:0], at),      # no vocabulary
                lambda: P.bakron_head_logprobs_backward(h, w, None, lse, lse),      # dlogp without targets
                lambda: P.bakron_head_logprobs_backward(h, w, at, lse, None, dentropy=lse),      # no entropy
                lambda: P.bakron_head_logprobs(h, w, at, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(P.BakronError):
            bad()


def test_offsets_past_32_bits():
    """A weight of 2.46e9 values: what lies behind the 2^31st is read and its gradient written."""
    t, v, d = 5, 300000, 8192
    g = torch.Generator(device="cuda").manual_seed(13)
    h = torch.randn(t, d, generator=g, device="cuda").bfloat16()
    w = torch.randn(v, d, generator=g, device="cuda", dtype=torch.bfloat16) * (2.5 / d ** 0.5)
    at = torch.tensor([v - 1, 7, v - 3, -100, v - 1], device="cuda")
    logp, ent, lse = P.bakron_head_logprobs(h, w, at)
    x = torch.cat([h.double() @ w[i:i + 20000].double().t() for i in range(0, v, 20000)], 1)
    want = torch.logsumexp(x, 1)
    slack = (d / 16 + 16) * 2.0 ** -23 * (h.double().abs() @ w[:1000].double().abs().t()).amax() * 2 + 2.0 ** -19 + 2.0 ** -22 * 20
    assert torch.all((lse.double() - want).abs() <= slack)
    c = torch.randn(t, generator=g, device="cuda")
    dh, dw = P.bakron_head_logprobs_backward(h, w, at, lse, c)
    G = -(torch.where(at >= 0, c.double(), 0.0)[:, None] * (x - lse.double()[:, None]).exp())
    G[torch.arange(t), at.clamp(min=0)] += torch.where(at >= 0, c.double(), 0.0)
    for s in (slice(0, 300), slice(v - 300, v)):
        rows = G[:, s].t() @ h.double()
        # an entry of G: a rounding, the logits' error; one rounding of the result
        cut = G[:, s].abs().t() @ h.double().abs()
        assert torch.all((dw[s].double() - rows).abs() <= (1.01 * 2.0 ** -8 + 2 * slack) * cut + 1.01 * 2.0 ** -8 * rows.abs() + 1e-37)
    back = sum(G[:, i:i + 20000] @ w[i:i + 20000].double() for i in range(0, v, 20000))
    assert torch.linalg.norm(dh.double() - back) <= 2 * 2.0 ** -8 * torch.linalg.norm(back)
