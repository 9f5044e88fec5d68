"""bakron_token_logprobs and its gradient against their formulas in 64 bits.

Tolerances: exp and log in fp32 have a few 2^-23; the sum of v terms is added in parts
(at most v / 1024 + 64 additions in a row of 2^-24 each).  lse then has (that sum) plus
2^-22 |lse|, and logp the same plus 2^-22 |l|.  The entropy's terms p (l - m) are bounded
by entropy + 1 in sum, with |l - m| roundings in the exponent.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

INF = math.inf
SHAPES = [(1, 1), (2, 2), (3, 31), (1, 32), (5, 33), (4, 255), (2, 1000), (3, 1024), (2, 4099), (1, 32000), (7, 50021),
          (2, 131073), (700, 100), (1300, 2050)]


def _logits(rows, v, dtype, seed=0, scale=3.0):
    g = torch.Generator().manual_seed(rows + 7 * v + seed)
    return (scale * torch.randn(rows, v, generator=g)).to(dtype).cuda()


def _targets(rows, v, seed=0):
    g = torch.Generator().manual_seed(rows * 3 + v + seed)
    t = torch.randint(0, v, (rows,), generator=g)
    if rows > 2:
        t[1], t[2] = -100, v         # not scored
    return t.cuda()


def _ref(x, t):
    x = x.double()
    lse = torch.logsumexp(x, 1)
    z = x - x.amax(1, keepdim=True)     # before the log's addition, which a large maximum would swallow
    lp = z - z.exp().sum(1, keepdim=True).log()
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, 0).sum(1)
    ok = (t >= 0) & (t < x.shape[1])
    logp = torch.where(ok, lp.gather(1, t.clamp(0, x.shape[1] - 1)[:, None])[:, 0], 0)
    return logp, ent, lse, lp


def _order(x, k):
    """Indices of the k largest, the lower index first among equal ones."""
    v, i = torch.sort(x.float() + 0.0, dim=1, descending=True, stable=True)
    return i[:, :k].int()


def _check(x, t, top):
    rows, v = x.shape
    logp, ent, lse, tl, ti = P.bakron_token_logprobs(x, t, top)
    rlogp, rent, rlse, rlp = _ref(x, t)
    s = (v / 1024 + 64) * 2.0 ** -24
    big = x.double().clamp(min=-1e4).abs().amax(1)
    slack = s + 2.0 ** -21 * (rlse.abs() + big)
    assert torch.all((lse.double() - rlse).abs() <= slack)
    ok = torch.isfinite(rlogp)
    assert torch.all((logp.double() - rlogp).abs()[ok] <= slack[ok])
    assert torch.equal(logp[~ok].double(), rlogp[~ok])
    assert torch.all((ent.double() - rent).abs() <= (4 * s + 2.0 ** -20 * (big + 8)) * (rent + 1))
    if top:
        assert torch.equal(ti, _order(x, top))
        want = rlp.gather(1, ti.long())
        fin = torch.isfinite(want)
        assert torch.all((tl.double() - want).abs()[fin] <= slack[:, None].expand_as(want)[fin])
        assert torch.equal(tl[~fin].double(), want[~fin])
    else:
        assert tl is None and ti is None


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 1, 5, 20, 32])
def test_logprobs(rows, v, dtype, top):
    _check(_logits(rows, v, dtype), _targets(rows, v), min(top, v))


@pytest.mark.parametrize("v", [40, 1024, 5000, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["equal", "two", "steps", "rising", "falling", "last", "zeros"])
def test_ties_and_orders(v, dtype, kind):
    """Many equal values, sorted rows, and the best ones where a scan meets them last."""
    i = torch.arange(v)
    x = {"equal": torch.full((v,), 1.5), "two": (i % 2).float(), "steps": (i // 37 % 5).float(),
         "rising": i.float() / 64, "falling": -i.float() / 64, "last": (i >= v - 33).float() * 4,
         "zeros": torch.where(i % 3 == 0, 0.0, -0.0)}[kind]
    x = x.to(dtype).repeat(3, 1).cuda()
    _check(x, _targets(3, v), 32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [50, 3000])
def test_masked_rows(dtype, v):
    """-inf in places, a row of nothing else, one finite value, the type's lowest value."""
    x = _logits(8, v, dtype)
    low = torch.finfo(dtype).min
    x[0, v // 2:] = -INF
    x[1, :] = -INF
    x[2, :] = -INF
    x[2, v - 3] = 2.0
    x[3, 1:] = low
    x[4, :] = low
    x[5, ::2] = -INF
    x[6, : v - 1] = -INF
    t = torch.tensor([1, 0, v - 3, 0, 3, 2, 0, 5], device="cuda")
    k = 10
    logp, ent, lse, tl, ti = P.bakron_token_logprobs(x, t, k)
    rlogp, rent, rlse, rlp = _ref(x, t)
    keep = torch.tensor([0, 2, 3, 4, 5, 6, 7], device="cuda")
    assert torch.equal(ti, _order(x, k))
    assert lse[1] == -INF and ent[1] == 0 and logp[1] == -INF and torch.all(tl[1] == -INF)
    for got, want in ((lse, rlse), (ent, rent), (logp, rlogp)):
        got, want = got[keep].double(), want[keep]
        fin = torch.isfinite(want)
        assert torch.equal(got[~fin], want[~fin])
        assert torch.all((got - want).abs()[fin] <= 1e-5 * (1 + want.abs()[fin]))
    d = P.bakron_token_logprobs_backward(x, t, lse, torch.ones(8, device="cuda"), ent, torch.ones(8, device="cuda"))
    assert torch.all(d[1] == 0) and torch.isfinite(d.float()).all()
    p = rlp.exp()
    want = (torch.arange(v, device="cuda")[None] == t[:, None]).double() - p - \
        torch.where(p > 0, p * (rlp + rent[:, None]), 0)
    assert torch.all((d[keep].double() - want[keep]).abs() <= 1e-5 + 1.01 * 2.0 ** -8 * want[keep].abs())


def test_rows_that_are_no_distribution():
    for dtype in (torch.float32, torch.bfloat16):
        x = _logits(5, 3000, dtype)
        good = P.bakron_token_logprobs(x, _targets(5, 3000), 4)
        x[0, 17], x[1, 2999] = float("nan"), INF
        x[3] = float("nan")
        logp, ent, lse, tl, ti = P.bakron_token_logprobs(x, torch.full((5,), 3, device="cuda"), 4)
        for t in (lse, ent, logp):
            assert torch.isnan(t[[0, 1, 3]]).all() and torch.isfinite(t[[2, 4]]).all()
        assert torch.isnan(tl[[0, 1, 3]]).all() and torch.all(ti[3] == -1) and torch.all(ti[[0, 1, 2, 4]] >= 0)
        for a, b in zip((ent, lse, tl, ti), good[1:]):
            assert torch.equal(a[[2, 4]], b[[2, 4]])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v,shift,extra", [(1000, 1, 0), (1000, 3, 5), (8192, 0, 8), (8191, 8, 1), (33, 5, 2)])
def test_strides(dtype, v, shift, extra):
    xb = _logits(6, v + shift + extra, dtype)
    x, t = xb[:, shift:shift + v], _targets(6, v)
    _check(x, t, 20)
    same = P.bakron_token_logprobs(x.contiguous(), t, 20)
    assert torch.equal(P.bakron_token_logprobs(x, t, 20)[4], same[4])
    lse, ent = same[2], same[1]
    g, u = torch.randn(6, device="cuda"), torch.randn(6, device="cuda")
    ob = torch.full((6, v + 9), 7.0, dtype=dtype, device="cuda")
    P.bakron_token_logprobs_backward(x, t, lse, g, ent, u, out=ob[:, 2:2 + v])
    want = P.bakron_token_logprobs_backward(x.contiguous(), t, lse, g, ent, u)
    assert torch.equal(ob[:, 2:2 + v], want)
    assert torch.all(ob[:, :2] == 7) and torch.all(ob[:, 2 + v:] == 7)
    y = x.clone()
    assert torch.equal(P.bakron_token_logprobs_backward(y, t, lse, g, ent, u, out=y), want)      # in place


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("entropy", [False, True])
def test_backward(rows, v, dtype, entropy):
    x, t = _logits(rows, v, dtype), _targets(rows, v)
    _, ent, lse, _, _ = P.bakron_token_logprobs(x, t)
    gen = torch.Generator().manual_seed(v)
    g = torch.randn(rows, generator=gen).cuda()
    u = torch.randn(rows, generator=gen).cuda() if entropy else None
    d = P.bakron_token_logprobs_backward(x, t, lse, g, ent if entropy else None, u)
    lp = x.double() - lse.double()[:, None]
    p = lp.exp()
    ok = (t >= 0) & (t < v)
    g64 = torch.where(ok, g.double(), 0)[:, None]
    want = g64 * ((torch.arange(v, device="cuda")[None] == t[:, None]).double() - p)
    size = g64.abs() * (p + (torch.arange(v, device="cuda")[None] == t[:, None]))
    if entropy:
        e = p * (lp + ent.double()[:, None])
        want -= u.double()[:, None] * e
        size = size + u.double().abs()[:, None] * p * (lp.abs() + ent.double()[:, None].abs())
    # the exponent's rounding: 2^-23 of |l| + |lse|
    slack = (2.0 ** -20 + 2.0 ** -22 * (x.double().abs() + lse.double().abs()[:, None])) * size
    slack += (1.01 * 2.0 ** -8 if dtype == torch.bfloat16 else 0) * want.abs() + 1e-37
    assert torch.all((d.double() - want).abs() <= slack)


def test_backward_against_differences():
    """Along random directions, against central differences of the 64-bit formula."""
    rows, v = 5, 400
    x, t = _logits(rows, v, torch.float32), _targets(rows, v)
    g, u = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    _, ent, lse, _, _ = P.bakron_token_logprobs(x, t)
    d = P.bakron_token_logprobs_backward(x, t, lse, g, ent, u).double()

    def f(z):
        logp, e, _, _ = _ref(z, t)
        return (g.double() * logp).sum() + (u.double() * e).sum()

    for seed in range(4):
        w = _logits(rows, v, torch.float64, seed + 1, 1.0)
        h = 1e-4
        num = (f(x.double() + h * w) - f(x.double() - h * w)) / (2 * h)
        assert abs(float(num - (d * w).sum())) <= 1e-5 * float((d * w).abs().sum())


def test_shapes_streams_and_repeats():
    x = _logits(12, 5000, torch.bfloat16).reshape(3, 4, 5000)
    t = _targets(12, 5000).reshape(3, 4)
    a = P.bakron_token_logprobs(x, t, 6)
    assert a[0].shape == (3, 4) and a[3].shape == (3, 4, 6) and a[4].dtype == torch.int32
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = P.bakron_token_logprobs(x, t, 6, stream=s)
    s.synchronize()
    assert all(torch.equal(i, j) for i, j in zip(a, b))
    c = P.bakron_token_logprobs(x[:0], t[:0], 6)
    assert c[0].shape == (0, 4) and c[4].shape == (0, 4, 6)
    assert P.bakron_token_logprobs(x)[0] is None


def test_refusals():
    x, t = torch.zeros(3, 10, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for top in (-1, 11, 33):
        with pytest.raises(P.BakronError):
            P.bakron_token_logprobs(x, t, top)
    with pytest.raises(ValueError):
        P.bakron_token_logprobs(x.half(), t)
    with pytest.raises(ValueError):
        P.bakron_token_logprobs(x, t.int())
    with pytest.raises(ValueError):
        P.bakron_token_logprobs(x, t[:2])
    lse = torch.zeros(3, device="cuda")
    with pytest.raises(P.BakronError):
        P.bakron_token_logprobs_backward(x, t, lse, None)
    with pytest.raises(P.BakronError):
        P.bakron_token_logprobs_backward(x, t, lse, None, None, lse)
    with pytest.raises(ValueError):
        P.bakron_token_logprobs_backward(x, t, lse, lse, out=torch.zeros(3, 9, device="cuda"))
