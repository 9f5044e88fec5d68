"""bakron_linear_backward against dx = dy What in 64 bits.

An operand s (c - z) has one rounding to bf16 (2^-8, with the fp32 product's 2^-24 below 1.01
times that), so a sum errs by 1.01 * 2^-8 of its absolute terms; its fp32 additions lose at most
a unit in the last place each, one per 16 terms (and per part): (m / 16 + 128) 2^-23 of them; the
result has one rounding.  Where scales are powers of two and everything is a small integer,
operands and sums are exact and the result is the exact one, rounded.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

TOKENS = [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 128, 129, 200, 256, 257, 384, 385, 520]
WEIGHTS = [(1, 1, 15, 0), (5, 3, 1, 0), (64, 128, 15, 128), (130, 127, 3, 0), (300, 256, 255, 0), (257, 384, 15, 32),
           (700, 512, 7, 64), (513, 576, 255, 96), (1000, 1100, 200, 0), (2100, 129, 15, 0), (96, 2048, 15, 512)]


def _weight(m, n, qmax, group, seed, pow2):
    g = torch.Generator().manual_seed(seed + m + 3 * n)
    G = n // group if group else 1
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, dtype=torch.uint8)
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g).float()
    scales = torch.rand(m, G, generator=g) + 0.5
    if pow2:
        scales = torch.exp2(torch.randint(-2, 2, (m, G), generator=g).float())
    codes, zeros, scales = codes.cuda(), zeros.cuda(), scales.cuda()
    W = (codes.double().view(m, G, -1) - zeros.double()[:, :, None]) * scales.double()[:, :, None]
    return P.bakron_pack_weight(codes, scales, zeros, qmax, group), W.view(m, n)


def _check(dy, W, dx):
    want = dy.double() @ W
    terms = dy.double().abs() @ W.abs()
    slack = (1.01 * 2.0 ** -8 + (W.shape[0] / 16 + 128) * 2.0 ** -23) * terms + 1.01 * 2.0 ** -8 * want.abs()
    assert torch.all((dx.double() - want).abs() <= slack + 1e-37)


@pytest.mark.parametrize("m,n,qmax,group", WEIGHTS)
@pytest.mark.parametrize("t", TOKENS)
def test_backward(t, m, n, qmax, group):
    w, W = _weight(m, n, qmax, group, t, False)
    dy = torch.randn(t, m, generator=torch.Generator().manual_seed(t)).bfloat16().cuda()
    dx = P.bakron_linear_backward(dy, w, sync=True)
    _check(dy, W, dx)
    # few absolute terms' worth: the sum's error is no bias
    want = dy.double() @ W
    assert torch.linalg.norm(dx.double() - want) <= 4e-3 * torch.linalg.norm(want)
    assert torch.equal(P.bakron_linear_backward(dy, w), dx)


@pytest.mark.parametrize("m,n,qmax,group", WEIGHTS)
@pytest.mark.parametrize("t", TOKENS)
def test_exact(t, m, n, qmax, group):
    w, W = _weight(m, n, qmax, group, t + 1, True)
    dy = torch.randint(-2, 3, (t, m), generator=torch.Generator().manual_seed(t)).bfloat16().cuda()
    want = dy.double() @ W       # quarters, below 2^20: exact in fp32 and in any order
    assert torch.equal(P.bakron_linear_backward(dy, w), want.float().bfloat16())


@pytest.mark.parametrize("t", [3, 40, 300])
@pytest.mark.parametrize("shift,extra", [(0, 8), (1, 3), (8, 5)])
def test_strides(t, shift, extra):
    m, n = 264, 392
    w, W = _weight(m, n, 15, 0, 1, False)
    dy = torch.randn(t, shift + m + extra, device="cuda").bfloat16()[:, shift:shift + m]
    around = torch.full((t + 2, shift + n + extra), 7.0, device="cuda").bfloat16()
    out = around[1:t + 1, shift:shift + n]
    assert P.bakron_linear_backward(dy, w, out=out) is out
    assert torch.equal(out, P.bakron_linear_backward(dy.contiguous(), w))
    _check(dy, W, out)
    mask = torch.ones_like(around, dtype=torch.bool)
    mask[1:t + 1, shift:shift + n] = False
    assert torch.all(around[mask] == 7)
    dx = P.bakron_linear_backward(dy.reshape(1, t, m), w)
    assert dx.shape == (1, t, n) and torch.equal(dx[0], out)


def test_not_finite_and_none():
    """A NaN or an infinity of a token's gradient stays in its row; no tokens."""
    w, W = _weight(300, 200, 15, 0, 2, False)
    for t in (4, 40):
        dy = torch.randn(t, 300, device="cuda").bfloat16()
        dx = P.bakron_linear_backward(dy, w)
        bad = dy.clone()
        bad[1, 3], bad[2, 299] = float("nan"), float("inf")
        got = P.bakron_linear_backward(bad, w)
        assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()
        keep = [i for i in range(t) if i not in (1, 2)]
        assert torch.equal(got[keep], dx[keep])
    assert P.bakron_linear_backward(dy[:0], w).shape == (0, 200)


def test_against_the_product():
    """<dy, x What^T> = <dy What, x>: the product and its gradient use one weight."""
    m, n, t = 640, 896, 50
    w, W = _weight(m, n, 15, 128, 3, False)
    x, dy = torch.randn(t, n, device="cuda").bfloat16(), torch.randn(t, m, device="cuda").bfloat16()
    y, dx = P.bakron_linear(x, w, out_dtype=torch.float32), P.bakron_linear_backward(dy, w)
    a, b = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
    # the first has fp32 errors; the second bf16 roundings of W and dx, each sum in independent terms
    slack = 1.01 * 2.0 ** -8 * ((dx.double() * x.double()).abs().sum() + ((dy.double().abs() @ W.abs()) * x.double().abs()).sum())
    assert abs(float(a - b)) <= float(slack)


def test_streams_and_graphs():
    """On a side stream, and captured: replays take new gradients."""
    w, W = _weight(500, 700, 15, 0, 4, False)
    for t in (1, 12, 40, 300):
        dy = torch.randn(t, 500, device="cuda").bfloat16()
        want = P.bakron_linear_backward(dy, w)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = P.bakron_linear_backward(dy, w, stream=s)
        s.synchronize()
        assert torch.equal(got, want)
        static = torch.zeros_like(dy)
        with torch.cuda.stream(s):
            P.bakron_linear_backward(static, w)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = P.bakron_linear_backward(static, w)
        for k in range(2):
            static.copy_(dy if k else 2 * dy)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want if k else P.bakron_linear_backward(2 * dy, w))


@pytest.mark.parametrize("t", [40, 300, 600])
def test_timeout_is_reported(t, monkeypatch):
    w, W = _weight(700, 512, 15, 0, 5, False)
    dy = torch.randn(t, 700, device="cuda").bfloat16()
    monkeypatch.setenv("BAKRON_SPIN_CYCLES", "0")
    with pytest.raises(P.BakronError) as e:
        P.bakron_linear_backward(dy, w, sync=True)
    assert e.value.status == 4
    monkeypatch.delenv("BAKRON_SPIN_CYCLES")
    _check(dy, W, P.bakron_linear_backward(dy, w, sync=True))


def test_refusals():
    w, _ = _weight(64, 32, 15, 0, 6, False)
    dy = torch.zeros(20, 64, device="cuda", dtype=torch.bfloat16)
    for bad in (lambda: P.bakron_linear_backward(dy.float(), w), lambda: P.bakron_linear_backward(dy[:, :63], w),
                lambda: P.bakron_linear_backward(dy.cpu(), w),
                lambda: P.bakron_linear_backward(dy, w, out=torch.zeros(20, 33, device="cuda", dtype=torch.bfloat16)),
                lambda: P.bakron_linear_backward(dy, w, out=torch.zeros(20, 32, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(P.BakronError):
        P.bakron_linear_backward(dy, w, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))
