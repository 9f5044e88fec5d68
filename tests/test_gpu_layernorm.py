"""bakron_layernorm and bakron_layernorm_backward against their formulas in 64 bits.

A mean of d values errs by at most 75 rounded additions (64 in a thread, 10 joining them, the
quotient) of 2^-24 each, 2^-17 of the mean of their absolute values a.  So c = h - mu has E =
2^-17 a + 2^-23 |h|; the variance has 2^-17 of itself and twice mean(|c| E), which is below
2^-16 (a^2 + var), and rho half of its relative error.  y has a few more roundings: w rho (E +
2^-16 |c| (1 + a^2 / var)) and 2^-22 of its terms.  A result in bf16 adds 1.01 * 2^-8; in 8 bits a
value may land on either neighbour where y / scale lies within that of the middle of two.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

E4M3 = torch.float8_e4m3fn
SHAPES = [(1, 1), (3, 7), (1, 64), (5, 128), (2, 257), (33, 1000), (4, 1024), (7, 2048), (3, 4097), (2, 8192), (1, 8200),
          (3, 16384), (2, 16385), (1, 65536), (300, 96), (400, 2056), (400, 4100), (320, 8208), (310, 16384)]


def _data(rows, d, dtype, seed=0, offset=1.0):
    g = torch.Generator().manual_seed(rows + 31 * d + seed)
    x = (torch.randn(rows, d, generator=g) + offset * torch.randn(rows, 1, generator=g)) * (0.1 + 4 * torch.rand(1, d, generator=g))
    return x.to(dtype).cuda()


def _eps(dtype):
    return 1.01 * 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22


def _stats(h, eps):
    mu = h.mean(1, keepdim=True)
    c = h - mu
    var = c.square().mean(1, keepdim=True)
    a = h.abs().mean(1, keepdim=True)
    E = 2.0 ** -17 * a + 2.0 ** -23 * h.abs()
    spread = 1 + a.square() / (var + eps)      # how much the mean's error weighs beside the deviation
    return c, 1 / torch.sqrt(var + eps), E, spread


def _ref(x, res, w, b, eps):
    h = x.double() if res is None else x.double() + res.double()
    c, rho, E, spread = _stats(h, eps)
    y = c * rho * w.double()
    slack = w.double().abs() * rho * (E + 2.0 ** -16 * c.abs() * spread) + 2.0 ** -22 * y.abs()
    if b is not None:
        slack = slack + 2.0 ** -22 * b.double().abs()
        y = y + b.double()
    return y, slack


def _round_e4m3(v):
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(v / step) * step).clamp(-448, 448)


@pytest.mark.parametrize("rows,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("res", [False, True])
def test_norm(rows, d, dtype, res):
    x, w = _data(rows, d, dtype), _data(1, d, torch.float32, 3)[0]
    r = _data(rows, d, dtype, 5) if res else None
    b = _data(1, d, torch.float32 if d % 2 else torch.bfloat16, 6)[0] if rows != 3 else None
    w = w if rows % 2 else w.to(torch.bfloat16)
    y, scales, h = P.bakron_layernorm(x, w, b, 1e-5, residual=r)
    y64, slack = _ref(x, r, w, b, 1e-5)
    assert scales is None and (h is None) == (not res)
    if res:
        assert torch.equal(h, (x.float() + r.float()).to(dtype))
    assert torch.all((y.double() - y64).abs() <= _eps(dtype) * y64.abs() + 1.01 * slack + 1e-30)


@pytest.mark.parametrize("rows,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("res", [False, True])
def test_norm_in_8_bits(rows, d, dtype, res):
    x, w = _data(rows, d, dtype), _data(1, d, dtype, 3)[0]
    r, b = (_data(rows, d, dtype, 5) if res else None), _data(1, d, dtype, 6)[0]
    y, scales, h = P.bakron_layernorm(x, w, b, 1e-5, residual=r, out_dtype=E4M3)
    y64, slack = _ref(x, r, w, b, 1e-5)
    s64, off = y64.abs().amax(1), slack.amax(1)
    assert torch.all((scales.double() * 448 - s64).abs() <= off + 2.0 ** -22 * s64)
    s = s64[:, None] / 448
    q = y64 / s
    e = slack / s + q.abs() * (off / s64 + 2.0 ** -21)[:, None]
    a, b = _round_e4m3(q - e), _round_e4m3(q + e)
    got = y.to(torch.float32).double()
    assert torch.all((got >= torch.minimum(a, b)) & (got <= torch.maximum(a, b)))
    if res:
        assert torch.equal(h, (x.float() + r.float()).to(dtype))


@pytest.mark.parametrize("d", [40, 520, 4096, 20000])
@pytest.mark.parametrize("shift,extra", [(0, 8), (1, 3), (4, 0), (8, 24)])
def test_strides(d, shift, extra):
    xb = _data(5, d + shift + extra, torch.bfloat16)
    x, w = xb[:, shift:shift + d], _data(1, d + shift, torch.float32, 1)[0, shift:]
    b = _data(1, d + shift, torch.bfloat16, 2)[0, shift:]
    y, _, _ = P.bakron_layernorm(x, w, b, 1e-5)
    z, _, _ = P.bakron_layernorm(x.contiguous(), w.clone(), b.clone(), 1e-5)
    y64, slack = _ref(x, None, w, b, 1e-5)
    for v in (y, z):
        assert torch.all((v.double() - y64).abs() <= _eps(torch.bfloat16) * y64.abs() + 1.01 * slack)
    y3, _, _ = P.bakron_layernorm(x.reshape(1, 5, d), w, b, 1e-5)
    assert torch.equal(y3[0], y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_far_from_zero(dtype):
    """A mean 1000 times the deviation: the squares are of what the mean leaves."""
    x = _data(9, 3000, dtype, 1, offset=0) + 4000
    w = torch.ones(3000, device="cuda")
    y, _, _ = P.bakron_layernorm(x, w, None, 1e-5)
    c, rho, E, _ = _stats(x.double(), 1e-5)
    # E shifts c; the variance changes by its square, and by 2^-16 of itself
    slack = rho * (E + 2.0 ** -16 * c.abs() + c.abs() * (rho * E.amax(1, keepdim=True)) ** 2)
    assert torch.all((y.double() - c * rho).abs() <= _eps(dtype) * (c * rho).abs() + 1.01 * slack)


@pytest.mark.parametrize("d", [300, 8200, 20000])
def test_special_rows(d):
    """Constant rows, a NaN, an infinity, tiny and large values; no rows."""
    for dtype in (torch.float32, torch.bfloat16):
        x, b = _data(6, d, dtype), _data(1, d, dtype, 2)[0]
        x[0] = 3
        x[1, 5] = float("nan")
        x[2, 7] = float("inf")
        x[3] *= 1e-30
        x[4] *= 1e15
        w = torch.ones(d, device="cuda")
        y, _, _ = P.bakron_layernorm(x, w, b, 1e-5)
        q, s, _ = P.bakron_layernorm(x, w, b, 1e-5, out_dtype=E4M3)
        assert torch.equal(y[0], b)      # what is left of a constant row (3 d is exact) is its bias
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
        assert torch.isnan(s[1]) and torch.isnan(s[2]) and torch.isnan(q[1:3].float()).all()
        assert torch.isfinite(y[[0, 3, 4, 5]].float()).all() and torch.isfinite(s[[0, 3, 4, 5]]).all()
        z, s, _ = P.bakron_layernorm(x[:1], w, None, 1e-5, out_dtype=E4M3)
        assert torch.all(z.float() == 0) and s[0] == 1
    y, s, h = P.bakron_layernorm(x[:0], w, b, 1e-5, residual=x[:0], out_dtype=E4M3)
    assert y.shape == (0, d) and s.shape == (0,) and h.shape == (0, d)


def _check_back(dy, h, w, eps, dsum, got):
    dx, dw, db = got
    rows, dtype = h.shape[0], h.dtype
    dy, h, w = dy.double(), h.double(), w.double()
    c, rho, E, spread = _stats(h, eps)
    g = w * dy
    mgc = (g * c).mean(1, keepdim=True)
    dx64 = rho * (g - g.mean(1, keepdim=True) - c * rho.square() * mgc)
    slack = rho * spread * (2.0 ** -15 * (g.abs() + g.abs().mean(1, keepdim=True))
                            + rho.square() * ((2.0 ** -14 * c.abs() + E) * (g * c).abs().mean(1, keepdim=True)
                                              + c.abs() * (g.abs() * E).mean(1, keepdim=True)))
    if dsum is not None:
        dx64 = dx64 + dsum.double()
        slack = slack + 2.0 ** -22 * dsum.double().abs()
    assert torch.all((dx.double() - dx64).abs() <= _eps(dtype) * dx64.abs() + 1.01 * slack + 1e-30)
    adds = (rows / 152 + 64) * 2.0 ** -24
    terms = (dy * c * rho).abs()
    slack = ((2.0 ** -15 * spread + adds) * terms + dy.abs() * rho * E).sum(0)
    assert torch.all((dw.double() - (dy * c * rho).sum(0)).abs() <= slack + 1e-30)
    assert torch.all((db.double() - dy.sum(0)).abs() <= adds * dy.abs().sum(0) + 1e-30)


@pytest.mark.parametrize("rows,d", SHAPES + [(1000, 256), (2000, 33), (700, 4096), (650, 17000), (200, 9344), (200, 11003),
                                            (609, 520), (620, 1001), (640, 8200), (640, 11003), (620, 16384), (608, 8192), (609, 8192)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dsum", [False, True])
def test_backward(rows, d, dtype, dsum):
    h, dy = _data(rows, d, dtype), _data(rows, d, dtype, 2)
    w = _data(1, d, dtype if rows % 3 else torch.float32, 3)[0]
    s = _data(rows, d, dtype, 4) if dsum else None
    got = P.bakron_layernorm_backward(dy, h, w, 1e-5, dsum=s)
    _check_back(dy, h, w, 1e-5, s, got)
    again = P.bakron_layernorm_backward(dy, h, w, 1e-5, dsum=s)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_backward_against_differences():
    """The kernel's gradient along random directions against central differences of the
    64-bit formula: truncation 1e-8 relative, fp32 gradients 2^-14 of their terms."""
    rows, d, eps = 6, 200, 1e-5
    h, w, dy = _data(rows, d, torch.float32), _data(1, d, torch.float32, 1)[0], _data(rows, d, torch.float32, 2)
    dx, dw, db = P.bakron_layernorm_backward(dy, h, w, eps)

    def f(hh, ww, bb):
        c = hh - hh.mean(1, keepdim=True)
        return (dy.double() * (c / torch.sqrt(c.square().mean(1, keepdim=True) + eps) * ww + bb)).sum()

    for seed in range(4):
        v, u, b = (_data(n, d, torch.float64, k + seed) for n, k in ((rows, 10), (1, 20), (1, 30)))
        t = 1e-4
        num = (f(h.double() + t * v, w.double() + t * u, t * b) - f(h.double() - t * v, w.double() - t * u, -t * b)) / (2 * t)
        parts = [dx.double() * v, dw.double() * u[0], db.double() * b[0]]
        got, size = sum(p.sum() for p in parts), sum(p.abs().sum() for p in parts)
        assert abs(float(num - got)) <= 1e-4 * float(size)


def test_backward_strides():
    for d in (72, 1000, 17000):
        hb, db = _data(9, d + 5, torch.bfloat16), _data(9, d + 16, torch.bfloat16, 1)
        h, dy, w = hb[:, 3:3 + d], db[:, 8:8 + d], _data(1, d, torch.bfloat16, 2)[0]
        _check_back(dy, h, w, 1e-5, None, P.bakron_layernorm_backward(dy, h, w, 1e-5))
        _check_back(dy, h, w, 1e-5, None, P.bakron_layernorm_backward(dy.contiguous(), h.contiguous(), w, 1e-5))
    empty = P.bakron_layernorm_backward(dy[:0], h[:0], w, 1e-5)
    assert empty[0].shape == (0, d) and torch.all(empty[1] == 0) and torch.all(empty[2] == 0)


def test_refusals():
    x, w = torch.zeros(4, 32, device="cuda"), torch.ones(32, device="cuda")
    for bad in (lambda: P.bakron_layernorm(x.half(), w), lambda: P.bakron_layernorm(x, w[:31]),
                lambda: P.bakron_layernorm(x, w, w[:31]), lambda: P.bakron_layernorm(x, w, w.half()),
                lambda: P.bakron_layernorm(x, w, w.cpu()), lambda: P.bakron_layernorm(x, w, residual=x.bfloat16()),
                lambda: P.bakron_layernorm(x, w, out_dtype=torch.bfloat16),
                lambda: P.bakron_layernorm_backward(x[:3], x, w), lambda: P.bakron_layernorm_backward(x, x, w, dsum=x[:3])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(P.BakronError):
        P.bakron_layernorm(x, w, eps=-1.0)
    with pytest.raises(P.BakronError):
        P.bakron_layernorm(torch.zeros(1, 65537, device="cuda"), torch.ones(65537, device="cuda"))
