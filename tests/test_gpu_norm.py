"""bakron_rmsnorm and bakron_rmsnorm_backward against their formulas in 64 bits.

With fp32 arithmetic a sum of d squares errs by at most (8 + log2 of the threads) rounded
additions of 2^-24 each relative to itself (d <= 16384: 24 bits of slack below), so rho
has 2^-19 and y a few more roundings: 2^-18 |y|.  A result in bf16 adds 1.01 * 2^-8.  In 8 bits
the scale has 2^-18, and a value may land on either neighbour where y / scale lies within
2^-17 of the middle of two: it is compared to the two ends of that interval.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

E4M3 = torch.float8_e4m3fn
SHAPES = [(1, 1), (3, 7), (1, 64), (5, 128), (2, 257), (33, 1000), (4, 1024), (7, 2048), (3, 4097), (2, 8192), (1, 8200),
          (3, 16384), (2, 16385), (1, 65536), (300, 96)]


def _data(rows, d, dtype, seed=0):
    g = torch.Generator().manual_seed(rows + 31 * d + seed)
    x = torch.randn(rows, d, generator=g) * (0.1 + 4 * torch.rand(1, d, generator=g))
    return x.to(dtype).cuda()


def _eps(dtype):
    return 1.01 * 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -18


def _ref(x, res, w, eps):
    h = x.double() if res is None else x.double() + res.double()
    return h, h / torch.sqrt(h.square().mean(1, keepdim=True) + eps) * w.double()


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
    w = w if rows % 2 else w.to(torch.bfloat16)
    y, scales, h = P.bakron_rmsnorm(x, w, 1e-5, residual=r)
    h64, y64 = _ref(x, r, w, 1e-5)
    assert scales is None and (h is None) == (not res)
    if res:
        assert torch.equal(h, (x.float() + r.float()).to(dtype))
    assert torch.all((y.double() - y64).abs() <= _eps(dtype) * y64.abs() + 1e-30)


@pytest.mark.parametrize("rows,d", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("res", [False, True])
def test_norm_in_8_bits(rows, d, dtype, res):
    x, w = _data(rows, d, dtype), _data(1, d, dtype, 3)[0]
    r = _data(rows, d, dtype, 5) if res else None
    y, scales, h = P.bakron_rmsnorm(x, w, 1e-5, residual=r, out_dtype=E4M3)
    _, y64 = _ref(x, r, w, 1e-5)
    s64 = y64.abs().amax(1) / 448
    assert torch.all((scales.double() - s64).abs() <= 2.0 ** -18 * s64)
    q = y64 / s64[:, None]
    a, b = _round_e4m3(q * (1 - 2.0 ** -17)), _round_e4m3(q * (1 + 2.0 ** -17))
    got = y.to(torch.float32).double()
    assert torch.all((got >= torch.minimum(a, b)) & (got <= torch.maximum(a, b)))
    if res:
        assert torch.equal(h, (x.float() + r.float()).to(dtype))


@pytest.mark.parametrize("d", [40, 520, 4096, 20000])
@pytest.mark.parametrize("shift,extra", [(0, 8), (1, 3), (4, 0), (8, 24)])
def test_strides(d, shift, extra):
    xb = _data(5, d + shift + extra, torch.bfloat16)
    x, w = xb[:, shift:shift + d], _data(1, d + shift, torch.float32, 1)[0, shift:]
    for out in (None, E4M3):
        y, s, _ = P.bakron_rmsnorm(x, w, 1e-5, out_dtype=out)
        z, t, _ = P.bakron_rmsnorm(x.contiguous(), w.clone(), 1e-5, out_dtype=out)
        _, y64 = _ref(x, None, w, 1e-5)
        if out is None:
            for v in (y, z):
                assert torch.all((v.double() - y64).abs() <= _eps(torch.bfloat16) * y64.abs())
        else:
            assert torch.all((s - t).abs() <= 2.0 ** -17 * t)
    y3, _, _ = P.bakron_rmsnorm(x.reshape(1, 5, d), w, 1e-5)
    assert y3.shape == (1, 5, d)


def test_special_rows():
    """Zeros, a NaN, an infinity, tiny and large values; no rows."""
    d = 300
    for dtype in (torch.float32, torch.bfloat16):
        x = _data(6, d, dtype)
        x[0] = 0
        x[1, 5] = float("nan")
        x[2, 7] = float("inf")
        x[3] *= 1e-30
        x[4] *= 1e15
        w = torch.ones(d, device="cuda")
        y, _, _ = P.bakron_rmsnorm(x, w, 1e-5)
        q, s, _ = P.bakron_rmsnorm(x, w, 1e-5, out_dtype=E4M3)
        _, y64 = _ref(x, None, w, 1e-5)
        for v in (y, q.to(torch.float32) * s[:, None]):
            assert torch.all(v[0] == 0) and torch.isnan(v[1]).any() and torch.isnan(v[2]).any()
            assert torch.isfinite(v[[0, 3, 4, 5]].float()).all()
        assert s[0] == 1 and torch.isnan(s[1]) and torch.isnan(s[2])
        for i in (3, 4, 5):
            assert torch.all((y[i].double() - y64[i]).abs() <= _eps(dtype) * y64[i].abs() + 1e-37)
    y, s, h = P.bakron_rmsnorm(x[:0], w, 1e-5, residual=x[:0], out_dtype=E4M3)
    assert y.shape == (0, d) and s.shape == (0,) and h.shape == (0, d)


def test_scale_below_the_reciprocals_range():
    """A row whose scale's reciprocal overflows: quotients, still right."""
    x = torch.zeros(1, 64, device="cuda")
    x[0, :3] = torch.tensor([1e-18, -5e-19, 2e-19], device="cuda")
    w = torch.full((64,), 1e-20, device="cuda")
    q, s, _ = P.bakron_rmsnorm(x, w, 1.0, out_dtype=E4M3)      # y about 1e-38: s about 2e-41
    got = q.to(torch.float32)[0, :3].double()
    assert 0 < float(s[0]) < 1.2e-38
    assert torch.all((got - torch.tensor([448.0, -224.0, 89.6], device="cuda", dtype=torch.float64)).abs() <= 6.0)


def _back_ref(dy, h, w, eps, dsum):
    dy, h, w = dy.double(), h.double(), w.double()
    rho = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    dx = rho * (w * dy - h * rho.square() * (w * dy * h).mean(1, keepdim=True))
    return dx + (dsum.double() if dsum is not None else 0), (dy * h * rho).sum(0)


@pytest.mark.parametrize("rows,d", SHAPES + [(1000, 256), (2000, 33), (700, 4096), (650, 17000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dsum", [False, True])
def test_backward(rows, d, dtype, dsum):
    """dx: rho has 2^-19, the mean of w dy h 2^-19 of the sum of its absolute terms, and each
    term of dx a few roundings.  dw: a sum over the rows, each term with 2^-18, added in
    fp32 in parts (rows / 608 + 64 additions at most)."""
    h, dy, w = _data(rows, d, dtype), _data(rows, d, dtype, 2), _data(1, d, dtype, 3)[0]
    s = _data(rows, d, dtype, 4) if dsum else None
    dx, dw = P.bakron_rmsnorm_backward(dy, h, w, 1e-5, dsum=s)
    dx64, dw64 = _back_ref(dy, h, w, 1e-5, s)
    rho = 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + 1e-5)
    back = (w.double() * dy.double()).abs()
    slack = 2.0 ** -17 * rho * (back + h.double().abs() * rho.square() * (back * h.double().abs()).mean(1, keepdim=True))
    slack += _eps(dtype) * dx64.abs() + (2.0 ** -22 * s.double().abs() if dsum else 0)
    assert torch.all((dx.double() - dx64).abs() <= slack + 1e-30)
    terms = (dy.double() * h.double() * rho).abs().sum(0)
    assert torch.all((dw.double() - dw64).abs() <= (2.0 ** -18 + (rows / 608 + 64) * 2.0 ** -24) * terms + 1e-30)
    again = P.bakron_rmsnorm_backward(dy, h, w, 1e-5, dsum=s)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


def test_backward_against_differences():
    """The kernel's gradient along random directions against central differences of the
    64-bit formula: truncation 1e-8 relative, fp32 gradients 2^-17 of their terms."""
    rows, d, eps = 6, 200, 1e-5
    h, w, c = _data(rows, d, torch.float32), _data(1, d, torch.float32, 1)[0], _data(rows, d, torch.float32, 2)
    dx, dw = P.bakron_rmsnorm_backward(c, h, w, eps)

    def f(hh, ww):
        return (c.double() * hh / torch.sqrt(hh.square().mean(1, keepdim=True) + eps) * ww).sum()

    for seed in range(4):
        v, u = _data(rows, d, torch.float64, 10 + seed), _data(1, d, torch.float64, 20 + seed)[0]
        t = 1e-4
        num = (f(h.double() + t * v, w.double() + t * u) - f(h.double() - t * v, w.double() - t * u)) / (2 * t)
        got = (dx.double() * v).sum() + (dw.double() * u).sum()
        size = (dx.double() * v).abs().sum() + (dw.double() * u).abs().sum()
        assert abs(float(num - got)) <= 1e-5 * float(size)


def test_backward_strides_and_aliases():
    for d in (72, 1000, 17000):
        hb, db = _data(9, d + 5, torch.bfloat16), _data(9, d + 16, torch.bfloat16, 1)
        h, dy, w = hb[:, 3:3 + d], db[:, 8:8 + d], _data(1, d, torch.bfloat16, 2)[0]
        dx, dw = P.bakron_rmsnorm_backward(dy, h, w, 1e-5)
        dx2, dw2 = P.bakron_rmsnorm_backward(dy.contiguous(), h.contiguous(), w, 1e-5)
        dx64, dw64 = _back_ref(dy, h, w, 1e-5, None)
        for a, b in ((dx, dw), (dx2, dw2)):
            assert torch.linalg.norm(a.double() - dx64) <= 3e-3 * torch.linalg.norm(dx64)
            assert torch.linalg.norm(b.double() - dw64) <= 1e-5 * torch.linalg.norm(dw64)
    empty = P.bakron_rmsnorm_backward(dy[:0], h[:0], w, 1e-5)
    assert empty[0].shape == (0, d) and torch.all(empty[1] == 0)


def test_refusals():
    x, w = torch.zeros(4, 32, device="cuda"), torch.ones(32, device="cuda")
    with pytest.raises(ValueError):
        P.bakron_rmsnorm(x.half(), w)
    with pytest.raises(ValueError):
        P.bakron_rmsnorm(x, w[:31])
    with pytest.raises(ValueError):
        P.bakron_rmsnorm(x, w, residual=x.bfloat16())
    with pytest.raises(ValueError):
        P.bakron_rmsnorm(x, w, out_dtype=torch.bfloat16)
    with pytest.raises(P.BakronError):
        P.bakron_rmsnorm(x, w, eps=-1.0)
    with pytest.raises(P.BakronError):
        P.bakron_rmsnorm(torch.zeros(1, 65537, device="cuda"), torch.ones(65537, device="cuda"))
    with pytest.raises(ValueError):
        P.bakron_rmsnorm_backward(x[:3], x, w)
