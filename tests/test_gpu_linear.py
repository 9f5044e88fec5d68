"""bakron_pack_weight and bakron_linear against y = act(x What^T + b) + r in 64 bits.

Exact cases: with small integers as tokens, power-of-two scales and fp32 results every
sum is an integer below 2^24 (times the scale), so the result has no rounding at all.

Others: c - z and the tokens are exact operands.  A tensor core adds 16 (or 32) products
to a running sum and cuts at about 2^-23 of the largest term; n / 16 such steps, 17
terms in the last, and the fp32 sums over groups and parts stay within
(n / 16 + 64) 2^-22 A, A = sum |s (c - z) x|.  The activations' slopes are below 1.13;
the epilogue's fp32 operations add 2^-20 of their terms, and a bf16 result 1.01 * 2^-8 |y|.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

E4M3 = torch.float8_e4m3fn


def _weight(m, n, qmax, group, seed, pow2=False):
    g = torch.Generator().manual_seed(seed)
    G = n // group if group else 1
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, dtype=torch.uint8)
    scales = torch.exp2(-torch.randint(3, 7, (m, G), generator=g).float()) if pow2 else \
        (0.5 + torch.rand(m, G, generator=g)) * 0.1 / qmax
    zeros = torch.randint(0, qmax + 1, (m, G), generator=g).float()
    return codes.cuda(), scales.cuda(), zeros.cuda()


def _dense(codes, scales, zeros):
    k = codes.shape[1] // scales.shape[1]
    return scales.double().repeat_interleave(k, 1) * (codes.double() - zeros.double().repeat_interleave(k, 1))


def _act(v, name):
    return {None: lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu,
            "gelu": torch.nn.functional.gelu}[name](v)


def _check(y, x64, W, bias=None, act=None, res=None):
    n = W.shape[1]
    pre = x64 @ W.T
    slack = 1.2 * (n / 16 + 64) * 2.0 ** -22 * (x64.abs() @ W.abs().T)
    if bias is not None:
        pre = pre + bias.double()
    want = _act(pre, act)
    slack += 2.0 ** -20 * (pre.abs() + want.abs()) + 1e-30
    if bias is not None:
        slack += 2.0 ** -20 * bias.double().abs()
    if res is not None:
        slack += 2.0 ** -20 * res.double().abs()
        want = want + res.double()
    if y.dtype == torch.bfloat16:
        slack = slack + 1.01 * 2.0 ** -8 * want.abs()
    err = (y.double() - want).abs()
    assert torch.all(err <= slack), float((err / slack).max())


SHAPES = [(1, 1, 1), (1, 128, 128), (2, 33, 31), (5, 100, 129), (8, 257, 384), (9, 130, 1000), (16, 64, 257),
          (17, 128, 640), (31, 300, 513), (33, 129, 128), (64, 512, 1024), (100, 77, 2048), (129, 384, 640),
          (256, 256, 256), (300, 1000, 1500), (513, 130, 384)]


@pytest.mark.parametrize("rows,m,n", SHAPES)
@pytest.mark.parametrize("qmax", [6, 15, 200])
@pytest.mark.parametrize("xtype", ["bf16", "e4m3"])
def test_exact_sums(rows, m, n, qmax, xtype):
    """Integer tokens and power-of-two scales: equal to the last bit."""
    codes, scales, zeros = _weight(m, n, qmax, 0, rows + m + n, pow2=True)
    lim = 8 if qmax < 16 else 2       # sums below 2^24
    x = torch.randint(-lim, lim + 1, (rows, n), generator=torch.Generator().manual_seed(n)).cuda()
    assert n * lim * qmax < 2 ** 24
    w = P.bakron_pack_weight(codes, scales, zeros, qmax)
    y = P.bakron_linear(x.to(torch.bfloat16 if xtype == "bf16" else E4M3), w, out_dtype=torch.float32, sync=True)
    assert torch.equal(y.double(), x.double() @ _dense(codes, scales, zeros).T)


@pytest.mark.parametrize("rows", [1, 7, 16, 40, 150, 300])
@pytest.mark.parametrize("m,n,group", [(96, 96, 32), (200, 96, 96), (130, 640, 64), (256, 1024, 128), (300, 1536, 384),
                                       (128, 2304, 1152), (640, 512, 512)])
@pytest.mark.parametrize("qmax,xtype", [(3, "bf16"), (15, "e4m3"), (31, "bf16"), (255, "e4m3")])
def test_exact_sums_in_groups(rows, m, n, group, qmax, xtype):
    codes, scales, zeros = _weight(m, n, qmax, group, rows + m + n, pow2=True)
    lim = 4 if qmax < 16 else 1
    x = torch.randint(-lim, lim + 1, (rows, n), generator=torch.Generator().manual_seed(n)).cuda()
    w = P.bakron_pack_weight(codes, scales, zeros, qmax, group)
    y = P.bakron_linear(x.to(torch.bfloat16 if xtype == "bf16" else E4M3), w, out_dtype=torch.float32, sync=True)
    # scales 2^-3 .. 2^-6: sums in units of 2^-6 are integers below 2^24
    assert n * lim * qmax * 8 < 2 ** 24
    assert torch.equal(y.double(), x.double() @ _dense(codes, scales, zeros).T)


@pytest.mark.parametrize("rows,m,n,group", [(1, 1024, 4096, 128), (4, 515, 4096, 0), (13, 1000, 2000, 0),
                                            (24, 700, 11008, 128), (200, 1024, 4096, 128), (300, 640, 5000, 0),
                                            (1030, 515, 1056, 32), (700, 2304, 1000, 0)])
@pytest.mark.parametrize("qmax,xtype", [(15, "bf16"), (15, "e4m3"), (255, "bf16"), (255, "e4m3")])
@pytest.mark.parametrize("act,bias,res,out", [(None, False, True, "bf16"), ("silu", True, False, "bf16"),
                                              ("gelu", True, True, "f32"), ("relu", False, False, "f32")])
def test_matches_the_formula(rows, m, n, group, qmax, xtype, act, bias, res, out):
    codes, scales, zeros = _weight(m, n, qmax, group, rows + m)
    g = torch.Generator().manual_seed(7 * rows + n)
    dt = torch.bfloat16 if out == "bf16" else torch.float32
    x = torch.randn(rows, n, generator=g).cuda()
    b = torch.randn(m, generator=g).cuda() if bias else None
    r = torch.randn(rows, m, generator=g).to(dt).cuda() if res else None
    xs = None
    if xtype == "e4m3":
        xs = x.abs().amax(1) / 448
        x = (x / xs[:, None]).to(E4M3)
    else:
        x = x.bfloat16()
    w = P.bakron_pack_weight(codes, scales, zeros, qmax, group)
    y = P.bakron_linear(x, w, x_scales=xs, bias=b, activation=act, residual=r, out_dtype=dt, sync=True)
    x64 = x.to(torch.float32).double()
    _check(y, x64 if xs is None else x64 * xs.double()[:, None], _dense(codes, scales, zeros), b, act, r)


@pytest.mark.parametrize("rows", [3, 40, 200])
@pytest.mark.parametrize("xtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("shift,extra", [(0, 0), (0, 24), (1, 7), (8, 3), (3, 128)])
def test_strides_and_alignment(rows, xtype, shift, extra):
    """Rows that start anywhere; views into wider buffers, whose other entries stay."""
    m, n = 200, 320
    codes, scales, zeros = _weight(m, n, 15, 64, 5)
    w = P.bakron_pack_weight(codes, scales, zeros, 15, 64)
    g = torch.Generator().manual_seed(rows)
    xb = torch.randn(rows, n + shift + extra, generator=g).to(torch.bfloat16 if xtype == "bf16" else E4M3).cuda()
    x = xb[:, shift:shift + n]
    rb = torch.randn(rows, m + shift + extra, generator=g).bfloat16().cuda()
    r = rb[:, shift:shift + m]
    yb = torch.full((rows, m + shift + extra), 5.0, dtype=torch.bfloat16, device="cuda")
    y = P.bakron_linear(x, w, residual=r, out=yb[:, shift:shift + m], sync=True)
    _check(y, x.to(torch.float32).double(), _dense(codes, scales, zeros), None, None, r)
    assert torch.all(yb[:, :shift] == 5.0) and torch.all(yb[:, shift + m:] == 5.0)
    P.bakron_linear(x, w, residual=r, out=r, sync=True)            # into the residual itself
    assert torch.equal(r, y)


@pytest.mark.parametrize("rows", [2, 16, 20, 64, 200])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_row_keeps_to_itself(rows, bad):
    m, n = 140, 300
    codes, scales, zeros = _weight(m, n, 15, 0, 9)
    w = P.bakron_pack_weight(codes, scales, zeros, 15)
    x = torch.randn(rows, n, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    good = P.bakron_linear(x, w, sync=True)
    x[1, n - 1] = bad
    y = P.bakron_linear(x, w, sync=True)
    keep = torch.arange(rows, device="cuda") != 1
    assert torch.equal(y[keep], good[keep])
    hit = (codes[:, n - 1].float() != zeros[:, 0])
    assert not torch.isfinite(y[1][hit]).any()


def test_leading_dimensions_streams_and_repeats():
    m, n = 260, 512
    codes, scales, zeros = _weight(m, n, 15, 128, 2)
    x = torch.randn(3, 50, n, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    w = P.bakron_pack_weight(codes, scales, zeros, 15, 128)
    y = P.bakron_linear(x, w)
    assert y.shape == (3, 50, m)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        z = P.bakron_linear(x, w, stream=s)
        s.synchronize()
        assert torch.equal(y, z)                                   # the same bits every time
    t = P.bakron_linear(x.transpose(0, 1), w, sync=True)           # rows that are not evenly spaced
    assert torch.equal(t, y.transpose(0, 1))
    assert P.bakron_linear(x[:0], w).shape == (0, 50, m)


def test_the_solves_own_codes():
    """Codes, scales and zeros straight from a solve, and their values by dequantize()."""
    import workloads as WL
    W, A, B = WL.small_problem(160, 256, 4, device="cuda")
    f = P.bakron_prepare(A, B, 0.01)
    x = torch.randn(70, 256, generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    for bits, group in ((4, 0), (3, 64), (8, 32)):
        codes, s, z = P.bakron_solve(W, f, bits, group)
        w = P.bakron_pack_weight(codes, s, z, 2 ** bits - 1, group)
        y = P.bakron_linear(x, w, out_dtype=torch.float32, sync=True)
        _check(y, x.double(), P.dequantize(codes, s, z).double())


def test_refusals():
    codes, scales, zeros = _weight(64, 96, 15, 32, 1)
    x = torch.zeros(4, 96, dtype=torch.bfloat16, device="cuda")
    for bad in (zeros + 0.5, zeros - 16, zeros + 16, zeros * float("nan")):
        with pytest.raises(P.BakronError) as e:
            P.bakron_pack_weight(codes, scales, bad, 15, 32)
        assert e.value.status == 1
    with pytest.raises(P.BakronError):
        P.bakron_pack_weight(codes, scales, zeros.clamp(max=7), 7, 32)    # codes above qmax
    with pytest.raises(ValueError):
        P.bakron_pack_weight(codes, scales[:, :2], zeros, 15, 32)
    with pytest.raises((P.BakronError, ValueError)):
        P.bakron_pack_weight(codes, torch.ones(64, 4, device="cuda"), torch.ones(64, 4, device="cuda"), 15, 24)
    w = P.bakron_pack_weight(codes, scales, zeros, 15, 32)
    with pytest.raises(ValueError):
        P.bakron_linear(x[:, :95], w)
    with pytest.raises(ValueError):
        P.bakron_linear(x.float(), w)
    with pytest.raises(ValueError):
        P.bakron_linear(x, w, activation="tanh")
    with pytest.raises(ValueError):
        P.bakron_linear(x, w, bias=torch.zeros(63, device="cuda"))
    with pytest.raises(ValueError):
        P.bakron_linear(x, w, residual=torch.zeros(4, 64, device="cuda"))     # not the result's type
    with pytest.raises(ValueError):
        P.bakron_linear(x.cpu(), w)
