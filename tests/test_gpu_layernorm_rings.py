"""The layer norm's gradient with rings of every length, each of which wraps several times; its permitted aliases; rows that
hold a NaN or an infinity; sums of squares beyond fp32.  Bounds as in test_gpu_layernorm.py."""
import pytest
import torch

import test_gpu_layernorm as base

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

F32, BF16, E4M3 = 0, 1, 2
# rows, d, bytes an element: rings of 2, 3 and 4 rows, by CTAs of up to 256 threads and more; of 2 and 1 for longer rows
RINGS = [(4000, 4096, 4), (3000, 8192, 4), (4000, 3080, 4), (3000, 5120, 4), (3000, 6144, 4), (5000, 2560, 4), (6000, 4096, 2),
         (5000, 2560, 2), (4000, 8192, 2), (3000, 4608, 4), (2000, 12000, 2), (2000, 12000, 4)]


@pytest.mark.parametrize("rows,d,es", RINGS)
@pytest.mark.parametrize("dsum", [False, True])
def test_rings(rows, d, es, dsum):
    dtype = torch.float32 if es == 4 else torch.bfloat16
    h, dy, w = base._data(rows, d, dtype), base._data(rows, d, dtype, 2), base._data(1, d, dtype, 3)[0]
    s = base._data(rows, d, dtype, 4) if dsum else None
    base._check_back(dy, h, w, 1e-5, s, P.bakron_layernorm_backward(dy, h, w, 1e-5, dsum=s))


def _norm(x, res, w, b, sum_, y, scales):
    q = y.dtype == torch.float8_e4m3fn
    kind = F32 if x.dtype == torch.float32 else BF16
    rows, d = x.shape
    rc = P.lib().bakron_layernorm(x.data_ptr(), kind, rows, d, d, res.data_ptr(), d, w.data_ptr(), F32, b.data_ptr(), F32, 1e-5,
                                  sum_.data_ptr(), d, y.data_ptr(), E4M3 if q else kind, d, scales.data_ptr() if q else None,
                                  torch.cuda.current_stream().cuda_stream)
    assert rc == 0


@pytest.mark.parametrize("rows,d", [(3, 40), (5, 1001), (400, 2056), (400, 4104), (400, 4101), (320, 8208), (2, 20000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("q", [False, True])
def test_the_sum_in_place_of_an_input(rows, d, dtype, q):
    x, r = base._data(rows, d, dtype), base._data(rows, d, dtype, 5)
    w, b = base._data(1, d, torch.float32, 3)[0], base._data(1, d, torch.float32, 6)[0]
    kind = torch.float8_e4m3fn if q else dtype
    y, s, h = P.bakron_layernorm(x, w, b, 1e-5, residual=r, out_dtype=kind)
    for into in (0, 1):
        a = [x.clone(), r.clone()]
        got, scales = torch.empty_like(y), torch.empty(rows, device="cuda")
        _norm(a[0], a[1], w, b, a[into], got, scales)
        assert torch.equal(a[into], h) and torch.equal(a[1 - into], (x, r)[1 - into])
        assert torch.equal(got.view(torch.uint8), y.view(torch.uint8)) and (not q or torch.equal(scales, s))


@pytest.mark.parametrize("rows,d", [(3, 40), (37, 1001), (700, 2056), (700, 1001), (700, 9000), (640, 17000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_gradient_in_place_of_dsum(rows, d, dtype):
    h, dy, s = base._data(rows, d, dtype), base._data(rows, d, dtype, 2), base._data(rows, d, dtype, 4)
    w = base._data(1, d, torch.float32, 3)[0]
    dx, dw, db = P.bakron_layernorm_backward(dy, h, w, 1e-5, dsum=s)
    kind = F32 if dtype == torch.float32 else BF16
    L, into, w2, b2 = P.lib(), s.clone(), torch.empty_like(dw), torch.empty_like(db)
    size = L.bakron_layernorm_backward_workspace_bytes(rows, d)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert 0 == L.bakron_layernorm_backward(dy.data_ptr(), d, h.data_ptr(), d, kind, rows, d, w.data_ptr(), F32, 1e-5, into.data_ptr(),
                                            d, into.data_ptr(), d, w2.data_ptr(), b2.data_ptr(), ws.data_ptr(), size,
                                            torch.cuda.current_stream().cuda_stream)
    assert torch.equal(into, dx) and torch.equal(w2, dw) and torch.equal(b2, db)


@pytest.mark.parametrize("rows,d", [(7, 40), (40, 1001), (700, 2056), (700, 1001), (700, 9000), (640, 17000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_are_not_finite(rows, d, dtype):
    """A NaN or an infinity of h: its row of dx, and dw; of dy: its row of dx, dw and db at its column."""
    h, dy, w = base._data(rows, d, dtype), base._data(rows, d, dtype, 2), base._data(1, d, dtype, 3)[0]
    want = P.bakron_layernorm_backward(dy, h, w, 1e-5)
    bad, bad_dy = h.clone(), dy.clone()
    bad[2, 5], bad[4, d - 1] = float("nan"), float("inf")
    dx, dw, db = P.bakron_layernorm_backward(dy, bad, w, 1e-5)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[2] = keep[4] = False
    assert torch.equal(dx[keep], want[0][keep]) and torch.isnan(dx[2]).all() and torch.isnan(dx[4]).all()
    assert torch.isnan(dw).all() and torch.equal(db, want[2])
    bad_dy[3, 7] = float("inf")
    dx, dw, db = P.bakron_layernorm_backward(bad_dy, h, w, 1e-5)
    keep[:] = True
    keep[3] = False
    cols = torch.arange(d, device="cuda") != 7
    assert torch.equal(dx[keep], want[0][keep]) and not torch.isfinite(dx[3]).any()
    assert torch.equal(dw[cols], want[1][cols]) and torch.equal(db[cols], want[2][cols])
    assert not torch.isfinite(dw[7]) and torch.isinf(db[7])


@pytest.mark.parametrize("rows,d", [(3, 40), (700, 2056), (2, 20000)])
def test_squares_beyond_fp32(rows, d):
    """Entries of 1e20: rho is 0, so y is the bias, and dx what reaches h past the norm."""
    x, b = base._data(rows, d, torch.float32) * 1e20, base._data(1, d, torch.float32, 6)[0]
    w = base._data(1, d, torch.float32, 3)[0]
    y, _, _ = P.bakron_layernorm(x, w, b, 1e-5)
    assert torch.equal(y, b.expand(rows, d))
    dy, s = base._data(rows, d, torch.float32, 2), base._data(rows, d, torch.float32, 4)
    dx, dw, _ = P.bakron_layernorm_backward(dy, x, w, 1e-5, dsum=s)
    assert torch.equal(dx, s) and torch.all(dw == 0)
