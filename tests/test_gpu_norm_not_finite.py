"""bakron_rmsnorm on rows that hold a NaN or an infinity, entry by entry, as the formula has it: NaN
everywhere; or NaN at the infinity and x / sqrt(inf) = 0 elsewhere.  In 8 bits the scale is NaN,
and so is every entry.  The rows beside them are not touched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [3, 64, 1000, 4096, 8192, 20000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [4, 700])
@pytest.mark.parametrize("where", ["x", "residual"])
def test_not_finite(d, dtype, rows, where):
    import paper_2608_06291_gb300 as P
    P.build()
    g = torch.Generator(device="cuda").manual_seed(d + rows)
    x, r = (torch.randn(rows, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    w = torch.ones(d, device="cuda")
    good, good8, scales = P.bakron_rmsnorm(x, w, residual=r)[0], *P.bakron_rmsnorm(x, w, residual=r, out_dtype=torch.float8_e4m3fn)[:2]
    bad = x if where == "x" else r
    bad[0, d // 2], bad[1, d - 1], bad[2, 0] = float("nan"), float("inf"), -float("inf")
    y, _, h = P.bakron_rmsnorm(x, w, residual=r)
    assert torch.isnan(y[0]).all()
    for row, at in ((1, d - 1), (2, 0)):
        rest = torch.arange(d, device="cuda") != at
        assert torch.isnan(y[row, at]) and torch.all(y[row, rest] == 0) and torch.isinf(h[row, at])
    assert torch.equal(y[3:], good[3:])
    q, s, _ = P.bakron_rmsnorm(x, w, residual=r, out_dtype=torch.float8_e4m3fn)
    assert torch.isnan(s[:3]).all() and torch.isnan(q[:3].float()).all()
    assert torch.equal(s[3:], scales[3:]) and torch.equal(q[3:].float(), good8[3:].float())
