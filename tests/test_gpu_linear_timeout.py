"""bakron_linear when a bounded wait runs out: an error, and the context stays usable."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [40, 300])
@pytest.mark.parametrize("qmax,xtype", [(15, torch.bfloat16), (15, torch.float8_e4m3fn), (200, torch.bfloat16)])
def test_timeout_is_reported(rows, qmax, xtype, monkeypatch):
    import paper_2608_06291_gb300 as P
    P.build()
    g = torch.Generator().manual_seed(rows)
    m, n = 700, 2048
    codes = torch.randint(0, qmax + 1, (m, n), generator=g, dtype=torch.uint8).cuda()
    w = P.bakron_pack_weight(codes, torch.full((m, 1), 0.125, device="cuda"), torch.full((m, 1), 7.0, device="cuda"), qmax)
    x = torch.randint(-2, 3, (rows, n), generator=g).cuda()
    monkeypatch.setenv("BAKRON_SPIN_CYCLES", "0")
    with pytest.raises(P.BakronError) as e:
        P.bakron_linear(x.to(xtype), w, out_dtype=torch.float32, sync=True)
    assert e.value.status == 4
    monkeypatch.delenv("BAKRON_SPIN_CYCLES")
    y = P.bakron_linear(x.to(xtype), w, out_dtype=torch.float32, sync=True)
    assert torch.equal(y.double(), x.double() @ (0.125 * (codes.double() - 7.0)).T)
