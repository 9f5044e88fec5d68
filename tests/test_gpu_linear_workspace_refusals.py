"""What cannot be bakron_linear's workspace is refused before any launch; its size counts in bytes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _call(P, rows, workspace, sync=False):
    m, n = 300, 256
    g = torch.Generator().manual_seed(rows)
    codes = torch.randint(0, 16, (m, n), generator=g, dtype=torch.uint8).cuda()
    w = P.bakron_pack_weight(codes, torch.full((m, 1), 0.125, device="cuda"), torch.full((m, 1), 7.0, device="cuda"), 15)
    x = torch.randint(-2, 3, (rows, n), generator=g).bfloat16().cuda()
    y = P.bakron_linear(x, w, out_dtype=torch.float32, workspace=workspace, sync=sync)
    assert torch.equal(y.double(), x.double() @ (0.125 * (codes.double() - 7.0)).T)


def test_refusals():
    import paper_2608_06291_gb300 as P
    P.build()
    for ws in (torch.empty(4096, dtype=torch.uint8), torch.empty(8192, dtype=torch.uint8, device="cuda")[::2]):
        for rows in (4, 40):
            with pytest.raises(ValueError):
                _call(P, rows, ws)
    with pytest.raises(P.BakronError) as e:
        _call(P, 40, torch.empty(128, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 5
    _call(P, 40, torch.empty(64, dtype=torch.int32, device="cuda"), sync=True)      # 256 bytes
