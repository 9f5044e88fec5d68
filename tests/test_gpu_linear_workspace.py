"""bakron_linear's workspace: its first word is the status of the call, whatever it held before and
however many tokens there are."""
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


@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 300])
@pytest.mark.parametrize("dtype", [torch.uint8, torch.int32])
def test_the_status_is_this_calls(rows, dtype):
    import paper_2608_06291_gb300 as P
    P.build()
    ws = torch.full((4096,), 4, dtype=dtype, device="cuda")
    assert P.bakron_read_status(ws) != 0
    _call(P, rows, ws)
    assert P.bakron_read_status(ws) == 0
    _call(P, rows, ws.fill_(4), sync=True)


def test_a_few_tokens_touch_no_more_than_the_status():
    import paper_2608_06291_gb300 as P
    P.build()
    for size in (0, 3, 4, 64):
        whole = torch.full((256,), 9, dtype=torch.uint8, device="cuda")
        _call(P, 5, whole[:size])
        assert torch.all(whole[4:] == 9) and torch.all(whole[:4] == (0 if size >= 4 else 9))
