"""bakron_linear's activations over their whole range, one value a row: a 1 x 1 weight of 1
and fp32 results.  The value itself arrives as the bias, in fp32, so that it is not
rounded to the tokens' type.

relu is exact.  silu: the exponential's argument has a rounding of 2^-24 |v| log2(e) and the
quotient a few 2^-23, of |v| at most.  gelu: erf is within 1.5e-7 plus its fp32 roundings
(2^-22), times |v| / 2."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _values():
    v = torch.cat([torch.linspace(-100, 100, 4001), torch.linspace(-6, 6, 4001), torch.tensor([0.0, 1e-30, -1e-30, 1e30, -1e30])])
    return v.float().cuda()


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 40])
def test_activation(act, rows):
    import paper_2608_06291_gb300 as P
    P.build()
    v = _values()
    m = v.numel()
    w = P.bakron_pack_weight(torch.ones(m, 1, dtype=torch.uint8, device="cuda"), torch.ones(m, 1, device="cuda"),
                             torch.zeros(m, 1, device="cuda"), 1)
    y = P.bakron_linear(torch.zeros(rows, 1, dtype=torch.bfloat16, device="cuda"), w, bias=v, activation=act,
                        out_dtype=torch.float32, sync=True).double()
    x = v.double()
    want = {"relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[act](x)
    slack = {"relu": torch.zeros_like(x), "silu": x.abs() * (2.0 ** -21 + x.abs() * torch.sigmoid(x) * 2.0 ** -23),
             "gelu": x.abs() / 2 * (1.6e-7 + 2.0 ** -21)}[act] + 1e-37
    assert torch.all((y - want[None]).abs() <= slack[None])
    assert math.isnan(float(P.bakron_linear(torch.full((1, 1), float("nan"), dtype=torch.bfloat16, device="cuda"), w,
                                            activation=act)[0, 0]))
