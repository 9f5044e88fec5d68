"""The norm's gradient forms 1 / sqrt(mean(h^2) + eps) as the norm does: a square root and a quotient,
each rounded once.

One row with h = 2^k and dy = 2^-k: the mean is 4^k exactly and dw is rho itself, which is
then the fp32 quotient of 1 and the fp32 root of fp32(4^k + eps), to the last bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [7, 64, 1000, 4096, 17000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rho_has_two_roundings(d, dtype):
    import paper_2608_06291_gb300 as P
    P.build()
    w = torch.ones(d, device="cuda")
    eps = np.random.default_rng(d).uniform(0, 3, 100).astype(np.float32)
    for k in (0, 1):
        h = torch.full((1, d), 2.0 ** k, device="cuda").to(dtype)
        dy = torch.full((1, d), 2.0 ** -k, device="cuda").to(dtype)
        got = torch.stack([P.bakron_rmsnorm_backward(dy, h, w, float(e))[1] for e in eps]).cpu().numpy()
        want = np.float32(1) / np.sqrt(np.float32(4.0 ** k) + eps)
        assert want.dtype == np.float32
        assert np.array_equal(got, np.repeat(want[:, None], d, 1))
