"""The launch of the norm's gradient: every width has CTAs, whose threads cover a row and whose
rings fit an SM; and the widths where a ring just fits, in fp32, against the formula."""
import subprocess

import pytest
import torch

from paper_2608_06291_gb300 import buildlib

PLANS = r"""
#include "norm.cu"
#include <cstdio>
using namespace bakron;
namespace bakron { int cuda_fail(cudaError_t, const char*, int) { return 0; } }
int main() {
  int bad = 0;
  for (int es : {2, 4})
    for (int vec = 0; vec < 2; ++vec)
      for (int d = 1; d <= NORM_MAX_D; ++d) {
        if (vec && d % 8) continue;
        const BackPlan p(d, es, vec);
        const int nt = back_threads(d);
        const long long ring = (long long)p.ring * 3 * d * es;
        bool ok = p.ctas >= 1 && back_parts(1, d, es, vec) == 1 && back_parts(100000, d, es, vec) == ROW_SMS * p.ctas;
        if (nt) ok = ok && nt % 32 == 0 && (long long)nt * BACK_VPT * 8 >= d && p.ctas * nt <= 1024;
        // what a launch may ask for; an SM's 228 KB, with a kilobyte and the slots (256 B) beside each CTA's ring
        ok = ok && (p.ring == 0 || (nt && vec && p.ring >= 2)) && ring <= NB_SMEM && p.ctas * (ring + 1024 + 256) <= 228 * 1024;
        if (!ok && bad++ < 20) std::printf("d %d, %d bytes, vec %d: ring %d, ctas %d\n", d, es, vec, p.ring, p.ctas);
      }
  return bad ? 1 : 0;
}
"""


def test_every_width_has_a_plan(tmp_path):
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(PLANS)
    subprocess.run([buildlib.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-O0", "-std=c++17",
                    "--expt-relaxed-constexpr", "-I", buildlib.CSRC, "-I", buildlib.INCLUDE, str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("d", [9336, 9344, 9352, 9360, 9368, 9376, 9384, 9392, 16384])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [3, 400])
@pytest.mark.parametrize("dsum", [False, True])
def test_wide_rows(d, dtype, rows, dsum):
    """rho has 2^-19 of itself, a mean of d products 2^-19 of its absolute terms, every other
    operation of an fp32 result 2^-24; a bf16 result 1.01 * 2^-8.  dw: 2^-18 a term and one
    rounding of 2^-24 for each of the rows' additions."""
    import paper_2608_06291_gb300 as P
    P.build()
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    h, dy, s = (torch.randn(rows, d, generator=g, device="cuda").to(dtype) for _ in range(3))
    w = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    dx, dw = P.bakron_rmsnorm_backward(dy, h, w, 1e-5, dsum=s if dsum else None)
    h64, y64, w64, s64 = h.double(), dy.double(), w.double(), s.double() if dsum else torch.zeros_like(s).double()
    rho = 1 / torch.sqrt(h64.square().mean(1, keepdim=True) + 1e-5)
    back = w64 * y64
    want = rho * (back - h64 * rho.square() * (back * h64).mean(1, keepdim=True)) + s64
    size = rho * (back.abs() + h64.abs() * rho.square() * (back * h64).abs().mean(1, keepdim=True)) + s64.abs()
    slack = 2.0 ** -17 * size + (1.01 * 2.0 ** -8 if dtype == torch.bfloat16 else 0) * want.abs()
    assert torch.all((dx.double() - want).abs() <= slack)
    terms = (y64 * h64 * rho).abs().sum(0)
    assert torch.all((dw.double() - (y64 * h64 * rho).sum(0)).abs() <= (2.0 ** -18 + rows * 2.0 ** -24) * terms)
