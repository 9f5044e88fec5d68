"""The launch of the layer norm's gradient: every width and number of rows has CTAs, whose threads cover a
row and whose rings fit an SM beside one another, and parts that the workspace holds."""
import subprocess

from paper_2608_06291_gb300 import buildlib

PLANS = r"""
#include "layernorm.cu"
#include <cstdio>
using namespace bakron;
namespace bakron { int cuda_fail(cudaError_t, const char*, int) { return 0; } }
int main() {
  int bad = 0;
  for (int rows : {1, 37, LB_FEW, LB_FEW + 1, 4096, 100000})
    for (int es : {2, 4})
      for (int vec = 0; vec < 2; ++vec)
        for (int d = 1; d <= NORM_MAX_D; ++d) {
          if (vec && d % 8) continue;
          const LayerPlan p(rows, d, es, vec);
          const long long ring = (long long)p.ring * 3 * d * es;
          bool ok = p.ctas >= 1 && p.nt >= 32 && p.nt <= 1024 && p.nt % 32 == 0 && p.few == (rows <= LB_FEW);
          if (p.vpt) {
            // threads cover a row; registers: 128 or 64 a thread; what a launch may ask for, and
            // an SM's 228 KB, with a kilobyte and the slots (512 B) beside each CTA's ring
            ok = ok && !p.few && (long long)p.nt * p.vpt * 8 >= d && p.ctas * p.nt <= (p.paired ? 512 : 1024);
            ok = ok && (p.ring == 1 || (vec && p.vpt == 2)) && p.ring <= (p.paired ? 4 : 2) && (!p.paired || p.ring >= 2) && ring <= LB_SMEM && p.ctas * (ring + 1024 + 512) <= 228 * 1024;
            ok = ok && p.parts(rows) >= 1 && p.parts(rows) <= rows;
          }
          const size_t need = align256((size_t)rows * 8) + (size_t)p.parts(rows) * d * 8;
          ok = ok && need <= bakron_layernorm_backward_workspace_bytes(rows, d);
          if (!ok && bad++ < 20) std::printf("rows %d d %d, %d bytes, vec %d: vpt %d nt %d ring %d, ctas %d\n", rows, d, es, vec,
                                             p.vpt, p.nt, p.ring, p.ctas);
        }
  return bad ? 1 : 0;
}
"""


def test_every_width_has_a_plan(tmp_path):
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(PLANS)
    subprocess.run([buildlib.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-O1", "-std=c++17",
                    "--expt-relaxed-constexpr", "-I", buildlib.CSRC, "-I", buildlib.INCLUDE, str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
