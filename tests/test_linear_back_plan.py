"""How the quantised product's gradient shares out shared memory for few tokens: every size's rings fit, hold
what their warps take in turn (a slot always belongs to one team), and every block has one owner."""
import subprocess

from paper_2608_06291_gb300 import buildlib

PLANS = r"""
#include "linear_back.cu"
#include <cstdio>
using namespace bakron;
namespace bakron {
int cuda_fail(cudaError_t, const char*, int) { return 0; }
long long spin_cycles_from_env() { return 0; }
bool get_encode() { return false; }
PFN_cuTensorMapEncodeTiled_v12000 g_encode;
}
extern "C" int bakron_read_status(void*, void*) { return 0; }
int main() {
  int bad = 0;
  for (int rows = 1; rows <= FUSED_TOKENS; ++rows)
    for (int k = 0; k < 4; ++k)
      for (int n : {1, 128, 129, 4096, 11003, 131072})
        for (int m : {1, 127, 4096, 28672, 131072}) {
          const bool w8 = k & 1, one = k & 2;
          const FusedPlan p(rows, m, n, w8, one);
          const size_t want = 1024 + (size_t)p.na * FB_A + (size_t)p.nb * p.bn * 256 +
                              (size_t)p.nc * ((w8 ? 16384 : 8192) + 640 * (one ? 1 : 4));
          bool ok = p.bn % 16 == 0 && p.bn >= 16 && p.bn <= FB_MAX_BN && p.bn * p.token_tiles >= rows &&
                    p.bn * (p.token_tiles - 1) < rows;
          ok = ok && (p.teams == 2 || p.teams == 4) && p.na % p.teams == 0 && p.nc % p.teams == 0 && p.na <= FB_RING &&
               p.nb <= FB_RING && p.nc <= FB_RING && p.nb >= 2 && p.smem == want && p.smem + 1024 <= 227 * 1024;
          ok = ok && p.ctas >= 1 && p.ctas <= ROW_SMS && (int64_t)p.ctas <= (int64_t)p.tiles * p.nk;
          if (rows % 37 == 1) {      // the shares, and whose part of a tile is where
            FusedParams F{};
            F.tiles = p.tiles;
            F.nk = p.nk;
            const Shares s(F, p.ctas);
            ok = ok && s.begin(0) == 0 && s.begin(p.ctas) == (int64_t)p.tiles * p.nk;
            for (int c = 0; c < p.ctas; ++c) {
              ok = ok && s.begin(c) < s.begin(c + 1) && s.owner(s.begin(c)) == c && s.owner(s.begin(c + 1) - 1) == c;
              const int first = (int)(s.begin(c) / p.nk), last = (int)((s.begin(c + 1) - 1) / p.nk);
              ok = ok && s.slot(c, first) == 2 * c && (last == first || s.slot(c, last) == 2 * c + 1);
            }
          }
          if (!ok && bad++ < 20) std::printf("rows %d m %d n %d w8 %d one %d: bn %d teams %d na %d nb %d nc %d smem %zu\n", rows,
                                             m, n, w8, one, p.bn, p.teams, p.na, p.nb, p.nc, p.smem);
        }
  return bad ? 1 : 0;
}
"""


def test_every_size_has_a_plan(tmp_path):
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(PLANS)
    subprocess.run([buildlib.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-O1", "-std=c++17",
                    "--expt-relaxed-constexpr", "-I", buildlib.CSRC, "-I", buildlib.INCLUDE, str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
