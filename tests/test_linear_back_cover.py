"""That the GPU tests' sizes reach what the kernels of the quantised product's gradient do at real ones: several chunks
a warp one after another, rings that wrap three times, sums of more than 4096 products, and each kernel."""
import subprocess

from paper_2608_06291_gb300 import buildlib
import test_gpu_linear_back as small
import test_gpu_linear_back_long as long

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
  int t, m, n, qmax, group;
  while (std::scanf("%d %d %d %d %d", &t, &m, &n, &qmax, &group) == 5) {
    const bool w8 = qmax > 15, one = one_grid(n, group);
    const FewPlan f(m, n, w8, one);
    const FusedPlan p(t, m, n, w8, one);
    const bool fused = fused_is_faster(p, t, m, n, w8);
    std::printf("%d %d %d %d %d\n", t <= FEW_BACK ? 0 : fused ? 1 : 2, f.per / FW_WARPS, (int)((int64_t)p.tiles * p.nk / p.ctas),
                p.tiles > p.ctas, p.teams);
  }
}
"""


def test_sizes(tmp_path):
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(PLANS)
    subprocess.run([buildlib.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-O1", "-std=c++17",
                    "--expt-relaxed-constexpr", "-I", buildlib.CSRC, "-I", buildlib.INCLUDE, str(src), "-o", str(exe)],
                   check=True, capture_output=True)

    def plans(module):
        cases = [(t,) + w for t in module.TOKENS for w in module.WEIGHTS]
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
        return [c + tuple(map(int, line.split())) for c, line in zip(cases, out.splitlines())]

    few, fused, written = range(3)
    rows = plans(long)
    assert len(rows) == len(long.TOKENS) * len(long.WEIGHTS)
    for wide in (False, True):      # 4 and 8 bits
        mine = [r for r in rows if (r[3] > 15) == wide]
        assert any(r[5] == few and r[0] <= 4 and r[6] >= 8 for r in mine) and any(r[5] == few and r[0] > 4 and r[6] >= 8 for r in mine)
        assert any(r[5] == fused and r[7] >= 24 for r in mine) and any(r[5] == fused and r[7] > 32 for r in mine)
        assert any(r[5] == fused and r[8] for r in mine) and any(r[5] == written for r in mine)
    # a grid for each of a block's four chunks, and one for all
    assert any(r[4] == 32 and r[5] == fused and r[7] >= 24 for r in rows) and any(r[4] == 64 and r[5] == few and r[6] >= 8 for r in rows)
    assert {r[9] for r in rows if r[5] == fused} == {2, 4}
    assert {r[5] for r in plans(small)} == {few, fused, written}
