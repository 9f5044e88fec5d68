"""That the GPU tests' sizes launch every ring of the layer norm's gradient, and that each wraps at least twice."""
import subprocess

from paper_2608_06291_gb300 import buildlib
import test_gpu_layernorm_rings as rings

PLANS = r"""
#include "layernorm.cu"
#include <cstdio>
using namespace bakron;
namespace bakron { int cuda_fail(cudaError_t, const char*, int) { return 0; } }
int main() {
  int rows, d, es;
  while (std::scanf("%d %d %d", &rows, &d, &es) == 3) {
    const LayerPlan p(rows, d, es, true);
    std::printf("%d %d %d %d %d\n", p.paired, p.ring, p.nt <= 256, p.vpt, p.parts(rows));
  }
}
"""


def test_every_ring_is_launched_and_wraps(tmp_path):
    src, exe = tmp_path / "plans.cu", tmp_path / "plans"
    src.write_text(PLANS)
    subprocess.run([buildlib.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-O1", "-std=c++17",
                    "--expt-relaxed-constexpr", "-I", buildlib.CSRC, "-I", buildlib.INCLUDE, str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    text = "\n".join(" ".join(map(str, r)) for r in rings.RINGS)
    out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
    seen = set()
    for (rows, _, _), line in zip(rings.RINGS, out.splitlines()):
        paired, ring, few_threads, vpt, parts = map(int, line.split())
        assert vpt and rows // parts >= 2 * ring
        seen.add((bool(paired), ring, bool(few_threads) if paired else None))
    assert seen >= {(True, r, f) for r in (2, 3, 4) for f in (True, False)} | {(False, 1, None), (False, 2, None)}
