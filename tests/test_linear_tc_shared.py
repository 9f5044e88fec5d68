"""k_linear_tc's shared memory: for every shape of its tile, what the kernel lays out (rings,
barriers, TMEM's address, the abort flag) fits what a launch asks for, wherever in its 1024
bytes of alignment the block's memory begins."""
import re
import subprocess

from paper_2608_06291_gb300 import buildlib

SIZES = r"""
#include "linear_tc.cu"
#include <cstdio>
using namespace bakron;
namespace bakron {
bool get_encode() { return false; }
PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
long long spin_cycles_from_env() { return 0; }
int cuda_fail(cudaError_t, const char*, int) { return 0; }
}
template <class S> int one() {
  const int bars = COUNT;
  const long long end = 1023 + 2ll * S::NX * S::BOX + (long long)S::NW * S::WS + S::STAGE_BYTES + (long long)S::NG * S::GS +
                        8 * bars + 8;
  const bool ok = end <= S::SMEM;
  if (!ok) std::printf("%d tokens, W8 %d, X8 %d: %lld bytes past the end\n", S::BN, S::W8, S::X8, end - S::SMEM);
  return ok ? 0 : 1;
}
template <bool W8, bool X8> int all() {
  return one<TcShape<32, W8, X8>>() + one<TcShape<64, W8, X8>>() + one<TcShape<128, W8, X8>>() + one<TcShape<192, W8, X8>>();
}
int main() { return all<false, false>() + all<false, true>() + all<true, false>(); }
"""


def _count():
    """The barriers as the kernel lays them out, one array after another."""
    with open(buildlib.CSRC + "/linear_tc.cu") as f:
        chain = re.search(r"uint64_t \*xF = bars,(.*?);", f.read(), re.S).group(1)
    sizes = re.findall(r"\w+ = \w+ \+ (S::\w+)", chain)
    assert len(sizes) == chain.count("=") == 9
    return " + ".join(sizes) + " + 1"


def test_the_layout_fits(tmp_path):
    src, exe = tmp_path / "sizes.cu", tmp_path / "sizes"
    src.write_text(SIZES.replace("COUNT", _count()))
    # PTX is enough: no kernel runs
    subprocess.run([buildlib.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-O0", "-std=c++17",
                    "--expt-relaxed-constexpr", "-I", buildlib.CSRC, "-I", buildlib.INCLUDE, str(src), "-o", str(exe)],
                   check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
