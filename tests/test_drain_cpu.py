"""What a loader of the tensor-core kernels waits for before its CTA retires, when another role has given up: every stage whose last
load is still in flight, and no other.  The choice of the phase (csrc/tc.cuh, last_fill) runs here against a model of the
barriers: a wait for parity p returns while the current phase has the other parity."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "tc.cuh"
template <int STAGES> int check() {
  int bad = 0;
  for (int fills = 0; fills <= 4 * STAGES; ++fills) {
    int stage = 0, filled[STAGES] = {};
    uint32_t phase = 0;
    for (int i = 0; i < fills; ++i) {
      ++filled[stage];
      if (++stage == STAGES) stage = 0, phase ^= 1u;
    }
    for (int landed = 0; landed < (1 << STAGES); ++landed)          // which of the last fills have landed; those before have
      for (int s = 0; s < STAGES; ++s) {
        const bool here = landed >> s & 1 || filled[s] == 0;
        const int complete = filled[s] - (here ? 0 : 1);            // phases of the stage's barrier that are over
        const bool returns = (uint32_t)(complete & 1) != vtc::last_fill(s, stage, phase);
        bad += returns != here;
      }
  }
  return bad;
}
int main() {
  const int bad = check<1>() + check<2>() + check<3>() + check<4>() + check<5>();
  printf("%d\n", bad);
  return bad != 0;
}
"""


def test_the_loader_waits_for_what_is_in_flight(tmp_path):
    src, exe = tmp_path / "drain.cu", tmp_path / "drain"
    src.write_text(PROGRAM)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17",
                           "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include"), "-I",
                           os.path.join(ROOT, "paper_2406_17611_b200", "csrc"), str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)], capture_output=True, text=True, timeout=60).stdout.strip() == "0"


def test_the_kernels_wait_before_they_free_tmem():
    """Each loader and each issuer ends with its drain, on the way that passes too: who gave up may be another role, later."""
    base = os.path.join(ROOT, "paper_2406_17611_b200", "csrc")
    for name, kernels in (("gemm_tc.cu", 2), (os.path.join("ops", "fp8_product.cu"), 1)):
        text = open(os.path.join(base, name)).read()
        assert text.count("tmem_dealloc(") == kernels
        assert text.count("      drain_loads<") == kernels and text.count("      drain_umma(") == kernels
        assert "mbar_try_wait(" not in text
