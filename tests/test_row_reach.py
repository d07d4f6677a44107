"""The rows whose covering 16-byte vectors may reach beyond their matrix, as the block norms' kernels decide it, against every narrow matrix there is
(no device is needed)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
#include <cstdio>
#include "jp_internal.h"
int main() {                                                   // the kernels' test: t < n, t + n >= T
  long missed = 0, guarded = 0, rows = 0;
  for (int es = 2; es <= 4; es += 2)
    for (int T = 1; T <= 20; ++T)
      for (int H = 1; H <= 10; ++H)
        for (int ld = H; ld <= 12; ++ld)
          for (int t = 0; t < T; ++t) {
            bool front = false, behind = false;               // wherever the matrix starts
            for (int start = 0; start < 16; start += es) {
              const int lo = 64 + start, hi = lo + ((T - 1) * ld + H) * es, row = lo + t * ld * es, end = row + H * es;
              front |= row / 16 * 16 < lo;
              behind |= (end + 15) / 16 * 16 > hi;
            }
            const int n = jp::rows_near_an_end(ld * es);
            const bool f = t < n, b = t + n >= T;
            missed += (front && !f) + (behind && !b);
            guarded += (T == 20 && ld == 12) && (f || b);
            rows += T == 20 && ld == 12;
          }
  std::printf("%ld %d", missed, guarded * 9 < rows);
}
"""


def test_rows_that_reach_beyond_the_matrix(tmp_path):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PROGRAM)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2602_06107_b200", "csrc"),
                    "-I", os.path.join(cuda, "include"), "-c", "-o", str(exe) + ".o", str(src)], check=True)
    subprocess.run(["g++", "-o", str(exe), str(exe) + ".o", "-L", os.path.join(cuda, "lib64"), "-lcudart"], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True, env={**os.environ, "LD_LIBRARY_PATH": os.path.join(cuda, "lib64")}).stdout
    assert out.split() == ["0", "1"]     # (and of wide rows hardly any but the first and the last)
