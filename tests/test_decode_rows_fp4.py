"""How decode attention over caches held in 4 bits is cut into pieces, compiled for the host.  No GPU needed."""
import os
import subprocess

import pytest

from paper_2605_23258_amd import build

# every pair of lengths, few and many (sequence, head) pairs, both costs of an approximated row, two and three workgroups per CU: a piece for each kind of row that there is
# and none for one that there is not, no more than the workspace holds, no piece without a step, and one where nothing is cached
PROGRAM = r"""
#include <cstdio>
#include "decode_rows.hpp"
int main() {
  const int rows[] = {0, 1, 127, 128, 129, 1000, 5000, 40000, 1000001, 2147483647};
  const int pairs[][2] = {{1, 1}, {1, 8}, {3, 2}, {16, 8}, {100, 1}, {24, 8}, {65535, 1}, {4096, 64}, {65535, 65535}};
  for (int ret : rows)
    for (int apx : rows)
      for (auto& p : pairs)
        for (int kind = 0; kind < 4; ++kind) {
          int r = -1, a = -1;
          vec::pick_splits_fp4(p[0], p[1], ret, apx, kind & 1 ? vec::kFp4Turned : vec::kFp4Approx, kind & 2 ? 2 : 3, r, a);
          const long long steps_r = (ret + 127ll) / 128, steps_a = (apx + 127ll) / 128;
          const bool ok = r >= 0 && a >= 0 && r + a >= 1 && r + a <= vec::kMaxSplits && (steps_a > 0 ? a >= 1 && a <= steps_a : a == 0) &&
                          (steps_r > 0 ? r >= 1 && r <= steps_r : r == (steps_a == 0 ? 1 : 0));
          // and together no more workgroups than run at the same time, unless the pairs alone are more
          const long long at_once = 256ll * (kind & 2 ? 2 : 3), n = (long long)p[0] * p[1];
          const bool fits = n * (r + a) <= at_once || r + a <= 2;
          if (!ok || !fits) {
            printf("rows %d, %d of %d x %d, kind %d: %d and %d pieces\n", ret, apx, p[0], p[1], kind, r, a);
            return 1;
          }
        }
  return 0;
}
"""


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs the ROCm toolchain")
def test_pieces_of_4_bit_caches(tmp_path):
    (tmp_path / "pieces.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "pieces")
    subprocess.run([os.path.join(os.path.dirname(build.HIPCC), "amdclang++"), "-std=c++17", "-O2", "-w", "-I", build.CSRC,
                    str(tmp_path / "pieces.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
