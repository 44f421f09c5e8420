"""Places and steps of the fp32 products (csrc/f32_shape.h), asked on the host, up to the largest numbers of rows."""
import os
import subprocess

import pytest

from paper_2410_23608_amd import build as spa_build

ROCM = os.path.dirname(os.path.dirname(spa_build.HIPCC))
CLANGXX = os.path.join(ROCM, "lib", "llvm", "bin", "clang++")
MAIN = r"""
#include <cstdio>
#include "f32_shape.h"
using namespace spa;
int main() {
  const int most = 2147483647;
  for (int step : {16, 32, 64}) {
    for (int n : {-5, 0}) if (f32_steps(n, step) != 0) return 1;
    for (int n : {1, 15, 16, 17, 63, 64, 65, 1000, most - 64, most - 63, most - 33, most - 32, most - 1, most}) {
      const int steps = f32_steps(n, step);
      if ((long)steps * step < n || (long)(steps - 1) * step >= n) return 2;
      for (int s : {0, steps / 2, steps - 1})
        for (int i = 0; i < step; ++i) {
          const long at = (long)s * step + i;
          if (f32_inside(s * step, i, n) != (at < n)) return 3;
          if (f32_at(s * step, i, n) != (at < n ? at : n - 1)) return 4;
        }
    }
  }
  return 0;
}
"""


def test_places_and_steps_up_to_the_largest_numbers(tmp_path):
    if not os.path.exists(CLANGXX):
        pytest.skip("needs ROCm's clang++")
    (tmp_path / "main.cpp").write_text(MAIN)
    cmd = [CLANGXX, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I",
           os.path.join(ROCM, "include"), "-I", spa_build.CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr)
