"""Workgroups of a launch with the small tiles of the projections (csrc/gemm_shape.h), asked on the host."""
import os
import subprocess

import pytest

from paper_2410_23608_amd import build as spa_build

ROCM = os.path.dirname(os.path.dirname(spa_build.HIPCC))
CLANGXX = os.path.join(ROCM, "lib", "llvm", "bin", "clang++")
MAIN = r"""
#include <cstdio>
#include "gemm_shape.h"
int main() {
  for (int m : {1, 64, 196, 392, 1000, 2000, 4000, 8000, 16000, 20000, 21000})
    for (int n : {8, 64, 72, 384, 768, 2000}) {
      if (!spa::tiny_tiles(m, true, n)) continue;
      const long tiles = spa::gemm_tiles<long>(m, n, 64), few = spa::tiny_groups(m, n, false), all = spa::tiny_groups(m, n, true);
      if (few % 8 || few < tiles || few >= tiles + 8) return 1;
      // every tile has a workgroup; with other rows two waves each are the eight of a 128 x 128 tile, unless that is more than a round
      const long waves = 8 * ((spa::gemm_tiles<long>(m, n, 128) + 7) / 8 * 8);
      if (all % 8 || all < few || (2 * all < waves && all < 512) || (all > few && all > 512)) return 2;
    }
  return 0;
}
"""


def test_workgroups_for_tiles_and_other_rows(tmp_path):
    if not os.path.exists(CLANGXX):
        pytest.skip("needs ROCm's clang++")
    (tmp_path / "main.cpp").write_text(MAIN)
    cmd = [CLANGXX, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I",
           os.path.join(ROCM, "include"), "-I", spa_build.CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    assert subprocess.run([str(tmp_path / "main")]).returncode == 0
