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


RULE = r"""
#include <cstdio>
#include "f32_shape.h"
int main() {
  int side; long rows, cols, kc;
  while (std::scanf("%d %ld %ld %ld", &side, &rows, &cols, &kc) == 4) std::printf("%d\n", (int)spa::f32_by_element((spa::F32Side)side, rows, cols, kc));
}
"""
FORWARD, INPUT, WEIGHT = 0, 1, 2


@pytest.fixture(scope="module")
def by_element(tmp_path_factory):
    if not os.path.exists(CLANGXX):
        pytest.skip("needs ROCm's clang++")
    d = tmp_path_factory.mktemp("f32_rule")
    (d / "main.cpp").write_text(RULE)
    cmd = [CLANGXX, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I",
           os.path.join(ROCM, "include"), "-I", spa_build.CSRC, str(d / "main.cpp"), "-o", str(d / "main")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]

    def ask(side, calls):
        text = "\n".join(f"{side} {rows} {cols} {kc}" for rows, cols, kc in calls)
        out = subprocess.run([str(d / "main")], input=text, capture_output=True, text=True, check=True).stdout
        return [line == "1" for line in out.split()]

    return ask


def test_the_side_that_measured_faster(by_element):
    """(rows, columns, contraction) -> a thread an element, at the sizes stated at the rule and others that differ by a fifth and more."""
    forward = {(1000000, 1, 1): 1, (300000, 4, 4): 1, (300000, 1, 16): 1, (300000, 16, 8): 0, (300000, 64, 4): 0, (20000, 4, 16): 1, (20000, 512, 4): 0, (1000, 64, 8): 1,
               (300000, 4, 8): 1, (300000, 16, 4): 1, (20000, 1, 32): 1, (1000, 512, 8): 0, (64, 64, 32): 0, (1000, 1000, 1): 1, (1, 64, 64): 0, (1, 1000, 1000): 0,
               (8, 4096, 4096): 0, (100, 64, 64): 0, (20000, 64, 64): 0, (1000000, 32, 32): 0, (1000000, 8, 1): 1, (1000000, 1, 8): 1, (300000, 4, 16): 1}
    back = {(300000, 16, 8): 1, (300000, 64, 8): 0, (300000, 16, 16): 1, (300000, 64, 16): 0, (1000, 512, 8): 1, (20000, 512, 8): 0, (1000, 1, 8): 1, (64, 64, 32): 0,
            (1000, 1000, 1000): 0, (200000, 32, 8): 1, (100, 64, 192): 0}
    weight = {(64, 64, 1): 1, (64, 64, 8): 1, (64, 64, 32): 0, (1000, 1000, 1): 1, (1000, 1000, 4): 0, (1024, 4096, 2): 0, (1024, 4096, 1): 1, (64, 64, 100): 0, (64, 64, 100000): 0}
    for side, sizes in ((FORWARD, forward), (INPUT, back), (WEIGHT, weight)):
        assert by_element(side, list(sizes)) == [bool(v) for v in sizes.values()], side


def test_the_sides_of_the_calls_compared_on_the_gpu(by_element):
    """Each pair of tests/test_gpu_f32_short.py: few columns a thread an element, many in tiles."""
    for side, many, pairs in ((FORWARD, 512, [(1, 64), (3, 16), (4, 1), (8, 4), (8, 33), (16, 3)]), (INPUT, 4000, [(1, 64), (4, 16), (8, 1), (8, 33), (16, 4)])):
        assert all(by_element(side, [(1000, few, kc) for kc, few in pairs]))
        assert not any(by_element(side, [(1000, many, kc) for kc, _ in pairs if kc > 4]))
    assert all(by_element(WEIGHT, [(70, 33, m) for m in (1, 4, 8)])) and by_element(WEIGHT, [(1500, 1500, m) for m in (1, 4, 8)]) == [True, False, False]


def test_the_largest_calls(by_element):
    """No overflow, and tiles where there is work."""
    most = 2 ** 31 - 1
    assert by_element(FORWARD, [(most, 1, 1), (most, most, most)]) == [True, False]
    assert by_element(INPUT, [(most, most, most)]) == by_element(WEIGHT, [(most, most, most)]) == [False]
