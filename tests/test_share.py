"""How workgroups share rows or keys (csrc/share.h), asked on the host, up to the longest sequences; and what is refused beyond them."""
import os
import subprocess

import pytest

from paper_2410_23608_amd import build as spa_build
from paper_2410_23608_amd import spa

ROCM = os.path.dirname(os.path.dirname(spa_build.HIPCC))
CLANGXX = os.path.join(ROCM, "lib", "llvm", "bin", "clang++")
MAIN = r"""
#include "share.h"
using spa::share_of;
template <int STEP>
int check(int n, int splits) {
  long at = 0;
  int live = 0;
  const spa::Share first = share_of<STEP>(n, splits, 0);
  for (int s = 0; s < splits; ++s) {
    const spa::Share sh = share_of<STEP>(n, splits, s);
    if (sh.live != first.live) return 1;
    if (sh.n <= 0) continue;
    if (sh.from != at || sh.from % STEP || sh.n > first.n || (s + 1 < first.live && (sh.n != first.n || sh.n % STEP)) || s != live) return 2;
    at += sh.n;
    ++live;
  }
  if (at != (n > 0 ? n : 0)) return 3;
  return n > 0 && live != first.live ? 4 : 0;
}
int main() {
  const int most = 2147483647 - 257;
  for (int splits : {2, 3, 4, 7, 37, 512, 1023, 1024})
    for (int n : {0, 1, 63, 64, 65, 127, 128, 129, 1000, 16000, 1000003, 1431655765, 1500000000, most - 64, most - 1, most})
      if (const int bad = check<64>(n, splits) + 10 * check<128>(n, splits)) return bad;
  const spa::Share all = share_of<64>(most, 1, 0);
  return all.from == 0 && all.n == most && all.live == 1 ? 0 : 99;
}
"""


def test_shares_up_to_the_longest_sequences(tmp_path):
    if not os.path.exists(CLANGXX):
        pytest.skip("needs ROCm's clang++")
    (tmp_path / "main.cpp").write_text(MAIN)
    cmd = [CLANGXX, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I",
           os.path.join(ROCM, "include"), "-I", spa_build.CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr)


def test_longer_ones_are_refused():
    lib, F, most = spa.lib, 4096, 2 ** 31 - 258
    for max_q, max_k in ((1, most + 1), (1, 2 ** 31 - 2), (most + 1, 1)):
        sizes = (1, max_q, max_k, 1, 1, 32, 1)
        assert lib.spa_cross_attention_workspace_bytes(*sizes) == lib.spa_cross_attention_bwd_workspace_bytes(*sizes) == 0
        assert lib.spa_cross_attention(F, F, F, 32, 32, 32, F, F, None, *sizes, 0.0, F, None, F, 1 << 60, None) == -1
        assert "2^31 - 257" in lib.spa_last_error().decode()
        assert lib.spa_cross_attention_bwd(F, F, F, 32, 32, 32, F, F, F, F, F, None, *sizes, 0.0, F, F, F, 32, 32, 32, F, 1 << 60, None) == -1
        assert "2^31 - 257" in lib.spa_last_error().decode()
    assert lib.spa_cross_attention_workspace_bytes(1, 1, most, 1, 1, 32, 1) > 0
