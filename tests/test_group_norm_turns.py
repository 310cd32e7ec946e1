"""How a block of group norm walks the turns of a long sample (from the last to the first),
on the CPU: a small program is compiled against the kernels' header."""
import os
import subprocess

import pytest

from paper_1910_13444_amd import build

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "group_norm_parts.h"
using namespace pigan;

// the loop of the results' kernels: turns of U rows, f(first point, points from there on)
template <class F> static bool walk(const Turns& tn, F&& f) {
  if (tn.left <= 0) return true;
  const int64_t most = tn.left / tn.by + 1;
  int left = tn.left - tn.last();
  int64_t p = tn.first + tn.last(), turns = 0;
  for (;;) {
    if (++turns > most || left < 1 || left > tn.left) return false;
    f(p, left);
    if (!tn.before(left)) break;
    left += tn.by;
    p -= tn.by;
  }
  return p == tn.first && left == tn.left;
}

int main() {
  int bad = 0;
  GnPlan pl{};
  // short samples: every point once
  for (int rows : {1, 3, 32, 256})
    for (int splits : {1, 2, 7, 40})
      for (int U : {2, 4})
        for (int64_t P : {1, 2, 31, 257, 4097, 70001}) {
          pl.rows = rows;
          std::vector<int> seen(P, 0);
          for (int split = 0; split < splits; ++split)
            for (int row = 0; row < rows; ++row)
              if (!walk(Turns(pl, P, U, split, splits, row), [&](int64_t p, int left) {
                    for (int v = 0; v < U; ++v)
                      if (v == 0 || v * rows < left) p + v * rows < P && p >= 0 ? (void)++seen[p + v * rows] : (void)++bad;
                  })) ++bad;
          for (int n : seen) bad += n != 1;
        }
  // the longest ones: every turn begins within the sample, the last one at the first point
  for (int64_t P : {(int64_t)0x7fffffff, (int64_t)0x7fffffff - 393216, (int64_t)0x7fffffff - 655361, (int64_t)0x7ffffffe})
    for (int rows : {1, 32, 256})
      for (int splits : {1, 384, 768, 1280})
        for (int U : {2, 4})
          for (int split : {0, 1, splits / 2, splits - 1})
            for (int row : {0, rows - 1}) {
              pl.rows = rows;
              if (split >= splits || (int64_t)splits * U * rows < 3000) continue;   // millions of turns
              const Turns tn(pl, P, U, split, splits, row);
              if (!walk(tn, [&](int64_t p, int left) { bad += p < 0 || p >= P || p + left != P; })) ++bad;
            }
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_turns_stay_within_a_sample(tmp_path):
    if not os.path.exists(build.hipcc()) or not os.path.exists(build.LIB):
        pytest.skip("hipcc or the library is not available")
    src, exe = tmp_path / "turns.cpp", str(tmp_path / "turns")
    src.write_text(PROGRAM)
    r = subprocess.run([build.hipcc(), *build.common_flags(), "-xhip", str(src), "-xnone", build.LIB,
                        "-Wl,-rpath," + os.path.dirname(build.LIB), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100,
                       env={**os.environ, "HIP_VISIBLE_DEVICES": "-1", "ROCR_VISIBLE_DEVICES": "-1"})
    assert r.returncode == 0, r.stdout + r.stderr
