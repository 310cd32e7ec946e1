"""Group norm's argument block and refusals, and the checks of overlapping operands
against byte by byte ones (these run without a GPU)."""
import os
import subprocess

import pytest
import torch

from paper_1910_13444_amd import build, pigan

needs_lib = pytest.mark.skipif(not os.path.exists(pigan.LIB_PATH), reason="libpigan.so not built")

PROGRAM = r"""
#include <stddef.h>
#include <stdio.h>
#include "pigan.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu\n", sizeof(pigan_group_norm), offsetof(pigan_group_norm, eps),
         offsetof(pigan_group_norm, S), offsetof(pigan_group_norm, n), offsetof(pigan_group_norm, x),
         offsetof(pigan_group_norm, dx), offsetof(pigan_group_norm, dbeta));
  return 0;
}
"""


def test_argument_block_has_the_headers_layout(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(PROGRAM)
    r = subprocess.run(["gcc", "-I", os.path.dirname(pigan.HEADER), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = [int(v) for v in subprocess.check_output([str(exe)], text=True).split()]
    assert got == [pigan.GROUP_NORM_ARGS.size, 12, 16, 40, 48, 48 + 4 * 32, 48 + 5 * 32 + 40]


FAKE = 4096   # never dereferenced
S, P, C, N = 3, 5, 24, 4
FIELD = (FAKE, C, P * C, S * P * C)
FAR = (1 << 24, C, P * C, S * P * C)
NONE = (0, 0, 0, 0)


def _args(G=1, dt=1, act=2, eps=1e-5, s=S, p=P, c=C, n=N, x=FIELD, y=FAR, dy=FIELD, add=NONE, dx=FAR, gamma=FAKE, beta=FAKE,
          mean=FAKE, rstd=FAKE, dgamma=1 << 25, dbeta=1 << 26):
    return pigan.GROUP_NORM_ARGS.pack(G, dt, act, eps, s, p, c, n, *x, *y, *dy, *add, *dx, gamma, beta, mean, rstd, dgamma,
                                      dbeta)


BAD = [dict(G=0), dict(G=65536), dict(dt=3), dict(act=5), dict(act=-1), dict(s=-1), dict(s=1 << 31), dict(p=0), dict(p=1 << 31),
       dict(c=0), dict(c=1 << 31), dict(n=0), dict(n=5), dict(n=25), dict(n=-4), dict(x=NONE), dict(x=(FAKE + 1, C, P * C, 0)),
       dict(x=(FAKE, C - 1, P * C, 0)), dict(x=(FAKE, C, P * C - 1, 0)), dict(x=(FAKE, 1 << 45, 1 << 45, 0)),
       dict(x=(FAKE, C, 1 << 46, 0)), dict(G=2, x=(FAKE, C, P * C, S * P * C - 1)), dict(gamma=FAKE + 1), dict(beta=FAKE + 2),
       dict(mean=FAKE + 1), dict(s=1 << 30, p=1 << 30)]
OVERLAPS = [dict(y=(FAKE + 2, C, P * C, 0)), dict(y=(FAKE, C, P * C + 1, 0)), dict(mean=1 << 24), dict(gamma=1 << 24)]


@needs_lib
@pytest.mark.parametrize("bad", BAD + [dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(y=NONE),
                                       dict(y=(1 << 24, C - 1, P * C, 0))] + OVERLAPS + [dict(rstd=FAKE, mean=FAKE)])
def test_forward_refuses(bad):
    L = pigan.lib()
    assert L.pigan_group_norm_forward(_args(**bad), 1 << 30, 1 << 30, None) == pigan.EINVAL
    assert L.pigan_last_error()


@needs_lib
@pytest.mark.parametrize("bad", BAD + [dict(dy=NONE), dict(dy=(FAKE, 3, P * C, 0)), dict(dx=(1 << 24, 3, P * C, 0)),
                                       dict(add=(FAKE + 1, C, P * C, 0)), dict(mean=0), dict(rstd=0),
                                       dict(dx=NONE, dgamma=0, dbeta=0), dict(dgamma=(1 << 25) + 2), dict(dgamma=1 << 26),
                                       dict(dx=(FAKE + 2, C, P * C, 0)), dict(x=FAR), dict(dgamma=FAKE), dict(s=1, p=4000, dbeta=1 << 30)])
def test_backward_refuses(bad):
    L = pigan.lib()
    assert L.pigan_group_norm_backward(_args(**bad), 1 << 30, 1 << 30, None) == pigan.EINVAL
    assert L.pigan_last_error()


@needs_lib
def test_workspaces():
    L = pigan.lib()
    for query, call in ((L.pigan_group_norm_forward_workspace, L.pigan_group_norm_forward),
                        (L.pigan_group_norm_backward_workspace, L.pigan_group_norm_backward)):
        assert query(None) == 0 and query(_args(n=5)) == 0 and call(None, None, 0, None) == pigan.EINVAL
        assert query(_args(s=0)) == 1
        long = dict(p=1 << 20, x=(1 << 32, C, C << 20, 0), y=(1 << 34, C, C << 20, 0), dy=(1 << 35, C, C << 20, 0),
                    dx=(1 << 36, C, C << 20, 0))
        a = _args(**long)
        need = query(a)
        assert need > 1
        assert call(a, 1 << 40, need - 1, None) == pigan.EWORKSPACE
        assert call(a, None, need, None) == pigan.EWORKSPACE
        assert call(a, (1 << 40) + 16, need, None) == pigan.EINVAL
        assert call(a, 1 << 32, need, None) == pigan.EINVAL   # over x
    assert L.pigan_group_norm_forward(_args(s=0, x=NONE, y=NONE), None, 0, None) == pigan.OK


OVERLAP = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include "operands.h"
using namespace pigan;
static Runs random_runs(const char* name, int64_t base) {
  int64_t len = 1 + rand() % 6, n[3], st[3], extent = len;
  for (int i = 0; i < 3; ++i) {
    n[i] = 1 + rand() % 4;
    st[i] = extent + (rand() % 2 ? 0 : rand() % 9);
    extent += (n[i] - 1) * st[i];
  }
  return Runs(name, (void*)(base + rand() % 200), len).repeat(n[0], st[0]).repeat(n[1], st[1]).repeat(n[2], st[2]);
}
static void bytes(const Runs& r, int level, int64_t at, std::set<int64_t>& to) {
  if (level == 0) { for (int64_t i = 0; i < r.len; ++i) to.insert(at + i); return; }
  for (int64_t i = 0; i < r.n[level - 1]; ++i) bytes(r, level - 1, at + i * r.st[level - 1], to);
}
int main() {
  int wrong = 0, met = 0, apart = 0;
  for (int k = 0; k < 200000; ++k) {
    Runs a = random_runs("a", 1000), b = random_runs("b", 1000);
    if (k % 2) {   // of equal strides
      const int64_t p = b.p;
      b = a;
      b.p = p;
      for (int i = 0; i < b.levels; ++i) b.n[i] = 1 + rand() % b.n[i];
    }
    bool alike = a.levels == b.levels;
    for (int i = 0; i < a.levels && alike; ++i) alike = a.st[i] == b.st[i];
    if (a.levels && b.levels && !alike) continue;   // told only where they begin at one address
    std::set<int64_t> x, y;
    bytes(a, a.levels, a.p, x);
    bytes(b, b.levels, b.p, y);
    bool meet = false;
    for (int64_t v : x) meet = meet || y.count(v);
    wrong += meet != share(a, b) || share(a, b) != share(b, a);
    (meet ? met : apart)++;
  }
  std::printf("%d %d %d\n", wrong, met, apart);
  return wrong || met < 1000 || apart < 1000;
}
"""


def test_overlaps_are_told_exactly(tmp_path):
    if not os.path.exists(build.hipcc()) or not os.path.exists(build.LIB):
        pytest.skip("hipcc or the library is not available")
    src, exe = tmp_path / "overlap.cpp", str(tmp_path / "overlap")
    src.write_text(OVERLAP)
    r = subprocess.run([build.hipcc(), *build.common_flags(), "-xhip", str(src), "-xnone", build.LIB,
                        "-Wl,-rpath," + os.path.dirname(build.LIB), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100,
                       env={**os.environ, "HIP_VISIBLE_DEVICES": "-1", "ROCR_VISIBLE_DEVICES": "-1"})
    assert r.returncode == 0, r.stdout + r.stderr


@needs_lib
def test_binding_refuses():
    def zeros(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype)
    x = zeros(2, 3, 8)
    for call in (lambda: pigan.group_norm(x, 2), lambda: pigan.group_norm_backward(x, x, zeros(2, 2), zeros(2, 2))):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    like = zeros(1)
    for t, what in ((zeros(2, 3, 8, dtype=torch.float16), "must be torch.float32"), (zeros(2, 3, 7), "shape"),
                    (zeros(2, 8, 3).transpose(1, 2), "unit stride"), (zeros(2, 1, 8).expand(2, 3, 8), "overlapping points"),
                    (zeros(1, 3, 8).expand(2, 3, 8), "overlapping samples")):
        with pytest.raises(ValueError, match=what):
            pigan._field(t, "x", like, (2, 3, 8))
    with pytest.raises(ValueError, match="overlapping groups"):
        pigan._field(zeros(1, 2, 3, 8).expand(4, 2, 3, 8), "x", like, (4, 2, 3, 8))
    assert pigan._field(zeros(2, 5, 9)[:, 1:4, :8], "x", like, (2, 3, 8))[1:3] == (9, 45)
