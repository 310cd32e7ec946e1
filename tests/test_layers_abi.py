"""Layers of normalised residual networks: the binding's argument blocks have
the header's layout, and invalid arguments are refused on the host before any
HIP call (these run without a GPU)."""
import os
import subprocess

import pytest
import torch

from paper_1910_13444_amd import pigan

needs_lib = pytest.mark.skipif(not os.path.exists(pigan.LIB_PATH), reason="libpigan.so not built")

PROGRAM = r"""
#include <stddef.h>
#include <stdio.h>
#include "pigan.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu\n", sizeof(pigan_linear), offsetof(pigan_linear, M), offsetof(pigan_linear, x),
         offsetof(pigan_linear, dx), offsetof(pigan_linear, db));
  printf("%zu %zu %zu\n", sizeof(pigan_act_args), offsetof(pigan_act_args, M), offsetof(pigan_act_args, g));
  printf("%zu %zu %zu %zu %zu\n", sizeof(pigan_norm), offsetof(pigan_norm, eps), offsetof(pigan_norm, x),
         offsetof(pigan_norm, gamma), offsetof(pigan_norm, dbeta));
  return 0;
}
"""


def test_argument_blocks_have_the_headers_layout(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(PROGRAM)
    r = subprocess.run(["gcc", "-I", os.path.dirname(pigan.HEADER), str(src), "-o", str(exe)], capture_output=True,
                       text=True)
    assert r.returncode == 0, r.stderr
    lines = [[int(v) for v in ln.split()] for ln in subprocess.check_output([str(exe)], text=True).splitlines()]
    mat = 24
    assert lines[0] == [pigan.LINEAR_ARGS.size, 16, 40, 40 + 6 * mat, 40 + 7 * mat + 16]
    assert lines[1] == [pigan.ACT_ARGS.size, 16, 32 + 2 * mat]
    assert lines[2] == [pigan.NORM_ARGS.size, 24, 32, 32 + 5 * mat, 32 + 5 * mat + 40]


FAKE = 4096   # never dereferenced
M, K, N = 10, 24, 16


def _linear(G=1, dt=1, act=0, reserved=0, m=M, k=K, n=N, x=None, w=None, y=None, pre=(0, 0, 0), add=(0, 0, 0),
            g=None, dx=None, bias=FAKE, dw=FAKE, db=FAKE):
    d = dict(x=x or (FAKE, K, M * K), w=w or (FAKE, K, N * K), y=y or (FAKE, N, M * N), g=g or (FAKE, N, M * N),
             dx=dx or (FAKE, K, M * K))
    return pigan.LINEAR_ARGS.pack(G, dt, act, reserved, m, k, n, *d["x"], *d["w"], *d["y"], *pre, *add, *d["g"],
                                  *d["dx"], bias, dw, db)


BAD_LINEAR = [dict(G=0), dict(G=65536), dict(dt=3), dict(dt=-1), dict(act=5), dict(act=-1), dict(reserved=1),
              dict(m=-1), dict(m=1 << 31), dict(k=0), dict(n=0), dict(n=1 << 31), dict(x=(0, K, 0)),
              dict(x=(FAKE + 1, K, 0)), dict(x=(FAKE, K - 1, 0)), dict(x=(FAKE, 1 << 41, 0)), dict(w=(0, K, 0)),
              dict(w=(FAKE, 3, 0)), dict(G=2, x=(FAKE, K, M * K - 1)), dict(G=2, w=(FAKE, K, 0)),
              dict(G=2, x=(FAKE, K, 1 << 47))]


@needs_lib
@pytest.mark.parametrize("bad", BAD_LINEAR + [dict(y=(0, N, 0)), dict(y=(FAKE, N - 1, 0)), dict(pre=(FAKE, 1, 0)),
                                              dict(add=(FAKE + 1, N, 0)), dict(bias=FAKE + 2)])
def test_linear_forward_refuses(bad):
    L = pigan.lib()
    assert L.pigan_linear_forward(_linear(**bad), FAKE, 1 << 40, None) == pigan.EINVAL
    assert pigan.lib().pigan_last_error()


@needs_lib
@pytest.mark.parametrize("bad", BAD_LINEAR + [dict(g=(0, N, 0)), dict(g=(FAKE, N - 1, 0)), dict(dx=(FAKE, 1, 0)),
                                              dict(act=1), dict(pre=(FAKE, K, 0)), dict(act=1, pre=(FAKE, 2, 0)),
                                              dict(add=(FAKE, 2, 0)), dict(dw=FAKE + 1), dict(db=FAKE + 2),
                                              dict(dx=(0, 0, 0), dw=0, db=0)])
def test_linear_backward_refuses(bad):
    L = pigan.lib()
    assert L.pigan_linear_backward(_linear(**bad), FAKE, 1 << 40, None) == pigan.EINVAL
    assert pigan.lib().pigan_last_error()


@needs_lib
def test_workspaces():
    L = pigan.lib()
    assert L.pigan_linear_forward_workspace(_linear(k=0)) == 0 and L.pigan_linear_forward_workspace(None) == 0
    assert L.pigan_linear_backward_workspace(_linear(dt=9)) == 0 and L.pigan_linear_backward_workspace(None) == 0
    assert L.pigan_linear_forward_workspace(_linear()) == 1
    big = dict(dt=0, m=30000, x=(FAKE, K, 0), y=(FAKE, N, 0), g=(FAKE, N, 0), dx=(FAKE, K, 0), n=600, w=(FAKE, K, 0))
    big.update(y=(FAKE, 600, 0), g=(FAKE, 600, 0), k=K)
    for query, call in ((L.pigan_linear_forward_workspace, L.pigan_linear_forward),
                        (L.pigan_linear_backward_workspace, L.pigan_linear_backward)):
        a = _linear(**big)
        need = query(a)
        assert need > 3 * 2 * 30000 * K
        assert call(a, FAKE, need - 1, None) == pigan.EWORKSPACE
        assert call(a, None, need, None) == pigan.EWORKSPACE
        assert call(a, FAKE + 16, need, None) == pigan.EINVAL
    # M = 0: nothing is launched
    assert L.pigan_linear_forward(_linear(m=0, x=(0, 0, 0), y=(0, 0, 0)), None, 0, None) == pigan.OK


def _norm(G=1, dt=1, m=M, n=N, eps=1e-5, reserved=0, x=None, y=None, dy=None, add=(0, 0, 0), dx=None, gamma=FAKE,
          beta=FAKE, mean=FAKE, rstd=FAKE, dgamma=FAKE, dbeta=FAKE):
    d = (FAKE, N, M * N)
    return pigan.NORM_ARGS.pack(G, dt, m, n, eps, reserved, *(x or d), *(y or d), *(dy or d), *add,
                                *(dx or (2 * FAKE, N, M * N)), gamma, beta, mean, rstd, dgamma, dbeta)


BAD_NORM = [dict(G=0), dict(dt=4), dict(m=-1), dict(n=0), dict(reserved=2), dict(x=(0, N, 0)), dict(x=(FAKE, 3, 0)),
            dict(x=(FAKE + 1, N, 0)), dict(G=2, x=(FAKE, N, 5)), dict(gamma=FAKE + 1), dict(mean=FAKE + 3)]


@needs_lib
@pytest.mark.parametrize("bad", BAD_NORM + [dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                                            dict(eps=float("inf")), dict(y=(0, N, 0)), dict(y=(FAKE, 1, 0))])
def test_layer_norm_forward_refuses(bad):
    assert pigan.lib().pigan_layer_norm_forward(_norm(**bad), None) == pigan.EINVAL


@needs_lib
@pytest.mark.parametrize("bad", BAD_NORM + [dict(dy=(0, N, 0)), dict(dy=(FAKE, 1, 0)), dict(dx=(2 * FAKE, 1, 0)),
                                            dict(add=(FAKE, 1, 0)), dict(mean=0), dict(rstd=0), dict(dx=(FAKE, N, 0)),
                                            dict(dx=(0, 0, 0), dgamma=0, dbeta=0)])
def test_layer_norm_backward_refuses(bad):
    assert pigan.lib().pigan_layer_norm_backward(_norm(**bad), FAKE, 1 << 40, None) == pigan.EINVAL


@needs_lib
def test_layer_norm_workspace():
    L = pigan.lib()
    a = _norm(m=5000)
    need = L.pigan_layer_norm_backward_workspace(a)
    assert need > 1 and L.pigan_layer_norm_backward_workspace(_norm(n=0)) == 0
    assert L.pigan_layer_norm_backward_workspace(_norm(m=5000, dgamma=0, dbeta=0)) == 1
    assert L.pigan_layer_norm_backward(a, FAKE, need - 1, None) == pigan.EWORKSPACE
    assert L.pigan_layer_norm_backward(a, None, need, None) == pigan.EWORKSPACE


@needs_lib
@pytest.mark.parametrize("bad", [dict(G=0), dict(dt=7), dict(act=0), dict(act=9), dict(reserved=1), dict(m=-2),
                                 dict(n=0), dict(dy=(0, N, 0)), dict(pre=(FAKE, 2, 0)), dict(g=(FAKE + 1, N, 0))])
def test_act_backward_refuses(bad):
    d = dict(G=1, dt=1, act=1, reserved=0, m=M, n=N, dy=(FAKE, N, 0), pre=(FAKE, N, 0), g=(FAKE, N, 0))
    d.update(bad)
    a = pigan.ACT_ARGS.pack(d["G"], d["dt"], d["act"], d["reserved"], d["m"], d["n"], *d["dy"], *d["pre"], *d["g"])
    assert pigan.lib().pigan_act_backward(a, None) == pigan.EINVAL


@needs_lib
def test_null_arguments():
    L = pigan.lib()
    assert L.pigan_linear_forward(None, None, 0, None) == pigan.EINVAL
    assert L.pigan_linear_backward(None, None, 0, None) == pigan.EINVAL
    assert L.pigan_act_backward(None, None) == pigan.EINVAL
    assert L.pigan_layer_norm_forward(None, None) == pigan.EINVAL
    assert L.pigan_layer_norm_backward(None, None, 0, None) == pigan.EINVAL


@needs_lib
def test_binding_refuses():
    """The Python entry points: host tensors, types, shapes, strides."""
    def zeros(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype)
    x, w = zeros(4, 8), zeros(6, 8)
    for call in (lambda: pigan.linear(x, w), lambda: pigan.linear_backward(zeros(4, 6), x, w),
                 lambda: pigan.act_backward(x, x, "tanh"), lambda: pigan.layer_norm(x),
                 lambda: pigan.layer_norm_backward(x, x, zeros(4), zeros(4))):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    like = zeros(1)
    with pytest.raises(ValueError, match="must be torch.float32"):
        pigan._mat(zeros(2, 3, dtype=torch.float16), "x", like, (2, 3))
    with pytest.raises(ValueError, match="shape"):
        pigan._mat(zeros(2, 3), "x", like, (3, 2))
    with pytest.raises(ValueError, match="unit stride"):
        pigan._mat(zeros(3, 2).t(), "x", like, (2, 3))
    with pytest.raises(ValueError, match="overlapping rows"):
        pigan._mat(zeros(3).expand(2, 3), "x", like, (2, 3))
    with pytest.raises(ValueError, match="overlapping groups"):
        pigan._mat(zeros(2, 3).expand(4, 2, 3), "x", like, (4, 2, 3))
    with pytest.raises(ValueError, match="contiguous"):
        pigan._vec(zeros(8)[::2], "bias", like, (4,))
    with pytest.raises(ValueError, match="unknown activation"):
        pigan._act("softplus")
    assert pigan._mat(zeros(2, 9)[:, 1:4], "x", like, (2, 3))[1] == 9
    assert pigan._mat(zeros(5, 1).t(), "x", like, (1, 5))[1] == 5
