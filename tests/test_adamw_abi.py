"""Tables of many tensors: argument blocks, what is refused, and how a table divides
its tensors (these run without a GPU)."""
import ctypes as C
import os
import struct
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
  printf("%zu %zu %zu\n", sizeof(pigan_tensor), offsetof(pigan_tensor, n), offsetof(pigan_tensor, copy_dt));
  printf("%zu %zu %zu\n", sizeof(pigan_tensors), offsetof(pigan_tensors, tensors), offsetof(pigan_tensors, v_scale));
  printf("%zu %zu %zu %zu\n", sizeof(pigan_adamw), offsetof(pigan_adamw, scale), offsetof(pigan_adamw, step), offsetof(pigan_adamw, t));
  printf("%d\n", PIGAN_ADAMW_WORKSPACE);
  return 0;
}
"""


def test_argument_blocks_have_the_headers_layout(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(PROGRAM)
    r = subprocess.run(["gcc", "-I", os.path.dirname(pigan.HEADER), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = [[int(v) for v in ln.split()] for ln in subprocess.check_output([str(exe)], text=True).splitlines()]
    assert got == [[pigan.TENSOR.size, 24, 44], [pigan.TENSORS_ARGS.size, 8, 40], [pigan.ADAMW_ARGS.size, 48, 72, 80],
                   [pigan.ADAMW_WORKSPACE]]


M = 1 << 20   # addresses, never dereferenced


def _tensor(p=M, g=2 * M, copy=0, n=100, decay=0.0, g_dt=0, copy_dt=0):
    return pigan.TENSOR.pack(p, g, copy, n, decay, g_dt, copy_dt)


def _args(*tensors, bits=8, m=4 * M, v=5 * M, ms=6 * M, vs=7 * M, n=None):
    buf = C.create_string_buffer(b"".join(tensors))
    a = pigan.TENSORS_ARGS.pack(len(tensors) if n is None else n, bits, C.addressof(buf), m, v, ms, vs)
    return a, buf


def _table(*tensors, **kw):
    a, keep = _args(*tensors, **kw)
    L = pigan.lib()
    count, size = L.pigan_tensors_states(a), L.pigan_tensors_table_bytes(a)
    table = (C.c_uint64 * max(1, -(-size // 8)))()
    return L.pigan_tensors_table(a, table, size), table, size, count


@needs_lib
@pytest.mark.parametrize("bits,states", [(0, 0), (32, 1 + 4097 + 300), (8, 256 + 17 * 256 + 512)])
def test_a_table_covers_every_tensor(bits, states):
    st, table, size, count = _table(_tensor(n=1), _tensor(n=0, p=0, g=0), _tensor(p=M + 64, g=2 * M + 2, n=4097, g_dt=1),
                                    _tensor(p=3 * M, n=300, copy=M + (1 << 18), copy_dt=2, decay=0.5), bits=bits)
    assert st == pigan.OK and count == states
    raw = bytes(table)[:size]
    n_tensors, tbits, n_pieces, got = struct.unpack_from("2i2q", raw, 8)
    assert (n_tensors, tbits, n_pieces, got) == (4, bits, 1 + 5 + 1, states)   # pieces of 1024 elements
    entries_at, pieces_at, total = struct.unpack_from("3q", raw, 32)
    assert total == size and pieces_at - entries_at == 4 * 56
    assert [struct.unpack_from("2I", raw, pieces_at + 8 * k) for k in range(7)] == \
        [(0, 0), *((2, k) for k in range(5)), (3, 0)]
    starts = [struct.unpack_from("3P2qd2i", raw, entries_at + 56 * k)[4] for k in range(4)]
    assert starts == {8: [0, 256, 256, 256 + 17 * 256], 32: [0, 1, 1, 4098], 0: [0, 1, 1, 4098]}[bits]


BAD = [dict(n=-1), dict(n=1 << 41), dict(g=0), dict(g=2 * M + 2), dict(g=2 * M + 1, g_dt=1), dict(g_dt=3), dict(g_dt=-1)]
BAD_PARAMS = [dict(p=0), dict(p=M + 2), dict(copy=3 * M), dict(copy=3 * M, copy_dt=3), dict(copy=3 * M + 1, copy_dt=1),
              dict(decay=-0.1), dict(decay=float("inf")), dict(decay=float("nan")), dict(g=M + 8), dict(p=4 * M), dict(g=5 * M + 4),
              dict(copy=M + 4, copy_dt=1), dict(p=6 * M - 4), dict(copy=7 * M, copy_dt=1)]


@needs_lib
@pytest.mark.parametrize("bad", BAD + BAD_PARAMS)
def test_tensors_that_are_refused(bad):
    assert _table(_tensor(p=8 * M, g=9 * M), _tensor(**bad))[0] == pigan.EINVAL
    assert pigan.lib().pigan_last_error()
    if bad in BAD:
        assert _table(_tensor(**bad), bits=0)[0] == pigan.EINVAL


@needs_lib
def test_tables_that_are_refused():
    L = pigan.lib()
    t = _tensor()
    for kw in (dict(bits=16), dict(bits=-8), dict(n=-1), dict(m=0), dict(v=0), dict(ms=0), dict(vs=0), dict(m=4 * M + 2),
               dict(v=5 * M + 1), dict(ms=6 * M + 2), dict(m=5 * M), dict(ms=5 * M + 8), dict(v=M), dict(m=2 * M + 4)):
        assert _table(t, **kw)[0] == pigan.EINVAL, kw
    assert _table(t, t)[0] == pigan.EINVAL                       # a parameter twice
    assert _table(t, _tensor(p=M + 396))[0] == pigan.EINVAL
    assert _table(t, _tensor(p=M + 400))[0] == pigan.OK           # side by side, one gradient
    assert L.pigan_tensors_states(None) == -1 and L.pigan_tensors_table_bytes(None) == 0
    assert L.pigan_tensors_table(None, None, 0) == pigan.EINVAL
    a, keep = _args(t)
    size = L.pigan_tensors_table_bytes(a)
    buf = C.create_string_buffer(size + 16)
    at = (C.addressof(buf) + 7) // 8 * 8
    assert L.pigan_tensors_table(a, at, size) == pigan.OK
    assert L.pigan_tensors_table(a, at, size - 1) == pigan.EINVAL
    assert L.pigan_tensors_table(a, at + 4, size) == pigan.EINVAL
    assert L.pigan_tensors_table(pigan.TENSORS_ARGS.pack(2, 8, 0, 0, 0, 0, 0), at, size) == pigan.EINVAL


def _adamw(table, device=8 * M, lr=1e-3, b1=0.5, b2=0.9, eps=1e-8, scale=1.0, coef=0, skip=0, step=0, t=1, reserved=0):
    return pigan.ADAMW_ARGS.pack(table, device, lr, b1, b2, eps, scale, coef, skip, step, t, reserved)


@needs_lib
def test_calls_that_are_refused():
    L = pigan.lib()
    st, table, size, _ = _table(_tensor())
    assert st == pigan.OK
    at, nan, inf = C.addressof(table), float("nan"), float("inf")
    for kw in (dict(device=0), dict(device=8 * M + 4), dict(lr=inf), dict(lr=nan), dict(b1=1.0), dict(b1=-0.1), dict(b2=nan),
               dict(eps=-1.0), dict(eps=inf), dict(scale=0.0), dict(scale=nan), dict(scale=inf), dict(coef=M + 1), dict(skip=M + 2),
               dict(step=M + 3), dict(t=0), dict(reserved=1), dict(step=M, skip=M), dict(step=M, coef=M)):
        assert L.pigan_adamw_update(_adamw(at, **kw), 16 * M, 256, None) == pigan.EINVAL, kw
    assert L.pigan_adamw_update(_adamw(0), None, 0, None) == pigan.EINVAL
    assert L.pigan_adamw_update(_adamw(at + 8), None, 0, None) == pigan.EINVAL      # not a table
    assert L.pigan_adamw_update(None, None, 0, None) == pigan.EINVAL
    assert L.pigan_adamw_update(_adamw(at, step=M, t=0), None, 0, None) == pigan.EWORKSPACE
    assert L.pigan_adamw_update(_adamw(at, step=M, t=0), 16 * M, 255, None) == pigan.EWORKSPACE
    assert L.pigan_adamw_update(_adamw(at, step=M, t=0), 16 * M + 64, 256, None) == pigan.EINVAL
    st, grads, _, _ = _table(_tensor(), bits=0)
    assert st == pigan.OK
    assert L.pigan_adamw_update(_adamw(C.addressof(grads)), None, 0, None) == pigan.EINVAL
    need = L.pigan_grad_norm_workspace(at)
    assert need >= 8 and L.pigan_grad_norm_workspace(None) == 0

    def norm(table=at, device=8 * M, most=1.0, scale=1.0, out=(M, M + 4, M + 8), ws=16 * M, size=need):
        return L.pigan_grad_norm(table, device, most, scale, *out, ws, size, None)
    for kw in (dict(table=0), dict(device=0), dict(most=0.0), dict(most=nan), dict(most=-1.0), dict(scale=0.0), dict(scale=inf),
               dict(out=(0, 0, 0)), dict(out=(M + 1, 0, 0)), dict(out=(0, M + 2, 0)), dict(out=(M, M, 0)), dict(out=(16 * M, 0, 0)),
               dict(ws=16 * M + 8)):
        assert norm(**kw) == pigan.EINVAL, kw
    assert norm(size=need - 1) == norm(ws=0) == pigan.EWORKSPACE

    def values(n=512, m=M, ms=2 * M, v=3 * M, vs=4 * M, mo=5 * M, vo=6 * M):
        return L.pigan_state_values(n, m, ms, v, vs, mo, vo, None)
    for kw in (dict(n=-256), dict(n=100), dict(mo=0, vo=0), dict(m=0), dict(ms=0), dict(v=0), dict(vs=0), dict(m=M + 1),
               dict(v=M + 2), dict(ms=M + 2), dict(mo=M + 1), dict(mo=M), dict(vo=4 * M), dict(vo=5 * M + 2044)):
        assert values(**kw) == pigan.EINVAL, kw
    assert values(n=0) == pigan.OK


@needs_lib
def test_binding_refuses():
    z = torch.zeros(8, dtype=torch.float32)
    with pytest.raises(ValueError, match="device tensor"):
        pigan.TensorTable([z])
    with pytest.raises(ValueError, match="bits"):
        pigan.TensorTable([z], bits=8)
    with pytest.raises(ValueError, match="no tensors"):
        pigan.TensorTable([])
    with pytest.raises(ValueError, match="without params"):
        pigan.TensorTable([z], copies=[z])
