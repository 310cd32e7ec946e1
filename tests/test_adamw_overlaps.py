"""Operands of the optimizer's calls beside its tensors (count, factor, flag, workspace,
results) that share memory with them: refused, element by element (no GPU; the addresses
are never dereferenced)."""
import ctypes as C
import os
import random

import pytest

from paper_1910_13444_amd import pigan
from test_adamw_abi import M, _adamw, _table, _tensor, needs_lib

DEVICE = 1 << 40   # of the table's copy


def _last():
    return pigan.lib().pigan_last_error().decode()


def _layout(seed, bits):
    """Tensors in random places of one stretch of memory, with gaps or without: the table and
    the bytes that are its outputs and its gradients."""
    rng = random.Random(seed)
    at, outs, grads, tensors = M, [], [], []

    def place(size, to):
        nonlocal at
        at += rng.choice((0, 0, 4, 12))
        to.append((at, at + size))
        at += -(-size // 4) * 4
        return to[-1][0]

    for _ in range(12):
        n, g_dt, copy = rng.choice((1, 2, 3, 10, 257)), rng.randrange(3), rng.randrange(3) if bits else 0
        p = place(4 * n, outs) if bits else 0
        g = place((4, 2, 2)[g_dt] * n, grads)
        c = place(2 * n, outs) if copy else 0
        tensors.append(_tensor(p=p, g=g, copy=c, n=n, g_dt=g_dt, copy_dt=copy))
    tensors.append(_tensor(p=0, g=0, n=0))
    states = [1 << 30, 2 << 30, 3 << 30, (3 << 30) + 4096]
    st, table, size, count = _table(*tensors, bits=bits, **dict(zip(("m", "v", "ms", "vs"), states)))
    assert st == pigan.OK, _last()
    if bits:
        outs += [(s, s + n) for s, n in zip(states, (count * bits // 8,) * 2 + ((count // 64,) * 2 if bits == 8 else ()))]
    return table, size, outs, grads, at


def _inside(a, size, spans):
    return any(a < to and a + size > start for start, to in spans)


def _places(outs, grads, end):
    near = [p + d for s in outs + grads for p in s for d in (-8, -4, 0, 4)]
    return sorted({a // 4 * 4 for a in [*range(M - 8, end + 8, 4), *near] if a > 0})


@needs_lib
@pytest.mark.parametrize("bits", [8, 32])
def test_words_of_a_step(bits):
    """Every place of a word.  The workspace lies over the table, so nothing is launched: that is
    told where the word itself is apart."""
    L = pigan.lib()
    for seed in range(4):
        table, size, outs, grads, end = _layout(seed, bits)
        at = C.addressof(table)
        for a in _places(outs, grads, end):
            for name, with_grads in (("step", True), ("coef", False), ("skip", False)):
                words = {"step": 8 << 30, name: a}
                st = L.pigan_adamw_update(_adamw(at, device=DEVICE, t=0, **words), DEVICE, 256, None)
                assert st == pigan.EINVAL
                want = f"{name} overlaps a parameter, copy or state" if _inside(a, 4, outs) else \
                    f"{name} overlaps a gradient" if with_grads and _inside(a, 4, grads) else "the workspace overlaps the table"
                assert _last() == want, (hex(a), name)


@needs_lib
def test_workspaces_and_results():
    L = pigan.lib()
    table, size, outs, grads, end = _layout(9, 8)
    at, step = C.addressof(table), 8 << 30
    last = DEVICE + size - 1

    def update(ws, **kw):
        st = L.pigan_adamw_update(_adamw(at, device=DEVICE, t=0, **{"step": step, **kw}), ws, 256, None)
        assert st == pigan.EINVAL
        return _last()

    for a in outs:
        assert update((a[1] - 1) // 256 * 256) == "the workspace overlaps a parameter, copy or state"
    lone = [g for g in grads if not any(_inside(b // 256 * 256, 256, outs) for b in (g[0], g[1] - 1))]
    for g in lone:
        assert update(g[0] // 256 * 256) == "the workspace overlaps a gradient"
    assert update(last // 256 * 256) == "the workspace overlaps the table"
    assert update(16 << 30, step=last // 4 * 4) == "step overlaps the table"
    for word in ("step", "coef", "skip"):   # of the workspace's 256 bytes
        for off in (0, 4, 252):
            assert "overlaps" in update(16 << 30, **{word: (16 << 30) + off})
    assert "overlaps" in update(16 << 30, coef=step) and "overlaps" in update(16 << 30, skip=step)

    need = L.pigan_grad_norm_workspace(at)

    def norm(out, ws=16 << 30):
        st = L.pigan_grad_norm(at, DEVICE, 1.0, 1.0, *out, ws, need, None)
        assert st == pigan.EINVAL
        return _last()

    for k, name in enumerate(("norm", "coef", "nonfinite")):
        for a in sorted({x // 4 * 4 for g in grads for x in (g[0], g[1] - 1)}):
            assert norm([a if i == k else 0 for i in range(3)]) == f"{name} overlaps a gradient"
        assert norm([last // 4 * 4 if i == k else 0 for i in range(3)]) == f"{name} overlaps the table"
    assert norm((step, 0, 0), ws=DEVICE) == "the workspace overlaps the table"
    st, long, size, _ = _table(_tensor(g=2 * M, n=1000))
    assert st == pigan.OK
    for ws in (2 * M, 2 * M + 256, 2 * M + 3840):   # of its 4000 bytes
        assert L.pigan_grad_norm(long, DEVICE, 1.0, 1.0, step, 0, 0, ws, 1 << 20, None) == pigan.EINVAL
        assert _last() == "the workspace overlaps a gradient"


@needs_lib
def test_tables_of_gradients_alone():
    L = pigan.lib()
    for seed in range(3):
        table, size, outs, grads, end = _layout(20 + seed, 0)
        need = L.pigan_grad_norm_workspace(C.addressof(table))
        for a in _places([], grads, end):
            assert L.pigan_grad_norm(C.addressof(table), DEVICE, 1.0, 1.0, a, 0, 0, DEVICE, need, None) == pigan.EINVAL
            assert _last() == ("norm overlaps a gradient" if _inside(a, 4, grads) else "the workspace overlaps the table")
