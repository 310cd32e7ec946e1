"""Calls of the linear layer and layer norm at the edges of what they take, as
far as the host decides them (these run without a GPU)."""
import pytest

from paper_1910_13444_amd import pigan
from test_layers_abi import FAKE, K, M, N, _linear, _norm, needs_lib

NONE = (0, 0, 0)


@needs_lib
@pytest.mark.parametrize("dt", [0, 1, 2])
def test_no_rows_and_only_dx(dt):
    """An empty batch's dx has no elements, and an empty tensor's address is 0:
    there is nothing to do, and nothing wrong."""
    L = pigan.lib()
    a = _linear(dt=dt, m=0, x=(0, K, 0), g=(0, N, 0), dx=(0, K, 0), dw=0, db=0)
    assert L.pigan_linear_backward(a, None, 0, None) == pigan.OK
    a = _norm(dt=dt, m=0, x=(0, N, 0), dy=(0, N, 0), dx=(0, N, 0), mean=0, rstd=0, dgamma=0, dbeta=0)
    assert L.pigan_layer_norm_backward(a, None, 0, None) == pigan.OK


@needs_lib
@pytest.mark.parametrize("rows,ld,gs", [((1 << 24) + 1, 1 << 40, 16), ((1 << 24) + 1, 1 << 40, 1 << 46),
                                        ((1 << 31) - 1, 1 << 40, 1 << 46), ((1 << 23) + 1, 1 << 40, 1 << 40)])
def test_groups_whose_extent_passes_63_bits(rows, ld, gs):
    """(rows - 1) * ld wraps around: the group still does not fit its stride."""
    L = pigan.lib()
    far = (FAKE, ld, gs)
    assert L.pigan_layer_norm_forward(_norm(G=2, m=rows, x=far, y=far), None) == pigan.EINVAL
    assert L.pigan_linear_forward(_linear(G=2, m=rows, x=far, y=far), FAKE, 1 << 60, None) == pigan.EINVAL
    one = (FAKE, ld, 0)
    assert L.pigan_layer_norm_forward(_norm(m=1 << 6, x=one, y=one, eps=0.0), None) == pigan.EINVAL
    assert b"eps" in L.pigan_last_error()   # the strides themselves are in range


# Operands far apart from each other; a case moves one onto another.
AT = {n: 0x10000000 + 0x100000 * i for i, n in enumerate(
    ("x", "w", "y", "pre", "add", "g", "dx", "bias", "dw", "db", "dy", "gamma", "beta", "mean", "rstd", "dgamma", "dbeta"))}
WS = 0x40000000


def _refused(st):
    return st == pigan.EINVAL and b"overlaps" in pigan.lib().pigan_last_error()


def _forward_call(dt, at, ld={}):
    def mat(n, cols):
        return at[n], ld.get(n, cols), 0
    return pigan.lib().pigan_linear_forward(
        pigan.LINEAR_ARGS.pack(1, dt, 1, 0, M, N, N, *mat("x", N), *mat("w", N), *mat("y", N), *mat("pre", N),
                               *mat("add", N), 0, 0, 0, 0, 0, 0, at["bias"], 0, 0), WS, 1 << 20, None)


def _backward_call(dt, at, ld={}):
    def mat(n, cols):
        return at[n], ld.get(n, cols), 0
    return pigan.lib().pigan_linear_backward(
        pigan.LINEAR_ARGS.pack(1, dt, 1, 0, M, N, N, *mat("x", N), *mat("w", N), 0, 0, 0, *mat("pre", N), *mat("add", N),
                               *mat("g", N), *mat("dx", N), 0, at["dw"], at["db"]), WS, 1 << 20, None)


def _norm_call(dt, at, ld={}):
    def mat(n):
        return at[n], ld.get(n, N), 0
    return pigan.lib().pigan_layer_norm_forward(
        pigan.NORM_ARGS.pack(1, dt, M, N, 1e-5, 0, *mat("x"), *mat("y"), 0, 0, 0, 0, 0, 0, 0, 0, 0, at["gamma"], at["beta"],
                             at["mean"], at["rstd"], 0, 0), None)


def _norm_backward_call(dt, at, ld={}):
    def mat(n):
        return at[n], ld.get(n, N), 0
    return pigan.lib().pigan_layer_norm_backward(
        pigan.NORM_ARGS.pack(1, dt, M, N, 0.0, 0, *mat("x"), 0, 0, 0, *mat("dy"), *mat("add"), *mat("dx"), at["gamma"], 0,
                             at["mean"], at["rstd"], at["dgamma"], at["dbeta"]), WS, 1 << 20, None)


def _act_call(dt, at, ld={}):
    def mat(n):
        return at[n], ld.get(n, N), 0
    return pigan.lib().pigan_act_backward(
        pigan.ACT_ARGS.pack(1, dt, 1, 0, M, N, *mat("dy"), *mat("pre"), *mat("g")), None)


# (call, output, operand that it may not be)
APART = [(_forward_call, "y", i) for i in ("x", "w", "pre", "bias")] + \
        [(_forward_call, "pre", i) for i in ("x", "w", "add", "bias")] + \
        [(_backward_call, "dx", i) for i in ("g", "w", "x", "dw", "db")] + \
        [(_backward_call, o, i) for o in ("dw", "db") for i in ("g", "w", "x", "pre", "add")] + \
        [(_norm_call, "y", i) for i in ("gamma", "beta", "mean", "rstd")] + \
        [(_norm_call, o, "x") for o in ("mean", "rstd")] + \
        [(_norm_backward_call, "dx", i) for i in ("x", "gamma", "mean", "rstd", "dgamma", "dbeta")] + \
        [(_norm_backward_call, o, i) for o in ("dgamma", "dbeta") for i in ("dy", "x", "add", "gamma", "mean", "rstd")]
# (call, output, operand that it may only be as the same matrix)
SAME = [(_forward_call, "y", "add"), (_backward_call, "dx", "pre"), (_backward_call, "dx", "add"), (_norm_call, "y", "x"),
        (_norm_backward_call, "dx", "dy"), (_norm_backward_call, "dx", "add"), (_act_call, "g", "dy"), (_act_call, "g", "pre")]


@needs_lib
@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("call,output,operand", APART)
def test_outputs_on_other_operands_are_refused(call, output, operand, dt):
    assert _refused(call(dt, {**AT, output: AT[operand]}))
    assert _refused(call(dt, {**AT, output: AT[operand] + 4}))


@needs_lib
@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("call,output,operand", SAME)
def test_outputs_on_a_part_of_an_operand_are_refused(call, output, operand, dt):
    es = 4 if dt == 0 else 2
    for shift in (1, -1, N, -N * (M - 1), N * M - 1):
        assert _refused(call(dt, {**AT, output: AT[operand] + shift * es}))
    assert _refused(call(dt, {**AT, output: AT[operand]}, {output: N + 8}))
    assert _refused(call(dt, {**AT, output: AT[operand] - 8 * es}, {output: N + 8, operand: N + 8}))


@needs_lib
def test_the_workspace_on_an_operand_is_refused():
    big = dict(dt=0, m=30000, k=K, n=600, bias=0, w=(AT["w"], K, 0))
    need = pigan.lib().pigan_linear_forward_workspace(_linear(**big, x=(AT["x"], K, 0), y=(0x80000000, 600, 0)))
    assert need > 1
    for operand in ("x", "y"):
        d = dict(x=(0x50000000, K, 0), y=(0x80000000, 600, 0))
        d[operand] = (WS + 256, d[operand][1], 0)
        assert _refused(pigan.lib().pigan_linear_forward(_linear(**big, **d), WS, need, None))
