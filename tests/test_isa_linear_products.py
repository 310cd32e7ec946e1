"""The forward pass and dx of the linear layer, as compiled: the properties of
test_isa_linear.py's loads straight to LDS, for every kernel that makes them (by
themselves, and both reverse products in one launch), on the CPU.

A pass over each kernel's control flow bounds the LDS loads in flight.  Each
product of a kernel has one barrier before its loop, behind which the first
stage is read while at most the second one's loads are in flight; at the
barriers of its loop, at those behind it and at the kernel's end none may be.
Branches beyond a branch instruction's reach go through a register: their
targets are read from the address arithmetic before them."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_1910_13444_amd import build
from test_isa_linear import _bodies, _is_lds_load, _run, _successors
from test_isa_raw_lds_reads import _blocks

SOURCES = ("linear_fwd.hip", "linear_dx.hip")
_FAR = re.compile(r"s_add_u32 s\d+, s\d+, \((\.LBB\d+_\d+)-\.Lpost_getpc\d+\)&4294967295")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: assembly} of both files"""
    if not os.path.exists(build.hipcc()):
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("isa")

    def assembly(source):
        f = str(out / (source + ".s"))
        r = subprocess.run([build.hipcc(), *build.common_flags(), "--cuda-device-only", "-S",
                            os.path.join(build.CSRC, source), "-o", f], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        with open(f) as fh:
            return fh.read()

    with cf.ThreadPoolExecutor(2) as ex:
        texts = list(ex.map(assembly, SOURCES))
    bodies, meta = {}, []
    for t in texts:
        bodies |= _bodies(t)
        meta += re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)",
                           t.rsplit("amdhsa.kernels:", 1)[1], re.S)
    return bodies, meta


def _near(body):
    """The instructions, each far branch as a branch to its target."""
    out = []
    for line in body.splitlines():
        m = _FAR.search(line)
        if m:
            out.append(f"s_branch {m.group(1)}")
        elif not line.strip().startswith(("s_getpc_b64", "s_setpc_b64")) and "-.Lpost_getpc" not in line:
            out.append(line)
    return out


def _loops(succ):
    """blocks that lie on a cycle (Tarjan's components, without recursion)"""
    index, low, on, stack, loop, n = {}, {}, set(), [], set(), 0
    for root in range(len(succ)):
        if root in index:
            continue
        work = [(root, 0)]
        while work:
            v, k = work.pop()
            if k == 0:
                index[v] = low[v] = n
                n += 1
                stack.append(v)
                on.add(v)
            if k < len(succ[v]):
                work.append((v, k + 1))
                w = succ[v][k]
                if w not in index:
                    work.append((w, 0))
                elif w in on:
                    low[v] = min(low[v], index[w])
            else:
                if low[v] == index[v]:
                    part = []
                    while True:
                        w = stack.pop()
                        on.discard(w)
                        part.append(w)
                        if w == v:
                            break
                    if len(part) > 1 or v in succ[v]:
                        loop.update(part)
                if work:
                    u = work[-1][0]
                    low[u] = min(low[u], low[v])
    return loop


def _check(body, products):
    blocks = _blocks(_near(body))
    succ = _successors(blocks)
    states, todo = {0: 0}, [0]
    while todo:
        i = todo.pop()
        n = _run(blocks, states, i)
        for j in succ[i]:
            if states.get(j, -1) < n:
                states[j] = n
                todo.append(j)
    loop, barriers = _loops(succ), []
    for i in states:
        _run(blocks, states, i, barriers)   # and none in flight at an end of the kernel
    assert any(i in loop for _, i in barriers)
    assert all(n == 0 for n, i in barriers if i in loop), "a load into LDS in flight at a barrier of a loop"
    loads = sum(_is_lds_load(line) for i in states if i not in loop for line in blocks[i][1])
    first = [n for n, i in barriers if i not in loop and n]
    # two stages are requested before each product's loop
    assert len(first) == products and all(n == loads // (2 * products) for n in first), (first, loads)


def _loading(kernels):
    return {n: b for n, b in kernels[0].items() if any(_is_lds_load(x.strip()) for x in b.splitlines())}


def test_every_kernel_that_loads_to_lds(kernels):
    """Operands of two types, results of three, tiles of four kinds, whole and ragged
    columns, and both products in one launch (two tiles)."""
    names = list(_loading(kernels))
    assert sum("k_mm_piped" in n for n in names) == 2 * 3 * 4 * 2 and sum("k_mm_both" in n for n in names) == 3 * 2 * 2
    assert len(names) == 60


def test_no_load_into_lds_is_in_flight_at_a_barrier(kernels):
    for name, body in _loading(kernels).items():
        try:
            _check(body, 2 if "k_mm_both" in name else 1)
        except AssertionError as e:
            raise AssertionError(f"{name}: {e}") from e


def test_m0_belongs_to_the_loads(kernels):
    for name, body in _loading(kernels).items():
        lines = [x for x in (raw.split(";")[0].strip() for raw in body.splitlines()) if x and not x.startswith(".")]
        for k, line in enumerate(lines):
            if _is_lds_load(line):
                assert lines[k - 1] == "s_nop 0" and lines[k - 2].startswith("s_add_u32 m0,"), f"{name}: {lines[k - 2:k + 1]}"
            elif re.match(r"\S+\s+m0\b", line):
                assert _is_lds_load(lines[k + 2]), f"{name}: {line}"


def test_the_pass_finds_a_missing_wait(kernels):
    """The oracle's own check, on both kinds of kernels."""
    for kind, products in (("k_mm_piped", 1), ("k_mm_both", 2)):
        name, body = next((n, b) for n, b in _loading(kernels).items() if kind in n)
        with pytest.raises(AssertionError):
            _check(re.sub(r"s_waitcnt vmcnt\(0\)", "s_waitcnt vmcnt(8)", body), products)


def test_no_spills(kernels):
    assert len(kernels[1]) >= 60
    for name, scratch, spills in kernels[1]:
        assert int(spills) == 0 and int(scratch) == 0, f"{name} spills {spills}, {scratch} bytes of scratch"
