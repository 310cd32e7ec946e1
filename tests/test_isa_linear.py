"""Properties of the compiled linear layer and layer norm kernels that parity
tests cannot show, on the gfx950 assembly, on the CPU.

The pipelined products send their operands straight from memory to LDS by loads
written as inline assembly, of which the compiler knows nothing: no wait is
placed for them but the source's own.  A forward pass over each kernel's
control-flow graph bounds the LDS loads that may be in flight (loads return in
order, so after s_waitcnt vmcnt(N) at most the N newest are) and shows that none
is at a barrier of the loop or at the kernel's end, and at the one barrier
before the loop at most the second stage's half of them.  M0, each load's LDS
address, is set by the load's own sequence alone."""
import os
import re
import subprocess

import pytest

from paper_1910_13444_amd import build
from test_isa_raw_lds_reads import _blocks

# rows of 8192 to 16384 16-bit columns: a thread's sixteen columns, their sums and the
# next row's pieces beside each other are more than 1024 threads' 128 registers
KNOWN = {r"k_norm_bwdIDF16[b_]Li1024ELi2ELb1ELb1ELb1E": 24, r"k_norm_bwdIDF16[b_]Li1024ELi2ELb1ELb1ELb0E": 57}

_VMCNT = re.compile(r"vmcnt\((\d+)\)")


def _assembly(tmp_path_factory, source):
    if not os.path.exists(build.hipcc()):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("isa") / (source + ".s"))
    r = subprocess.run([build.hipcc(), *build.common_flags(), "--cuda-device-only", "-S",
                        os.path.join(build.CSRC, source), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    with open(out) as f:
        return f.read()


@pytest.fixture(scope="module")
def dw(tmp_path_factory):
    return _assembly(tmp_path_factory, "linear_dw.hip")


@pytest.fixture(scope="module")
def norm(tmp_path_factory):
    return _assembly(tmp_path_factory, "norm.hip")


def _bodies(asm):
    return {m.group(1): asm[m.end():asm.find(".Lfunc_end", m.end())] for m in re.finditer(r"^(_Z\w+):", asm, re.M)}


def _is_lds_load(line):
    return line.startswith("buffer_load") and re.search(r"\blds\b", line) is not None


def _run(blocks, states, i, barriers=None):
    """LDS loads in flight at block i's end; `barriers` gathers (count, block)."""
    n = states[i]
    for line in blocks[i][1]:
        if _is_lds_load(line):
            n = min(n + 1, 64)
        elif line.startswith("s_waitcnt"):
            m = _VMCNT.search(line)
            n = min(n, int(m.group(1))) if m else n
        elif line.startswith("s_barrier") and barriers is not None:
            barriers.append((n, i))
        elif line.startswith("s_endpgm"):
            assert n == 0, "loads into LDS in flight at the kernel's end"
    return n


def _successors(blocks):
    label = {b[0]: i for i, b in enumerate(blocks) if b[0] is not None}
    return [[label[s] for s in b[2]] + ([i + 1] if b[3] and i + 1 < len(blocks) else []) for i, b in enumerate(blocks)]


def _check_pipeline(body):
    blocks = _blocks(body.splitlines())
    succ = _successors(blocks)
    states, todo = {0: 0}, [0]
    while todo:
        i = todo.pop()
        n = _run(blocks, states, i)
        for j in succ[i]:
            if states.get(j, -1) < n:
                states[j] = n
                todo.append(j)
    reach = {i: set() for i in states}
    for i in reach:
        stack = list(succ[i])
        while stack:
            j = stack.pop()
            if j not in reach[i]:
                reach[i].add(j)
                stack.extend(succ[j])
    barriers = []
    for i in states:
        _run(blocks, states, i, barriers)
    loads_before = sum(_is_lds_load(line) for i in states if i not in reach[i] for line in blocks[i][1])
    loop = [n for n, i in barriers if i in reach[i]]
    outside = sorted(n for n, i in barriers if i not in reach[i])
    assert len(loop) >= 2 and max(loop) == 0
    assert outside[-1] <= loads_before // 2 and max(outside[:-1], default=0) == 0


def _piped(asm):
    found = {n: b for n, b in _bodies(asm).items() if "k_mm_piped" in n}
    assert len(found) == 8 and all(any(_is_lds_load(x.strip()) for x in b.splitlines()) for b in found.values())
    return found


def test_no_load_into_lds_is_in_flight_at_a_barrier(dw):
    for name, body in _piped(dw).items():
        try:
            _check_pipeline(body)
        except AssertionError as e:
            raise AssertionError(f"{name}: {e}") from e


def test_m0_belongs_to_the_loads(dw):
    for name, body in _piped(dw).items():
        lines = [x for x in (raw.split(";")[0].strip() for raw in body.splitlines()) if x and not x.startswith(".")]
        for k, line in enumerate(lines):
            if _is_lds_load(line):
                assert lines[k - 1] == "s_nop 0" and lines[k - 2].startswith("s_add_u32 m0,"), f"{name}: {lines[k - 2:k + 1]}"
            elif re.match(r"\S+\s+m0\b", line):
                assert _is_lds_load(lines[k + 2]), f"{name}: {line}"


def test_the_pass_finds_a_missing_wait(dw):
    """The oracle's own check: without the loop's waits the property does not hold."""
    name, body = next(iter(_piped(dw).items()))
    with pytest.raises(AssertionError):
        _check_pipeline(re.sub(r"s_waitcnt vmcnt\(0\)", "s_waitcnt vmcnt(8)", body))


@pytest.mark.parametrize("source", ["dw", "norm"])
def test_no_spills(source, request):
    meta = request.getfixturevalue(source).rsplit("amdhsa.kernels:", 1)[1]
    kernels = re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)", meta, re.S)
    assert len(kernels) >= 13
    for name, scratch, spills in kernels:
        allowed = max([n for part, n in KNOWN.items() if re.search(part, name)], default=0)
        assert int(spills) <= allowed and (allowed or int(scratch) == 0), f"{name} spills {spills}, {scratch} bytes of scratch"
