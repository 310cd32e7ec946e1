"""The argument checks of group norm, the gradients' norm and AdamW once more against the
library's host-sanitized copy (as test_abi_sanitized.py).  CPU only."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = ["test_group_norm_abi.py", "test_group_norm_strides.py", "test_adamw_abi.py", "test_adamw_overlaps.py"]


def test_operators_checks_under_host_sanitizers(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_1910_13444_amd import build_sanitized as bs
    try:
        rt = bs.asan_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    lib = bs.build_sanitized(jobs=4)
    log = tmp_path / "san"
    env = dict(os.environ, LD_PRELOAD=rt, PIGAN_LIBRARY=lib,
               ASAN_OPTIONS=f"detect_leaks=0:halt_on_error=1:log_path={log}",
               UBSAN_OPTIONS=f"halt_on_error=1:print_stacktrace=1:log_path={log}")
    # test_overlaps_are_told_exactly builds a program of its own
    r = subprocess.run([sys.executable, "-m", "pytest", *(os.path.join(ROOT, "tests", t) for t in TESTS), "-q",
                        "-p", "no:cacheprovider", "-k", "not told_exactly"], env=env, cwd=ROOT, capture_output=True, text=True,
                       timeout=600)
    reports = "".join(p.read_text() for p in tmp_path.glob("san*"))
    assert r.returncode == 0 and not reports, (r.stdout[-3000:] + r.stderr[-3000:] + reports[:4000])
    assert " passed" in r.stdout
