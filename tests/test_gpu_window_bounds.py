"""The bounds-checking build of the library on windows, shared prefixes and slot maps: the tests that reach their kernels at
their edges run again in a child process on librap_b200_dbg.so, where hand-computed indexes are checked on the device (a
failed check is recorded and the access skipped).  All of them assert a clean status word."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

EDGE_CASES = "lengths_at_every_border or head_shapes or batches or ragged or long_blocks or many_rows or shared_prefixes or without_a_group or conversation or one_prompt"


def test_edge_cases_pass_with_every_index_checked():
    from paper_2602_02599_b200 import build
    env = dict(os.environ, RAP_LIBRARY=build.build_debug())
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_gpu_window.py"), "-m", "gpu", "-x", "-q", "-k", EDGE_CASES],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout


def test_long_sequences_pass_with_every_index_checked():
    from paper_2602_02599_b200 import build
    env = dict(os.environ, RAP_LIBRARY=build.build_debug())
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_gpu_window.py"), "-m", "gpu", "-x", "-q", "-k", "long_units or long_sums or last_positions"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
