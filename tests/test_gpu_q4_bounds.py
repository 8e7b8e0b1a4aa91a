"""The bounds-checking build of the library on the 4-bit cache: the tests that reach its kernels at their edges run again in a
child process on librap_b200_dbg.so, where every hand-computed index is checked on the device (a failed check is recorded and
the access skipped).  All of them assert a clean status word.  The other file of this kind covers the other caches."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

EDGE_CASES = ("lengths_at_every_border or head_shapes or odd_widths or longer_sequences or twenty_thousand or many_sequences or "
              "read_cache_up_to or append or decode_step or prompt_chunk or (rows_both_ways and 1003)")


def test_edge_cases_pass_with_every_index_checked():
    from paper_2602_02599_b200 import build
    env = dict(os.environ, RAP_LIBRARY=build.build_debug())
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_gpu_q4.py"), "-m", "gpu", "-x", "-q", "-k", EDGE_CASES],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
