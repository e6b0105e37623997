"""The speculative-decoding cases against the bounds-checking build of the library: no kernel computes a
global offset outside what the call's shapes imply (each case asserts its status word)."""
import os
import subprocess
import sys

import pytest

from paper_2409_04992_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CASES = ["tests/test_gpu_tree_attention.py", "tests/test_gpu_kv_pages.py", "tests/test_gpu_verify.py",
         "tests/test_gpu_speculative_step.py"]


def test_no_bounds_flag_in_the_checked_build():
    library = build.build(checked=True)
    done = subprocess.run([sys.executable, "-m", "pytest", *CASES, "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider"],
                          cwd=ROOT, env=dict(os.environ, INSTINFER_LIBRARY=str(library)), capture_output=True, text=True, timeout=1800)
    assert done.returncode == 0, done.stdout[-4000:] + done.stderr[-2000:]
    assert " passed" in done.stdout
