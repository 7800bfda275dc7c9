"""The cases at the ends of what 4-bit caches and beam search take, against the bounds-checking build."""
import os
import subprocess
import sys

import pytest

from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu
TESTS = os.path.dirname(os.path.abspath(__file__))


def test_edges_under_the_bounds_checking_build():
    env = dict(os.environ, KVS_LIBRARY=kbuild.build(bounds=True))
    out = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider"] +
                         [os.path.join(TESTS, f) for f in ("test_gpu_pack4_edges.py", "test_gpu_beam_edges.py")],
                         capture_output=True, text=True, timeout=900, env=env)
    assert out.returncode == 0 and " passed" in out.stdout and "skipped" not in out.stdout, out.stdout[-3000:] + out.stderr[-1000:]
