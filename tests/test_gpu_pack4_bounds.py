"""The 4-bit cache and beam search against the bounds-checking build."""
import os
import subprocess
import sys

import pytest

from paper_2410_18517_b200 import build as kbuild

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pack4_and_beam_under_the_bounds_checking_build():
    lib = kbuild.build(bounds=True)
    env = dict(os.environ, KVS_LIBRARY=lib, PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests")]))
    out = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "pack4_bounds_cases.py")], capture_output=True, text=True,
                         timeout=1500, env=env)
    assert out.returncode == 0, out.stdout[-3000:] + out.stderr[-3000:]
    assert "ALL 4-BIT AND BEAM BOUNDS CASES PASSED" in out.stdout
