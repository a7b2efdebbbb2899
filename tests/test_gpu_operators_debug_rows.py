"""Trees over rows of different lengths and long rows in parts under the debug build's index checks and guard regions."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_and_parts_under_the_debug_build():
    from paper_2608_08878_gb300 import build
    build.build_debug()
    files = ["debug_build_checks.py", "test_gpu_tree_rows.py", "test_gpu_every_tile.py"]
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-k", "not past_32_bits"]
                         + [os.path.join(ROOT, "tests", f) for f in files],
                         cwd=ROOT, env=dict(os.environ, DC_LIBRARY="debug"), capture_output=True, text=True, timeout=900)
    assert res.returncode == 0, res.stdout[-4000:] + res.stderr[-2000:]
    assert " passed" in res.stdout
