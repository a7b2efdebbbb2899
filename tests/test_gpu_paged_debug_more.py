"""The paged cache's tests of values, order and prefixes under the debug build: every index that its kernels compute for memory that
others own is checked there."""

import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_more_of_the_paged_cache_under_the_debug_build():
    from paper_2608_08878_gb300 import build
    build.build_debug()
    files = ("debug_build_checks.py", "test_gpu_large_scores.py", "test_gpu_paged_order.py", "test_gpu_paged_prefix_values.py")
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu"] + [os.path.join(ROOT, "tests", f) for f in files],
                         cwd=ROOT, env=dict(os.environ, DC_LIBRARY="debug"), capture_output=True, text=True, timeout=1500)
    assert res.returncode == 0, res.stdout[-4000:] + res.stderr[-2000:]
    assert " passed" in res.stdout


@pytest.mark.parametrize("name,least", [("dc_paged_append.cu", 2), ("dc_paged_attend.cu", 7), ("dc_paged_select.cu", 6)])
def test_the_kernels_have_checks(name, least):
    """Each site by a number of its own, so that a report names its place."""
    with open(os.path.join(ROOT, "paper_2608_08878_gb300", "csrc", name)) as f:
        sites = re.findall(r"DC_INB\(.*?, (\d+)\)", f.read())
    assert len(sites) >= least and len(set(sites)) == len(sites)
