"""The random cases of the paged calls, long runs of absent pages and the largest sizes against the checked build of the library, whose
paged kernels compare table entries, tiles, rows, scratch parts and tickets with their extents."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_random_paged_cases_on_the_checked_build():
    from paper_2503_08879_b200 import build
    env = dict(os.environ, SAGEKV_LIB=build.build(checks=True))
    probe = subprocess.run([sys.executable, "-c", "from paper_2503_08879_b200 import binding as B; print(B.lib.sagekv_checked_build())"],
                           cwd=ROOT, env=env, capture_output=True, text=True)
    assert probe.returncode == 0 and probe.stdout.strip() == "1", probe.stderr[-2000:]
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "tests/test_gpu_paged_fuzz.py", "tests/test_gpu_paged_absent.py",
                          "tests/test_gpu_paged_limits.py", "tests/test_gpu_paged_edges.py"], cwd=ROOT, env=env, capture_output=True, text=True)
    assert res.returncode == 0, (res.stdout[-3000:], res.stderr[-2000:])
