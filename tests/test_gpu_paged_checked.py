"""The paged cache's tests once more against the checked build of the library: every test asserts a clean status word where it
expects one, so a green run means that no kernel stepped outside its buffers on any of them."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_paged_cases_on_the_checked_build():
    from paper_2503_08879_b200 import build
    env = dict(os.environ, SAGEKV_LIB=build.build(checks=True))
    probe = subprocess.run([sys.executable, "-c", "from paper_2503_08879_b200 import binding as B; print(B.lib.sagekv_checked_build())"],
                           cwd=ROOT, env=env, capture_output=True, text=True)
    assert probe.returncode == 0 and probe.stdout.strip() == "1", probe.stderr[-2000:]
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "tests/test_gpu_paged_attn.py", "tests/test_gpu_paged_cache.py"],
                         cwd=ROOT, env=env, capture_output=True, text=True)
    assert res.returncode == 0, (res.stdout[-3000:], res.stderr[-2000:])
