"""The two forms of a shared beginning (few rows, tiles) on the small calls of the other tests, which by the rules attend without sharing: the same tests in child processes."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("setting", ["1", "2"])
def test_shared_beginnings_by(_built_library, setting):
    env = dict(os.environ, QLINEAR_PAGED_SHARED=setting)
    cmd = [sys.executable, "-m", "pytest", os.path.join("tests", "test_contexts_gpu.py"), "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", "-k", "(shared or prefix or share or nothing_seen or streams or millions) and not prompts_behind"]
    r = subprocess.run(cmd, env=env, cwd=ROOT, timeout=600, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-4000:]
