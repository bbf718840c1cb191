"""The cache's tests again on the bounds-checked build of the library (a child process: the library is chosen at its first use):
every plain global access and every bulk copy's source tested against its buffer, the report empty after every test."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_cache_touches_nothing_outside_its_buffers():
    if os.environ.get("MXQ_LIBRARY") == "checked":
        pytest.skip("already inside the checked run")
    env = dict(os.environ, MXQ_LIBRARY="checked")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_kv.py"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0 and " passed" in r.stdout, tail
