"""Shared pages, infinities and calls on other streams again on the bounds-checked build of the library (a child process: the library
is chosen at its first use): every access tested against its buffer, the report empty after every test."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(os.environ.get("MXQ_LIBRARY") == "checked", reason="already inside the checked run")
def test_nothing_outside_its_buffers():
    files = ["tests/test_gpu_kv_shared_pages.py", "tests/test_gpu_kv_nonfinite.py", "tests/test_gpu_streams.py"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"] + files, cwd=ROOT,
                       env=dict(os.environ, MXQ_LIBRARY="checked"), capture_output=True, text=True, timeout=1200)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:] + r.stderr[-2000:]
