"""The tests of the norm, the rotated append, the logit rules, the adapters and the decoder that uses them again on the bounds-checked
build of the library (a child process: the library is chosen at its first use), the report empty after every test."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = ["tests/test_gpu_%s.py" % n for n in ("norm", "kv_rope", "logits", "lora", "decoder_step")]


def test_the_step_s_operators_touch_nothing_outside_their_buffers():
    if os.environ.get("MXQ_LIBRARY") == "checked":
        pytest.skip("already inside the checked run")
    env = dict(os.environ, MXQ_LIBRARY="checked")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"] + FILES,
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:] + r.stderr[-2000:]
