"""The bounded waits of the adapters' tcgen05 kernel: a stage that never arrives ends the call with a status bit and NaN, not with a hang, what
is still in flight lands before the CTA ends, and the next call is right again.  The hook that leaves a request out exists in the
bounds-checked build only, so a child process runs it (what is left out is the request: the kernel waits for a barrier that nothing
completes, up to its limit)."""
import os
import subprocess
import sys

import pytest

import paper_2503_13565_b200 as mxq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys, time
import torch
import paper_2503_13565_b200 as mxq
rank, stage = (int(x) for x in sys.argv[1:])
m, n, k, count = 4095, 40, 4096, 6
g = torch.Generator(device="cuda").manual_seed(1)
rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
x, a, b, base = rn(m, k).bfloat16(), (rn(count, rank, k) / 64).bfloat16(), rn(count, n, rank).bfloat16(), rn(m, n)
ids = torch.randint(-1, count, (m,), generator=g, device="cuda").int()
ids[:128] = torch.arange(128, device="cuda").int() % 7 - 1          # the first window has all adapters, and rows without one
run = lambda: mxq.mxq_lora(x, a, b, ids, base=base)
want = run()
torch.cuda.synchronize()
assert mxq.mxq_linear_device_status() == 0 and bool(want.isfinite().all())
mxq.mxq_debug_lora_lost_stage(stage)
t = time.time()
out = run()
torch.cuda.synchronize()
took = time.time() - t
assert 0.9 < took < 8, took
assert mxq.mxq_linear_device_status() == 1 << 30
nan = torch.isnan(out).any(-1)
assert torch.equal(nan, torch.isnan(out).all(-1)) and not bool(nan[128:].any())
lost = sorted(set(ids[:128][nan[:128]].tolist()))                   # the first CTA has every fourth adapter of the window
assert lost == [0, 4] and torch.equal(nan[:128], (ids[:128] == 0) | (ids[:128] == 4)), lost
assert torch.equal(out[~nan], want[~nan])
assert torch.equal(run(), want) and mxq.mxq_linear_device_status() == 0
assert mxq.mxq_debug_bounds_report() == {"checked": True, "refused": 0}
print("lost stage ok, %.1f s" % took)
"""


@pytest.mark.gpu
@pytest.mark.parametrize("rank,stage", [(64, 0), (64, 2), (64, 9), (16, 5), (128, 31), (64, 63)])
def test_a_stage_that_never_arrives(rank, stage):
    env = dict(os.environ, MXQ_LIBRARY="checked")
    r = subprocess.run([sys.executable, "-c", CHILD, str(rank), str(stage)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "lost stage ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


@pytest.mark.skipif(os.environ.get("MXQ_LIBRARY") == "checked", reason="this process runs the checked build itself")
def test_the_ordinary_build_has_no_such_hook():
    with pytest.raises(mxq.MxqError):
        mxq.mxq_debug_lora_lost_stage(3)
