"""The bounded waits of mxq_kv_attention: a tile that never arrives ends the call with a status bit and NaN, not with a hang, and
the next call is right again.  The hook that leaves a request out exists in the bounds-checked build only, so a child process runs it
(what is left out is the request: the kernel waits for a barrier that nothing completes, up to its limit)."""
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
d, hq, m, tile = (int(x) for x in sys.argv[1:])
lens, h = [40000, 7000, 100], 2
cache = mxq.KVCache.new(1, sum(-(-n // 64) for n in lens), h, d, 64)
tables, t_lens = cache.new_sequences(3, max(lens))
mxq.mxq_kv_resize(cache, tables, t_lens, torch.tensor(lens, dtype=torch.int32, device="cuda"))
g = torch.Generator(device="cuda").manual_seed(1)
for b, n in enumerate(lens):
    k, v = (torch.randn(1, n, h, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    mxq.mxq_kv_append(cache, 0, k, v, tables[b:b + 1], t_lens[b:b + 1])
q = torch.randn(3, m, hq, d, generator=g, device="cuda").bfloat16()
ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(3, m, hq, h, d))
run = lambda: mxq.mxq_kv_attention(q, cache, 0, tables, t_lens, workspace=ws, with_lse=True)
want, wl = run()
torch.cuda.synchronize()
assert mxq.mxq_linear_device_status() == 0
mxq.mxq_debug_kv_lost_tile(tile)
t = time.time()
out, lse = run()
torch.cuda.synchronize()
took = time.time() - t
assert 0.9 < took < 8, took
assert mxq.mxq_linear_device_status() == 1 << 29
assert bool(torch.isnan(out[0, :, :hq // 2]).all()) and bool(torch.isnan(lse[0, :, :hq // 2]).all())      # the tile's rows
nan = torch.isnan(lse)
assert torch.equal(torch.isnan(out).any(-1), nan) and not bool(nan.all())
assert torch.equal(out[~nan], want[~nan]) and torch.equal(lse[~nan], wl[~nan])      # and nothing else is touched
ws.zero_()
out, lse = run()
assert torch.equal(out, want) and torch.equal(lse, wl) and mxq.mxq_linear_device_status() == 0
assert mxq.mxq_debug_bounds_report() == {"checked": True, "refused": 0}
print("lost tile ok, %.1f s" % took)
"""


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,m,tile", [(64, 2, 1, 0), (128, 8, 1, 131), (64, 8, 4, 1200), (128, 32, 2, 77)])
def test_a_tile_that_never_arrives(d, hq, m, tile):
    env = dict(os.environ, MXQ_LIBRARY="checked")
    r = subprocess.run([sys.executable, "-c", CHILD, str(d), str(hq), str(m), str(tile)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "lost tile ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


@pytest.mark.skipif(os.environ.get("MXQ_LIBRARY") == "checked", reason="this process runs the checked build itself")
def test_the_ordinary_build_has_no_such_hook():
    with pytest.raises(mxq.MxqError):
        mxq.mxq_debug_kv_lost_tile(3)
