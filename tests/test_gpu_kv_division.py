"""mxq_kv_attention where its work is divided into items of every size: half a CTA's share, big and small ones, hundreds of parts
per segment, more than 32 tiles per warp.  Ragged lengths, sequences without rows, missing pages, a running maximum that keeps
rising and values whose size drifts along the sequence; against the 64-bit form of tests/kv_exact.py."""
import math
import os
import random
import subprocess
import sys

import pytest
import torch

import kv_exact
import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHECKED = os.environ.get("MXQ_LIBRARY") == "checked"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def filled(lens, h, d, page, seed, missing=()):
    """A cache with sequences of these lengths on scattered pages: keys drift towards a direction along the sequence (the maximum
    keeps rising), values swell and shrink by 2^12 and vary from token to token.  missing: (sequence, page place) without a page."""
    need = [-(-n // page) for n in lens]
    cache = mxq.KVCache.new(1, sum(need) + 3, h, d, page)
    tables, t_lens = cache.new_sequences(len(lens), max(max(lens), 1))
    order = torch.randperm(sum(need) + 3, generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()
    at = 0
    for b, m in enumerate(need):
        tables[b, :m] = order[at:at + m]
        at += m
    t_lens.copy_(i32(lens))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mean = torch.randn(h, d, generator=gen, device="cuda")
    step = 65536
    for b, n in enumerate(lens):
        for a in range(0, n, step):
            m = min(step, n - a)
            pos = torch.arange(a, a + m, device="cuda", dtype=torch.float32)
            shape = (1, m, h, d)
            k = torch.randn(shape, generator=gen, device="cuda") + (0.8 * pos / n)[None, :, None, None] * mean
            size = torch.exp2(6 * torch.sin(pos * (14.0 / n)) + torch.randn(m, generator=gen, device="cuda"))
            v = torch.randn(shape, generator=gen, device="cuda") * size[None, :, None, None]
            mxq.mxq_kv_append(cache, 0, k.bfloat16(), v.bfloat16(), tables[b:b + 1], i32([a + m]))
    for b, w in missing:
        tables[b, w] = -1
    return cache, tables, t_lens, mean


def share_of(lens, rows, h, group, d):
    """(column blocks, tiles per CTA) as the kernel divides them"""
    nt = 1 if max(rows) * group <= 8 else 2
    per_sm = {(128, 1): 3, (64, 1): 4, (128, 2): 2, (64, 2): 3}[d, nt]
    grid = per_sm * torch.cuda.get_device_properties(0).multi_processor_count
    work = sum((-(-n // 32) if r else 1) * max(1, -(-r * group // (8 * nt))) * h for n, r in zip(lens, rows))
    return nt, work // grid


def run(lens, rows, h, hq, d, page, seed, missing=(), tree=False):
    m, group = max(rows), hq // h
    cache, tables, t_lens, mean = filled(lens, h, d, page, seed, missing)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (torch.randn(len(lens), m, hq, d, generator=gen, device="cuda") * 1.5 + 0.6 * mean.repeat_interleave(group, 0)).bfloat16()
    trees = None
    if tree:
        rng = random.Random(seed)
        trees = [[1 << i | rng.getrandbits(i) if i else 1 for i in range(m)] for _ in lens]
    ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(len(lens), m, hq, h, d))
    args = dict(rows=i32(rows), workspace=ws, with_lse=True, tree=torch.tensor(trees, dtype=torch.int64, device="cuda") if tree else None)
    out, lse = mxq.mxq_kv_attention(q, cache, 0, tables, t_lens, **args)
    again, lse2 = mxq.mxq_kv_attention(q, cache, 0, tables, t_lens, **args)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))
    assert int(ws[:4096].sum()) == 0 and mxq.mxq_linear_device_status() == 0
    exact = kv_exact.attention(cache, 0, q, tables, lens, rows, d ** -0.5, trees)
    # FP32 additions behind lse in a chain: four weights of every tile of a lane (an item has at most 256 tiles at these sizes, 64 per
    # warp), the lanes, the warps, a quarter of at most 512 parts
    kv_exact.check(out, lse, exact, d, adds=1024)


@pytest.mark.parametrize("d,h,hq,rows,lens", [
    (128, 8, 8, [1, 1, 1, 0, 1], [30011, 2048, 17, 9000, 12345]),              # one column block
    (128, 8, 32, [4, 2, 4, 0, 3], [20011, 5000, 4, 9000, 12345]),              # two, ragged rows
    (64, 16, 32, [1, 1, 0, 1], [20011, 2048, 5000, 10001]),
    (64, 8, 64, [2, 5, 0, 16], [10011, 7000, 900, 5001])])
def test_items_of_half_a_share(d, h, hq, rows, lens):
    nt, share = share_of(lens, rows, h, hq // h, d)
    assert 8 <= share < 96 and nt == (1 if max(rows) * (hq // h) <= 8 else 2), share
    run(lens, rows, h, hq, d, 64, 100 + d, missing=[(0, 70), (0, 71), (1, 0), (len(lens) - 1, 40)])


@pytest.mark.parametrize("d,h,hq,rows,lens", [
    (128, 32, 32, [1, 1, 0, 1], [40011, 700, 3000, 9001]),
    (128, 8, 32, [4, 2, 0, 4], [70011, 40000, 900, 30001]),
    (64, 32, 64, [1, 1, 0, 1], [40011, 7000, 3000, 20001]),
    (64, 8, 64, [2, 7, 0, 4], [50011, 33000, 900, 20001])])
@pytest.mark.parametrize("tree", [False, True])
def test_items_of_two_sizes(d, h, hq, rows, lens, tree):
    _, share = share_of(lens, rows, h, hq // h, d)
    assert share >= 96, share
    run(lens, rows, h, hq, d, 128, 200 + d, missing=[(0, 70), (1, 3), (len(lens) - 1, 100)], tree=tree and max(rows) > 1)


@pytest.mark.skipif(CHECKED, reason="the sizes before it take every branch of the checked build")
@pytest.mark.parametrize("d,h,hq,lens", [(128, 8, 8, [400011, 300007, 150000]), (64, 4, 8, [1000003, 900000, 500000])])
def test_more_than_32_tiles_per_warp(d, h, hq, lens):
    """Big items of three tenths of a share, at least 132 tiles: a warp looks its pages up anew."""
    nt, share = share_of(lens, [1] * 3, h, hq // h, d)
    assert nt == 1 and share * 3 // 10 >= 132, share
    far = [w for w in range(0, lens[0] // 256, 37)]
    run(lens, [1] * 3, h, hq, d, 256, 300 + d, missing=[(0, w) for w in far])


@pytest.mark.parametrize("d,h,hq,m,lens", [
    (64, 1, 8, 1, [1900001]), (64, 1, 7, 1, [260700] * 7), (64, 1, 16, 1, [456001] * 3), (64, 2, 32, 1, [455007] * 2),
    (128, 1, 8, 1, [700001] * 2), (128, 1, 16, 1, [1000001]), (128, 1, 1, 16, [1000001])])
def test_few_long_segments(d, h, hq, m, lens):
    """A segment of hundreds of CTAs' shares: as many parts as the join's table holds (the checked build tests the table's stores too)."""
    nt, share = share_of(lens, [m] * len(lens), h, hq // h, d)
    assert share >= 96 and max(lens) // 32 > 80 * share, share
    run(lens, [m] * len(lens), h, hq, d, 256, 400 + d)


@pytest.mark.skipif(CHECKED, reason="the sizes before it take every branch of the checked build")
@pytest.mark.parametrize("d,h,hq,rows,lens", [(128, 2, 8, [700, 33, 0], [700, 900, 50]), (64, 4, 4, [300, 1, 300], [300, 5000, 4001])])
def test_prompt_rows(d, h, hq, rows, lens):
    """A prompt that is the whole sequence, and chunks of one behind what is there already: many row tiles per segment."""
    run(lens, rows, h, hq, d, 64, 500 + d, missing=[(len(lens) - 1, 0)])


@pytest.mark.skipif(CHECKED, reason="already inside the checked run")
def test_nothing_outside_its_buffers_at_these_sizes():
    env = dict(os.environ, MXQ_LIBRARY="checked")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_kv_division.py"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:] + r.stderr[-2000:]
