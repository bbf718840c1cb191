"""mxq_kv_append_rope and mxq_rope_table: the rotation is defined to the bit (FP32, one rounding per operation), so are the queries in BF16
and the cached keys; compared with a step-by-step FP32 rotation and the cast of its results."""
import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq
import step_plain as plain

pytestmark = pytest.mark.gpu


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def table(positions, rotary, seed=0):
    f = 10000.0 ** (-2 * np.arange(rotary // 2) / rotary)
    a = np.arange(positions)[:, None] * f
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def setup(b, m, hq, hkv, d, lens, page=32, layers=2, seed=0, fused=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = mxq.KVCache.new(layers, sum(-(-n // page) for n in lens) + 3, hkv, d, page)
    tables, tl = cache.new_sequences(b, max(max(lens), 1) + 2 * page)
    cache.pages.fill_(0x5A)
    mxq.mxq_kv_resize(cache, tables, tl, i32(*lens))
    heads = hq + 2 * hkv
    qkv = (torch.randn(b, m, heads, d, generator=g, device="cuda") * torch.exp(torch.randn(heads, d, generator=g, device="cuda"))).bfloat16()
    return cache, tables, tl, qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]


def expected(q, k, v, where, there, tab, style):
    rot = tab.shape[1]
    ok = (where >= 0) & (where < len(tab))
    rows = np.where(ok[..., None], tab[np.clip(where, 0, len(tab) - 1)], np.float32(np.nan))[:, :, None]
    out = [plain.rotate(x.float().cpu().numpy(), rows[..., :rot // 2], rows[..., rot // 2:], rot, style) for x in (q, k)]
    there = there[:, :, None, None]
    with np.errstate(all="ignore"):
        return (np.where(there, plain.bf16(out[0]), 0), np.where(there, plain.cast_fp4(out[1]), 0), np.where(there, plain.cast_fp4(v.float().cpu().numpy()), 0))


def same(got, want):
    got = got.float().cpu().numpy()
    assert got.shape == want.shape and np.array_equal(got, want.astype(np.float32), equal_nan=True), np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))))[:5]


@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("b,m,hq,hkv,d,rot", [
    (1, 1, 32, 8, 128, 128), (1, 1, 1, 1, 64, 64), (3, 1, 9, 3, 64, 16), (2, 5, 12, 4, 64, 32), (5, 3, 7, 1, 128, 96), (2, 9, 16, 2, 128, 64),
    (2, 4, 8, 8, 128, 16), (1, 2, 5, 5, 128, 112), (64, 40, 40, 8, 128, 128), (50, 33, 12, 4, 64, 48)])
def test_rows_of_every_shape(b, m, hq, hkv, d, rot, style):
    rng = np.random.default_rng(b * 1000 + m)
    lens = [int(x) for x in rng.integers(m, m + 70, b)]
    rows = rng.integers(0, m + 1, b)
    cache, tables, tl, q, k, v = setup(b, m, hq, hkv, d, lens)
    tab = table(128, rot)
    rope = mxq.Rope(torch.from_numpy(tab).cuda(), style)
    before = cache.pages.clone()
    out = mxq.mxq_kv_append_rope(cache, 1, q, k, v, tables, tl, rope, rows=i32(*rows))
    i = np.arange(m)
    where, there = (np.array(lens) - rows)[:, None] + i, i < rows[:, None]
    wq, wk, wv = expected(q, k, v, where, there, tab, style)
    same(out, wq)
    gk, gv = mxq.mxq_kv_read(cache, 1, tables, tl, m, rows=i32(*rows))
    same(gk, wk), same(gv, wv)
    assert torch.equal(cache.pages[0], before[0])                      # the other layer is as it was
    # the values' bytes are the append's own, and so are the keys' where the angles are zero
    twin = mxq.KVCache(before.clone(), cache.refs, hkv, d, 32)
    mxq.mxq_kv_append(twin, 1, k, v, tables, tl, rows=i32(*rows))
    still = mxq.KVCache(before.clone(), cache.refs, hkv, d, 32)
    zero = torch.cat([torch.ones(1, rot // 2, device="cuda"), torch.zeros(1, rot // 2, device="cuda")], 1).repeat(4, 1)
    mxq.mxq_kv_append_rope(still, 1, None, k, v, tables, tl, mxq.Rope(zero, style), rows=i32(*rows), positions=torch.ones(b, m, dtype=torch.int32, device="cuda"))
    kz, vz = mxq.mxq_kv_read(still, 1, tables, tl, m, rows=i32(*rows))
    kt, vt = mxq.mxq_kv_read(twin, 1, tables, tl, m, rows=i32(*rows))
    assert torch.equal(kz, kt) and torch.equal(vz, vt) and torch.equal(gv, vt)


def test_positions_of_a_tree_in_place_queries_and_positions_outside_the_table():
    b, m, hq, hkv, d = 3, 6, 8, 2, 64
    lens, rows = [40, 6, 90], np.array([6, 4, 5])
    for rot, style in ((64, "halves"), (32, "halves"), (48, "pairs")):
        cache, tables, tl, q, k, v = setup(b, m, hq, hkv, d, lens)
        tab = table(88, rot)
        where = np.array([[34, 35, 35, 36, 36, 37], [2, 3, 3, 4, 0, 0], [85, 86, 88, -1, 87, 1 << 30]])
        want = expected(q, k, v, where, np.arange(m) < rows[:, None], tab, style)
        got = mxq.mxq_kv_append_rope(cache, 0, q, k, v, tables, tl, mxq.Rope(torch.from_numpy(tab).cuda(), style), rows=i32(*rows),
                                     positions=torch.tensor(where, dtype=torch.int32, device="cuda"), q_out=q)
        assert got is q
        same(q, want[0])
        for x, w in zip(mxq.mxq_kv_read(cache, 0, tables, tl, m, rows=i32(*rows)), want[1:]):
            same(x, w)
        assert np.isnan(want[1][2, 2, :, :32]).all() and not np.isnan(want[2]).any()


def test_rows_without_a_place():
    """More rows than tokens, an empty sequence, a page that is missing: nothing is written outside, queries of rows that are not there
    are zero, those of rows whose page is missing are rotated."""
    b, m, hq, hkv, d = 4, 8, 4, 2, 64
    cache, tables, tl, q, k, v = setup(b, m, hq, hkv, d, [3, 0, 40, 70])
    tables[2, 1] = -1                                   # tokens 32..39
    tables[3, 2] = 1 << 20
    before = cache.pages.clone()
    tab = table(100, 64)
    out = mxq.mxq_kv_append_rope(cache, 0, q, k, v, tables, tl, mxq.Rope(torch.from_numpy(tab).cuda()))
    place = np.array([3, 0, 40, 70])[:, None] - m + np.arange(m)
    wq, wk, wv = expected(q, k, v, place, place >= 0, tab, "halves")
    same(out, wq)
    gk, gv = mxq.mxq_kv_read(cache, 0, tables, tl, m)
    stored = (place >= 0) & ~((np.arange(b)[:, None] == 2) & (place >= 32)) & ~((np.arange(b)[:, None] == 3) & (place >= 64))
    same(gk, np.where(stored[:, :, None, None], wk, 0)), same(gv, np.where(stored[:, :, None, None], wv, 0))
    changed = (cache.pages != before).view(2, cache.num_pages, -1).any(-1)[0].nonzero().flatten().tolist()
    assert set(changed) <= {int(tables[0, 0]), int(tables[3, 1])}
    assert torch.equal(cache.pages[1], before[1])


def test_values_that_are_not_finite_and_keys_that_overflow():
    b, m, hq, hkv, d = 1, 4, 2, 2, 64
    cache, tables, tl, q, k, v = setup(b, m, hq, hkv, d, [4])
    k[0, 0, 0, 3] = float("inf")
    k[0, 1, 1, 40] = float("nan")
    v[0, 2, 0, 63] = float("-inf")
    k[0, 3, 0, 5], k[0, 3, 0, 37] = 3e38, -3e38         # the rotation's sum leaves FP32
    tab = np.concatenate([np.full((8, 32), np.float32(0.75)), np.full((8, 32), np.float32(0.66))], 1)
    mxq.mxq_kv_append_rope(cache, 0, None, k, v, tables, tl, mxq.Rope(torch.from_numpy(tab).cuda()))
    with np.errstate(all="ignore"):
        _, wk, wv = expected(q, k, v, np.arange(4)[None], np.ones((1, 4), bool), tab, "halves")
    gk, gv = mxq.mxq_kv_read(cache, 0, tables, tl, m)
    same(gk, wk), same(gv, wv)
    assert np.isnan(wk).any() and np.isnan(wv).sum() == 32


@pytest.mark.parametrize("rot", [16, 64, 128])
def test_table(rot):
    f = torch.tensor(500000.0 ** (-2 * np.arange(rot // 2) / rot), dtype=torch.float64, device="cuda")
    n = 200001
    t = mxq.mxq_rope_table(f, n, amplitude=1.25).cpu().numpy()
    a = np.arange(n)[:, None] * f.cpu().numpy()
    # amplitude * cosine in 64 bits, rounded once (the 64-bit angle is within 2^-53 of itself: 2e5 * 2^-53 in the cosine)
    for half, want in ((t[:, :rot // 2], 1.25 * np.cos(a)), (t[:, rot // 2:], 1.25 * np.sin(a))):
        assert (np.abs(half - want) <= 2.0 ** -24 * np.abs(want) + 1e-10).all()
