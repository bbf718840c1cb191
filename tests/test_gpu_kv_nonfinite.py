"""Infinities and NaN in mxq_kv_attention: in queries, in keys and in values, in segments that are whole and in segments that are
joined from many parts.  The rule of include/mxq.h: a score of NaN or +inf makes its row NaN, output and lse; scores of -inf are
weights of zero, and a row that has no others is empty (O = 0, lse = -inf)."""
import math

import pytest
import torch

import kv_exact
import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu

LENGTHS = [[60, 33], [5000, 9001]]      # whole segments; parts


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def cache_of(lens, h, d, seed, change):
    """Random keys and values, changed by change(sequence, k [n][h][d], v), cast into a cache."""
    cache = mxq.KVCache.new(1, sum(-(-n // 64) for n in lens) + 1, h, d, 64)
    tables, t_lens = cache.new_sequences(len(lens), max(lens))
    mxq.mxq_kv_resize(cache, tables, t_lens, i32(lens))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for b, n in enumerate(lens):
        k, v = (torch.randn(n, h, d, generator=gen, device="cuda") for _ in range(2))
        change(b, k, v)
        mxq.mxq_kv_append(cache, 0, k.bfloat16().unsqueeze(0), v.bfloat16().unsqueeze(0), tables[b:b + 1], t_lens[b:b + 1])
    return cache, tables, t_lens, gen


def attend(q, cache, tables, lens):
    ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(*q.shape[:3], cache.kv_heads, q.shape[3]))
    return mxq.mxq_kv_attention(q, cache, 0, tables, lens, workspace=ws, with_lse=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 3])
@pytest.mark.parametrize("lens", LENGTHS)
def test_nan_in_queries_and_keys(lens, m, d):
    """A NaN in a query: its row, lse too.  A key of NaN: the rows that see it (not those before it, not other heads).  A sequence
    of nothing but such keys: every row."""
    h, hq = 2, 8

    def change(b, k, v):
        k[-1, 0, 3] = math.nan                       # seen by the last row only
        if b == 1:
            k[:, 1, 40 % d] = math.inf               # a block with an Inf is held as NaN
    cache, tables, t_lens, gen = cache_of(lens, h, d, 7, change)
    q = torch.randn(2, m, hq, d, generator=gen, device="cuda").bfloat16()
    q[0, 0, 6, d - 1] = math.nan
    out, lse = attend(q, cache, tables, t_lens)
    kv_exact.check(out, lse, kv_exact.attention(cache, 0, q, tables, lens, [m] * 2, d ** -0.5), d, adds=1024)
    nan = torch.isnan(lse)
    want = torch.zeros_like(nan)
    want[:, -1, :4] = True
    want[1, :, 4:] = True
    want[0, 0, 6] = True
    assert torch.equal(nan, want) and torch.equal(torch.isnan(out).all(-1), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("others", [1.0, 1e30, 1e38])
@pytest.mark.parametrize("lens", LENGTHS)
def test_infinite_queries(lens, others, d):
    """Scores of -inf everywhere: an empty row, whatever the row's finite elements; one of +inf: NaN; +inf and -inf by halves: NaN."""
    def change(b, k, v):
        k[..., 0] = 2.0                              # (not rounded to zero, whatever its block holds)
        k[len(k) // 2, 1, 0] = -2.0
    cache, tables, t_lens, gen = cache_of(lens, 2, d, 8, change)
    q = (torch.randn(2, 2, 4, d, generator=gen, device="cuda") * others).clamp(-3e38, 3e38).bfloat16()
    q[:, 0, :, 0] = -math.inf                        # head 0's keys (rows 0, 1 of the group): all -inf; head 1's: one +inf
    q[:, 1, :, 0] = torch.tensor([math.inf, -math.inf, math.inf, -math.inf])
    finite = q[0, 1].clone()
    q[1, 1], q[1, 1, :, 0] = finite, 0.5
    if others != 1.0:
        q[1, 1] = 0.25
    out, lse = attend(q, cache, tables, t_lens)
    empty = torch.isneginf(lse) & (out == 0).all(-1)
    nan = torch.isnan(lse) & torch.isnan(out).all(-1)
    assert bool(empty[:, 0, :2].all()) and bool(nan[:, 0, 2:].all())
    assert nan[0, 1].tolist() == [True, False, True, True] and empty[0, 1].tolist() == [False, True, False, False]
    rest = kv_exact.attention(cache, 0, q[1:, 1:], tables[1:], lens[1:], [1], d ** -0.5)
    kv_exact.check(out[1:, 1:], lse[1:, 1:], rest, d, adds=1024)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENGTHS)
def test_nan_values(lens, d):
    """V of NaN: the output of every row that sees the token, not its lse, and no other row."""
    def change(b, k, v):
        v[-1] = math.nan
    cache, tables, t_lens, gen = cache_of(lens, 2, d, 9, change)
    q = torch.randn(2, 2, 4, d, generator=gen, device="cuda").bfloat16()
    out, lse = attend(q, cache, tables, t_lens)
    assert bool(torch.isfinite(out[:, 0]).all()) and bool(torch.isnan(out[:, 1]).all()) and bool(torch.isfinite(lse).all())
