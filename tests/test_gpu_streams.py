"""Calls on a stream= other than the current one, with everything they need allocated by the binding, while the current stream is
busy and the memory that was freed last holds other bytes than zeros."""
import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu

BUSY = 200_000_000      # clock cycles of the current stream: about a tenth of a second


def dirty(nbytes):
    """Leave freed blocks of all bits set, of the size about to be asked for, to the current stream's allocator."""
    blocks = [torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    del blocks


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture()
def sequences():
    """Three sequences of a two-layer cache, the first one long enough for its segments to be cut."""
    lens, h, d = [9000, 100, 64], 2, 64
    cache = mxq.KVCache.new(2, 400, h, d, 32)
    tables, t_lens = cache.new_sequences(5, 9600)
    mxq.mxq_kv_resize(cache, tables, t_lens, i32(*lens, 0, 0))
    g = torch.Generator(device="cuda").manual_seed(1)
    for layer in range(2):
        k, v = (torch.randn(5, 9000, h, d, generator=g, device="cuda").bfloat16() for _ in range(2))
        mxq.mxq_kv_append(cache, layer, k, v, tables, t_lens, rows=t_lens)
    q = torch.randn(5, 2, 8, d, generator=g, device="cuda").bfloat16()
    torch.cuda.synchronize()
    return cache, tables, t_lens, q


def test_attention_and_read(sequences):
    cache, tables, lens, q = sequences
    want, wl = mxq.mxq_kv_attention(q, cache, 1, tables, lens, with_lse=True)
    wk, wv = mxq.mxq_kv_read(cache, 1, tables, lens, 70)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        dirty(mxq.mxq_kv_attention_workspace_bytes(5, 2, 8, 2, 64))
        torch.cuda.synchronize()
        torch.cuda._sleep(BUSY)
        out, lse = mxq.mxq_kv_attention(q, cache, 1, tables, lens, with_lse=True, stream=side)
        k, v = mxq.mxq_kv_read(cache, 1, tables, lens, 70, stream=side)
        side.synchronize()
        with torch.cuda.stream(side):       # (what came back belongs to the side stream)
            same = torch.equal(out, want), torch.equal(lse, wl), torch.equal(k, wk), torch.equal(v, wv)
        assert all(same), same
    torch.cuda.synchronize()
    assert mxq.mxq_linear_device_status() == 0


def test_fork_and_compact(sequences):
    cache, tables, lens, _ = sequences
    twin_pages, twin_refs = cache.pages.clone(), cache.refs.clone()
    twin = mxq.KVCache(twin_pages, twin_refs, cache.kv_heads, cache.head_dim, cache.page_tokens)
    t2, l2 = tables.clone(), lens.clone()
    rows, keep, kept = i32(5, 5, 5, 0, 0), torch.tensor([[0, 2, 4, 0, 0]] * 5, dtype=torch.int32, device="cuda"), i32(3, 2, 1, 0, 0)
    src, dst = i32(0, 1), i32(3, 4)
    want = mxq.mxq_kv_compact(twin, t2, l2, rows, keep, kept)
    mxq.mxq_kv_resize(twin, t2, l2, want)
    mxq.mxq_kv_fork(twin, t2, l2, src, dst)
    side = torch.cuda.Stream()
    dirty(mxq.mxq_kv_fork_workspace_bytes(2))
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    got = mxq.mxq_kv_compact(cache, tables, lens, rows, keep, kept, stream=side)
    mxq.mxq_kv_resize(cache, tables, lens, got, stream=side)
    mxq.mxq_kv_fork(cache, tables, lens, src, dst, stream=side)
    blocks = [torch.full((512,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]      # (the current stream's allocations go on)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(tables, t2) and torch.equal(lens, l2) and torch.equal(cache.refs, twin.refs)
    assert np.array_equal(cache.pages.cpu().numpy(), twin.pages.cpu().numpy())
    del blocks


def test_layers_on_two_streams_at_once():
    """Split layers (whose workspace holds counters) on two streams side by side, nothing passed but the operands."""
    g = torch.Generator(device="cuda").manual_seed(2)
    w = [mxq.mxq_quantize(torch.randn(1024, 4096, generator=g, device="cuda").bfloat16()) for _ in range(2)]
    x = [torch.randn(m, 4096, generator=g, device="cuda").bfloat16() for m in (1, 8)]
    want = [[mxq.mxq_linear(a, *b) for a in x] for b in w]
    wc = mxq.mxq_quantize(x[1])
    draft = torch.zeros(7, dtype=torch.int32, device="cuda")
    wv = mxq.mxq_lm_head_accept(x[1], *w[0], draft)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    dirty(mxq.mxq_linear_workspace_bytes(8, 1024, 4096))
    dirty(mxq.mxq_lm_head_accept_workspace_bytes(8, 1024, 4096))
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    got = [[] for _ in sides]
    for _ in range(20):
        for i, s in enumerate(sides):
            got[i].append([mxq.mxq_linear(a, *w[i], stream=s) for a in x])
    codes = mxq.mxq_quantize(x[1], stream=sides[0])
    tokens = mxq.mxq_lm_head_accept(x[1], *w[0], draft, stream=sides[1])
    torch.cuda.synchronize()
    for i in range(2):
        for ys in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(ys, want[i]))
    assert all(torch.equal(a, b) for a, b in zip(codes + tokens, wc + wv))
    assert mxq.mxq_linear_device_status() == 0
