"""The key/value cache calls refuse bad arguments on the host, before anything is launched (fake pointers, no GPU)."""
import ctypes

import pytest

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import binding

A = 0x1000   # fake, aligned, never dereferenced
NULL, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 5


def struct(**kw):
    f = dict(pages=A, refs=A, num_pages=10, layers=2, kv_heads=8, head_dim=128, page_tokens=64)
    f.update(kw)
    c = binding._KvCacheStruct(**f)
    return c, ctypes.addressof(c)


def append(cache, layer=1, k=A, ks=1024, v=A, vs=1024, B=2, M=3, tables=A, W=4, lens=A, rows=None):
    return binding.lib().mxq_kv_append(cache, layer, k, ks, v, vs, B, M, tables, W, lens, rows, None)


def read(cache, layer=1, k=A, v=A, B=2, M=3, tables=A, W=4, lens=A, rows=None):
    return binding.lib().mxq_kv_read(cache, layer, k, v, B, M, tables, W, lens, rows, None)


def attention(cache, layer=1, q=A, qs=4096, B=2, M=3, hq=32, tables=A, W=4, lens=A, rows=None, tree=None, o=A, lse=None, ws=A, nws=1 << 40):
    return binding.lib().mxq_kv_attention(cache, layer, q, qs, B, M, hq, tables, W, lens, rows, tree, 0.1, o, lse, ws, nws, None)


def resize(cache, B=2, tables=A, W=4, lens=A, new=A):
    return binding.lib().mxq_kv_resize(cache, B, tables, W, lens, new, None)


def fork(cache, B=2, tables=A, W=4, lens=A, n=1, src=A, dst=A, ws=A, nws=1 << 20):
    return binding.lib().mxq_kv_fork(cache, B, tables, W, lens, n, src, dst, ws, nws, None)


def compact(cache, B=2, M=3, tables=A, W=4, lens=A, rows=None, keep=A, kept=A, out=A + 64):
    return binding.lib().mxq_kv_compact(cache, B, M, tables, W, lens, rows, keep, kept, out, None)


CALLS = [append, read, attention, resize, fork, compact]


@pytest.mark.parametrize("call", CALLS)
def test_every_call_checks_the_cache_and_the_sequences(call):
    ok, ptr = struct()
    assert call(None) == NULL
    for field in ("pages", "refs"):
        c, p = struct(**{field: None})
        assert call(p) == NULL
        c, p = struct(**{field: A + 8})
        assert call(p) == ALIGN
    for bad in (dict(num_pages=0), dict(num_pages=(1 << 24) + 1), dict(layers=0), dict(kv_heads=0), dict(kv_heads=257), dict(head_dim=96),
                dict(head_dim=0), dict(page_tokens=16), dict(page_tokens=48), dict(page_tokens=512)):
        c, p = struct(**bad)
        assert call(p) == SHAPE, bad
    for bad, want in ((dict(tables=None), NULL), (dict(lens=None), NULL), (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(W=0), SHAPE),
                      (dict(B=4096, W=1 << 19), SHAPE), (dict(tables=A + 2), ALIGN), (dict(lens=A + 1), ALIGN)):
        assert call(ptr, **bad) == want, bad


@pytest.mark.parametrize("call", [append, read, attention])
def test_calls_on_one_layer_check_it(call):
    c, p = struct()
    assert call(p, layer=2) == SHAPE and call(p, layer=-1) == SHAPE
    assert call(p, M=0) == SHAPE
    assert call(p, rows=A + 2) == ALIGN


def test_append_and_read():
    c, p = struct()
    assert append(p, k=None) == NULL and append(p, v=None) == NULL and read(p, k=None) == NULL and read(p, v=None) == NULL
    assert append(p, ks=1023) == SHAPE and append(p, vs=512) == SHAPE          # rows would overlap
    assert append(p, ks=1028) == ALIGN and append(p, k=A + 8) == ALIGN and read(p, v=A + 2) == ALIGN
    assert append(p, B=4096, M=1 << 20) == SHAPE and read(p, B=1024, M=1 << 17) == SHAPE


def test_attention():
    c, p = struct()
    assert attention(p, q=None) == NULL and attention(p, o=None) == NULL
    assert attention(p, hq=31) == SHAPE and attention(p, hq=4) == SHAPE and attention(p, qs=4088) == SHAPE
    assert attention(p, tree=A, M=65) == SHAPE
    assert attention(p, q=A + 8) == ALIGN and attention(p, o=A + 8) == ALIGN and attention(p, qs=4100) == ALIGN
    assert attention(p, lse=A + 2) == ALIGN and attention(p, tree=A + 4) == ALIGN and attention(p, ws=A + 8) == ALIGN
    assert attention(p, ws=None) == WORKSPACE and attention(p, nws=64) == WORKSPACE


def test_pages():
    c, p = struct()
    assert resize(p, new=None) == NULL and resize(p, new=A + 2) == ALIGN
    assert fork(p, src=None) == NULL and fork(p, dst=None) == NULL and fork(p, n=0) == SHAPE and fork(p, n=4097) == SHAPE
    assert fork(p, src=A + 2) == ALIGN and fork(p, ws=A + 8) == ALIGN and fork(p, ws=None) == WORKSPACE and fork(p, n=100, nws=64) == WORKSPACE
    assert compact(p, keep=None) == NULL and compact(p, kept=None) == NULL and compact(p, out=None) == NULL
    assert compact(p, M=0) == SHAPE and compact(p, M=65) == SHAPE and compact(p, out=A) == SHAPE      # lens_out is lens
    assert compact(p, rows=A + 2) == ALIGN and compact(p, keep=A + 1) == ALIGN


def test_sizes():
    assert mxq.mxq_kv_page_bytes(8, 128, 64) == 2 * 8 * 34 * 128 and mxq.mxq_kv_page_bytes(1, 64, 32) == 34 * 64
    assert mxq.mxq_kv_page_bytes(8, 128, 64) * 8 == 8 * 64 * 2 * 128 * 4.25
    for bad in ((0, 128, 64), (8, 32, 64), (8, 128, 40), (300, 64, 32)):
        assert mxq.mxq_kv_page_bytes(*bad) == 0
    assert mxq.mxq_kv_fork_workspace_bytes(0) == 0 and mxq.mxq_kv_fork_workspace_bytes(5) > 0
    assert mxq.mxq_kv_attention_workspace_bytes(1, 1, 32, 8, 128) >= 4096
    for bad in ((0, 1, 32, 8, 128), (1, 0, 32, 8, 128), (1, 1, 30, 8, 128), (1, 1, 32, 8, 80)):
        assert mxq.mxq_kv_attention_workspace_bytes(*bad) == 0
