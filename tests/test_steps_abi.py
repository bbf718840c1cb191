"""The norm, the rotated append, the logit rules and the adapters refuse bad arguments on the host, before anything is launched (fake
pointers, no GPU), and the binding checks shapes and types before it calls them."""
import ctypes

import pytest
import torch

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import binding

A = 0x1000   # fake, aligned, never dereferenced
NULL, SHAPE, ALIGN, DTYPE, WORKSPACE = 1, 2, 3, 4, 5
F32, BF16 = 0, 1
INF = float("inf")


def norm(x=A, xt=BF16, stride=64, res=A, rt=BF16, out=A, w=A, wt=BF16, eps=1e-5, M=3, K=64, y=A, codes=None, scales=None):
    return binding.lib().mxq_rmsnorm(x, xt, stride, res, rt, out, w, wt, eps, M, K, y, codes, scales, None)


@pytest.mark.parametrize("bad,want", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(y=None), NULL), (dict(codes=A), NULL), (dict(scales=A), NULL), (dict(res=None), NULL),
    (dict(M=0), SHAPE), (dict(M=1 << 31), SHAPE), (dict(K=0), SHAPE), (dict(K=48), SHAPE), (dict(K=32800, stride=32800), SHAPE),
    (dict(stride=56), SHAPE), (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=INF), SHAPE),
    (dict(xt=2), DTYPE), (dict(wt=-1), DTYPE), (dict(rt=7), DTYPE),
    (dict(x=A + 8), ALIGN), (dict(res=A + 4), ALIGN), (dict(out=A + 2), ALIGN), (dict(w=A + 8), ALIGN), (dict(y=A + 8), ALIGN),
    (dict(codes=A + 8, scales=A), ALIGN), (dict(codes=A, scales=A + 1), ALIGN), (dict(stride=68), ALIGN), (dict(xt=F32, stride=66), ALIGN)])
def test_norm(bad, want):
    assert norm(**bad) == want


def test_dequantize_mxfp8():
    call = lambda c=A, s=A, N=3, K=64, o=A, t=F32: binding.lib().mxq_dequantize_mxfp8(c, s, N, K, o, t, None)
    assert call(c=None) == NULL and call(s=None) == NULL and call(o=None) == NULL
    assert call(N=0) == SHAPE and call(K=40) == SHAPE and call(N=1 << 50) == SHAPE and call(t=2) == DTYPE
    assert call(c=A + 1) == ALIGN and call(s=A + 4) == ALIGN and call(o=A + 8) == ALIGN


def rope(cache={}, rp={}, q=A, qs=4096, hq=32, qo=A, qos=4096, k=A, ks=1024, v=A, vs=1024, B=2, M=3, tables=A, W=4, lens=A, rows=None, positions=None,
         layer=1):
    c = binding._KvCacheStruct(**dict(dict(pages=A, refs=A, num_pages=10, layers=2, kv_heads=8, head_dim=128, page_tokens=64), **cache))
    r = binding._RopeStruct(**dict(dict(table=A, positions=100, rotary_dim=128, style=0), **rp)) if rp is not None else None
    return binding.lib().mxq_kv_append_rope(ctypes.addressof(c), layer, q, qs, hq, qo, qos, k, ks, v, vs, B, M, tables, W, lens, rows,
                                            None if r is None else ctypes.addressof(r), positions, None)


@pytest.mark.parametrize("bad,want", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(q=None), NULL), (dict(qo=None), NULL), (dict(rp=None), NULL), (dict(rp=dict(table=None)), NULL),
    (dict(tables=None), NULL), (dict(lens=None), NULL), (dict(cache=dict(pages=None)), NULL), (dict(cache=dict(refs=None)), NULL),
    (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE), (dict(M=0), SHAPE), (dict(B=0), SHAPE), (dict(W=0), SHAPE), (dict(hq=0), SHAPE),
    (dict(hq=33), SHAPE), (dict(qs=4088), SHAPE), (dict(qos=4088), SHAPE), (dict(ks=1016), SHAPE), (dict(vs=512), SHAPE),
    (dict(B=4096, M=1 << 14), SHAPE), (dict(cache=dict(head_dim=96)), SHAPE),
    (dict(rp=dict(rotary_dim=0)), SHAPE), (dict(rp=dict(rotary_dim=24)), SHAPE), (dict(rp=dict(rotary_dim=144)), SHAPE),
    (dict(rp=dict(style=2)), SHAPE), (dict(rp=dict(positions=0)), SHAPE), (dict(rp=dict(positions=(1 << 31) + 1)), SHAPE),
    (dict(cache=dict(head_dim=64), rp=dict(rotary_dim=128)), SHAPE),
    (dict(q=A + 8), ALIGN), (dict(qo=A + 2), ALIGN), (dict(k=A + 8), ALIGN), (dict(v=A + 4), ALIGN), (dict(rp=dict(table=A + 4)), ALIGN),
    (dict(qs=4100), ALIGN), (dict(qos=4098), ALIGN), (dict(ks=1028), ALIGN), (dict(vs=1025), ALIGN), (dict(rows=A + 2), ALIGN), (dict(positions=A + 1), ALIGN)])
def test_append_rope(bad, want):
    assert rope(**bad) == want


def test_rope_table():
    call = lambda f=A, n=10, d=64, t=A: binding.lib().mxq_rope_table(f, n, d, 1.0, t, None)
    assert call(f=None) == NULL and call(t=None) == NULL and call(n=0) == SHAPE and call(n=(1 << 31) + 1) == SHAPE
    assert call(d=0) == SHAPE and call(d=40) == SHAPE and call(d=144) == SHAPE and call(f=A + 4) == ALIGN and call(t=A + 8) == ALIGN


def rules(**kw):
    return binding._LogitRulesStruct(**dict(dict(counts=A, penalties=A, bias_tokens=A, bias_values=A, allowed=A, bias_count=5, reserved=0), **kw))


def adjust(ru={}, logits=A, t=F32, B=2, R=4, V=100, draft=A, T=3, out=A):
    r = rules(**ru) if ru is not None else None
    return binding.lib().mxq_logits_adjust(logits, t, B, R, V, draft, T, None if r is None else ctypes.addressof(r), out, None)


def accept(ru={}, logits=A, t=F32, B=2, R=4, V=100, draft=A, T=3, ver=A, n=A, nxt=A, ws=A, nws=1 << 20):
    r = rules(**ru) if ru is not None else None
    return binding.lib().mxq_greedy_accept_rules(logits, t, B, R, V, draft, T, None if r is None else ctypes.addressof(r), ver, n, nxt, ws, nws, None)


@pytest.mark.parametrize("call", [adjust, accept])
@pytest.mark.parametrize("bad,want", [
    (dict(logits=None), NULL), (dict(ru=None), NULL), (dict(draft=None), NULL), (dict(ru=dict(bias_tokens=None)), NULL), (dict(ru=dict(bias_values=None)), NULL),
    (dict(B=0), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 31) - 100), SHAPE), (dict(T=65, R=65), SHAPE), (dict(T=-1), SHAPE), (dict(R=2), SHAPE),
    (dict(R=5), SHAPE), (dict(T=0, R=0), SHAPE), (dict(B=1 << 20), SHAPE), (dict(ru=dict(bias_count=-1)), SHAPE), (dict(ru=dict(bias_count=1025)), SHAPE),
    (dict(t=2), DTYPE), (dict(logits=A + 8), ALIGN), (dict(draft=A + 2), ALIGN), (dict(ru=dict(counts=A + 1)), ALIGN), (dict(ru=dict(penalties=A + 2)), ALIGN),
    (dict(ru=dict(allowed=A + 2)), ALIGN), (dict(ru=dict(bias_tokens=A + 2)), ALIGN), (dict(ru=dict(bias_values=A + 3)), ALIGN)])
def test_rules(call, bad, want):
    assert call(**bad) == want


def test_adjust_and_accept():
    assert adjust(out=None) == NULL and adjust(out=A + 4) == ALIGN
    assert accept(ver=None) == NULL and accept(n=None) == NULL and accept(nxt=None) == NULL
    assert accept(ws=None) == WORKSPACE and accept(nws=16) == WORKSPACE and accept(ws=A + 8) == ALIGN and accept(nxt=A + 2) == ALIGN
    assert mxq.mxq_greedy_accept_rules_workspace_bytes(2, 4, 100) >= 2 * 4 * 8 + 2 * 4
    for bad in ((0, 4, 100), (2, 0, 100), (2, 66, 100), (2, 4, 0)):
        assert mxq.mxq_greedy_accept_rules_workspace_bytes(*bad) == 0


def test_token_counts():
    call = lambda c=A, B=2, V=100, t=A, L=5, n=None, x=None: binding.lib().mxq_token_counts(c, B, V, t, L, n, x, 0, None)
    assert call(c=None) == NULL and call(t=None) == NULL and call(B=0) == SHAPE and call(V=0) == SHAPE and call(L=0) == SHAPE
    assert call(B=1 << 20, L=1 << 31) == SHAPE
    assert call(c=A + 2) == ALIGN and call(t=A + 1) == ALIGN and call(n=A + 2) == ALIGN and call(x=A + 3) == ALIGN


def lora(ad={}, x=A, M=5, ids=A, N=100, K=64, base=A, y=A, t=F32, ws=A, nws=1 << 30):
    s = binding._LoraStruct(**dict(dict(a=A, b=A, scale=A, rank=16, count=3), **ad)) if ad is not None else None
    return binding.lib().mxq_lora(x, M, None if s is None else ctypes.addressof(s), ids, N, K, base, y, t, ws, nws, None)


def linear_lora(ad={}, x=A, M=5, codes=A, scales=A, ids=A, N=100, K=64, y=A, t=F32, ws=A, nws=1 << 30):
    s = binding._LoraStruct(**dict(dict(a=A, b=A, scale=A, rank=16, count=3), **ad)) if ad is not None else None
    return binding.lib().mxq_linear_lora(x, M, codes, scales, N, K, None if s is None else ctypes.addressof(s), ids, y, t, ws, nws, None)


@pytest.mark.parametrize("call", [lora, linear_lora])
@pytest.mark.parametrize("bad,want", [
    (dict(x=None), NULL), (dict(ad=None), NULL), (dict(ad=dict(a=None)), NULL), (dict(ad=dict(b=None)), NULL), (dict(ids=None), NULL), (dict(y=None), NULL),
    (dict(M=0), SHAPE), (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=40), SHAPE), (dict(ad=dict(rank=0)), SHAPE), (dict(ad=dict(rank=12)), SHAPE),
    (dict(ad=dict(rank=136)), SHAPE), (dict(ad=dict(count=0)), SHAPE), (dict(ad=dict(count=65537)), SHAPE), (dict(M=(1 << 20) + 1), SHAPE),
    (dict(t=5), DTYPE), (dict(x=A + 8), ALIGN), (dict(ad=dict(a=A + 2)), ALIGN), (dict(ad=dict(b=A + 8)), ALIGN), (dict(ad=dict(scale=A + 2)), ALIGN),
    (dict(ids=A + 2), ALIGN), (dict(y=A + 4), ALIGN), (dict(ws=A + 8), ALIGN), (dict(ws=None), WORKSPACE), (dict(nws=64), WORKSPACE)])
def test_adapters(call, bad, want):
    assert call(**bad) == want


def test_adapters_beside_the_layer():
    assert linear_lora(M=17) == SHAPE and linear_lora(codes=None) == NULL and linear_lora(scales=None) == NULL
    assert linear_lora(codes=A + 8) == ALIGN and linear_lora(scales=A + 8) == ALIGN and lora(base=A + 8) == ALIGN
    assert mxq.mxq_linear_lora_workspace_bytes(17, 64, 64, 16, 1) == 0 and mxq.mxq_lora_workspace_bytes(0, 64, 64, 16, 1) == 0
    assert mxq.mxq_linear_lora_workspace_bytes(3, 64, 64, 16, 1) >= mxq.mxq_lora_workspace_bytes(3, 64, 64, 16, 1) + 3 * 64 * 4


def test_the_binding_checks_shapes_before_it_calls():
    t = lambda *s, d=torch.float32: torch.zeros(*s, dtype=d)
    with pytest.raises(TypeError):
        mxq.mxq_rmsnorm(t(2, 32), t(32))                              # not on the GPU
    with pytest.raises(ValueError):
        mxq.LogitRules(bias_tokens=t(2, 3, d=torch.int32))
    with pytest.raises(TypeError):
        mxq.LogitRules(counts=t(2, 3, d=torch.int32))
    with pytest.raises(ValueError):
        mxq.Rope(t(4, 32), style="thirds")
    with pytest.raises(ValueError):
        mxq.mxq_lora(t(2, 64, d=torch.bfloat16), t(3, 8, 32, d=torch.bfloat16), t(3, 10, 8, d=torch.bfloat16), t(2, d=torch.int32))
    with pytest.raises(ValueError):
        mxq.mxq_lora(t(2, 64, d=torch.bfloat16), t(3, 8, 64, d=torch.bfloat16), t(3, 10, 16, d=torch.bfloat16), t(2, d=torch.int32))
