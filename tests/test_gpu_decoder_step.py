"""The example that runs norms, adapters, rotated appends, attention and the rules together, against the same decoder in plain FP32 with the
roundings that the calls state: BF16 activations, 4-bit keys and values."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq
import step_plain as plain

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decoder_step", os.path.join(ROOT, "examples", "decoder_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def plain_logits(ex, w, tokens, adapter):
    """[len, VOCAB] of one sequence, every token attending to those before it."""
    bf = lambda x: x.bfloat16().float()
    weight = lambda pair: mxq.mxq_dequantize(*pair).float()
    norm = lambda h, g: bf(h / (h.square().mean(-1, keepdim=True) + 1e-5).sqrt() * g.float())
    n = len(tokens)
    pos = np.arange(n)[:, None] * 10000.0 ** (-2 * np.arange(ex.HEAD_DIM // 2) / ex.HEAD_DIM)
    cos, sin = np.cos(pos).astype(np.float32)[:, None], np.sin(pos).astype(np.float32)[:, None]
    turn = lambda x: plain.rotate(x.cpu().numpy(), cos, sin, ex.HEAD_DIM, "halves")
    h = w.embedding[torch.tensor(tokens, device="cuda")].float()
    for lay in w.layers:
        x = norm(h, lay["norm1"])
        y = x @ weight(lay["qkv"]).T
        if adapter >= 0:
            y = y + w.scale[adapter] * (x @ lay["a"][adapter].float().T) @ lay["b"][adapter].float().T
        y = bf(y).view(n, -1, ex.HEAD_DIM)
        q, k, v = y[:, :ex.HEADS], y[:, ex.HEADS:ex.HEADS + ex.KV_HEADS], y[:, ex.HEADS + ex.KV_HEADS:]
        cast = lambda a: torch.from_numpy(plain.cast_fp4(a)).float().cuda().repeat_interleave(ex.HEADS // ex.KV_HEADS, 1)
        q, k, v = bf(torch.from_numpy(turn(q)).cuda()), cast(turn(k)), cast(v.cpu().numpy())
        s = torch.einsum("mhd,nhd->hmn", q, k) * ex.HEAD_DIM ** -0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -torch.inf)
        a = bf(torch.einsum("hmn,nhd->mhd", torch.softmax(s, -1), v)).reshape(n, -1)
        h = bf(h + a @ weight(lay["out"]).T)
        x = norm(h, lay["norm2"])
        gu = x @ weight(lay["gate_up"]).T
        act = bf(torch.nn.functional.silu(gu[:, 0::2]) * gu[:, 1::2])
        h = bf(h + act @ weight(lay["down"]).T)
    return norm(h, w.norm) @ weight(w.head).T


def test_the_example_runs(example):
    server, prompts, streams = example.main(8)
    for s, p, n in zip(streams, prompts, server.lens.tolist()):
        assert len(s) - 1 == n and all(0 <= t < example.VOCAB for t in s)      # (the last token is not in the cache yet)
    counts = server.counts.cpu().numpy().view(np.uint32)
    for b, (s, p) in enumerate(zip(streams, prompts)):
        want = np.zeros(example.VOCAB, np.int64)
        for t in s[len(p):]:
            want[t] += 1
        want[p] |= 1 << 31
        assert np.array_equal(counts[b], want)
    assert int((server.cache.refs > 1).sum()) == 0


def test_a_batch_is_what_the_plain_decoder_computes(example):
    w = example.Weights(5)
    server = example.Server(w)
    rng = np.random.default_rng(1)
    prompts = [[int(t) for t in rng.integers(0, example.VOCAB, n)] for n in (23, 2, 37)]
    server.prefill(prompts)
    rows = example.ROWS
    server.grow([rows] * 3)
    new = [[p[-1]] + [int(t) for t in rng.integers(0, example.VOCAB, rows - 1)] for p in prompts]
    got = server.forward(example.i32(new))
    for b, (p, x) in enumerate(zip(prompts, new)):
        want = plain_logits(example, w, p[:-1] + x, b if b < 2 else -1)[-rows:]
        # some tens of BF16 roundings (2^-9 each) on the way through two layers, and a 4-bit element here and there that falls to the
        # other side of a border: as for the cache's example
        assert bool(((got[b] - want).abs() <= 2.0 ** -4 * want.abs().max()).all()), float((got[b] - want).abs().max() / want.abs().max())
        adjusted = mxq.mxq_logits_adjust(got, server.rules[rows], example.i32([x[1:] for x in new]))
    assert bool((adjusted[-1, :, 1::2] == -torch.inf).all()) and bool(adjusted[-1, :, 0::2].isfinite().all())
    assert mxq.mxq_linear_device_status() == 0


def test_steps_in_a_graph(example):
    """A decode step of the batch, captured and replayed on new tokens, leaves what the calls leave."""
    w = example.Weights(6)
    one, two = example.Server(w), example.Server(w)
    prompts = [[1, 2, 3, 4], [5, 6], [8, 8, 8, 8, 8]]
    for s in (one, two):
        s.prefill(prompts)
    tokens = example.i32([[4], [6], [8]])
    for s in (one, two):
        s.grow([1] * 3)
    two.forward(tokens)                     # (warm: workspaces kept for callers that pass none are made)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = two.forward(tokens)
        _, _, following = mxq.mxq_greedy_accept_rules(logits, None, two.rules[1], workspace=two.accept_ws)
    for _ in range(4):
        graph.replay()
        want = one.forward(tokens)
        assert torch.equal(logits, want)
        _, _, n = mxq.mxq_greedy_accept_rules(want, None, one.rules[1], workspace=one.accept_ws)
        assert torch.equal(n, following)
        tokens.copy_(n.view(3, 1))
        for s in (one, two):
            s.grow([1] * 3)
    for layer in range(example.LAYERS):
        a, b = (mxq.mxq_kv_read(s.cache, layer, s.tables, s.lens, 8) for s in (one, two))
        assert torch.equal(a[0][:, :-1], b[0][:, :-1]) and torch.equal(a[1][:, :-1], b[1][:, :-1])
