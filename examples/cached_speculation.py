"""Speculative decoding with a 4-bit key/value cache, end to end on the library's kernels.

A small decoder with random weights: per layer q, k, v from one fused MXFP4 projection, attention over the cache, the output
projection with the residual in its epilogue, a gated feed-forward block; MXFP4 vocabulary projection fused with the
verification.  (Norms and rotary positions are left out here; examples/decoder_step.py has them.)
The draft is the model's first layer; both keep their own cache.  What is shown:

  decode    specdec.decode drives both: mxq_kv_resize makes room before a pass and rolls back what was not accepted,
            mxq_kv_append and mxq_kv_attention serve one row (drafting) and several (verification)
  branch    one sequence forks into three (mxq_kv_fork shares its full pages and copies the last), each goes its own way,
            and two are freed again
  tree      a token tree of two branches verified in ONE pass with ancestor masks; mxq_kv_compact leaves the accepted path

    python examples/cached_speculation.py [tokens]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import specdec

VOCAB, HIDDEN, HEADS, KV_HEADS, HEAD_DIM, FFN, LAYERS = 2000, 768, 12, 4, 64, 2048, 3
MAX_TOKENS, PAGE, SLOTS = 512, 32, 4


def cast(gen, rows, cols, std):
    return mxq.mxq_quantize((torch.randn(rows, cols, generator=gen, device="cuda") * std).to(torch.bfloat16))


class Weights:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.embedding = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda").to(torch.bfloat16)
        self.layers = []
        for i in range(LAYERS):
            add = 1.0 if i == 0 else 0.1      # (later layers change less, so that a draft of one layer is right now and then)
            self.layers.append(dict(qkv=cast(g, (HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN, 0.05), out=cast(g, HIDDEN, HEADS * HEAD_DIM, 0.03 * add),
                                    gate_up=cast(g, 2 * FFN, HIDDEN, 0.03), down=cast(g, HIDDEN, FFN, 0.02 * add)))
        self.head = cast(g, VOCAB, HIDDEN, 0.05)


class CachedModel:
    """The first `layers` layers with a cache of their own: slot 0 decodes, the other slots are for branches."""

    def __init__(self, weights, layers):
        self.w, self.layers = weights, layers
        self.cache = mxq.KVCache.new(layers, 64, KV_HEADS, HEAD_DIM, PAGE)
        self.tables, self.lens = self.cache.new_sequences(SLOTS, MAX_TOKENS)
        self.workspace = mxq.new_workspace(max(mxq.mxq_kv_attention_workspace_bytes(1, m, HEADS, KV_HEADS, HEAD_DIM) for m in (1, 16)))
        self.linear_ws = mxq.new_workspace(max(mxq.mxq_linear_fused_workspace_bytes(16, n, k) for n, k in
                                               ((HIDDEN, HEADS * HEAD_DIM), (2 * FFN, HIDDEN), (HIDDEN, FFN))))
        self.head_ws = {}

    def lengths(self, slot, tokens):
        """New lengths with `slot` at `tokens` and the others as they are."""
        new = self.lens.clone()
        new[slot] = tokens
        return new

    def resize(self, slot, tokens):
        mxq.mxq_kv_resize(self.cache, self.tables, self.lens, self.lengths(slot, tokens))

    def forward(self, tokens, slot=0, tree=None):
        """Hidden states of the last len(tokens) positions of the slot, whose room is there already."""
        rows = len(tokens)
        h = self.w.embedding[torch.tensor(tokens, device="cuda")]
        tables, lens = self.tables[slot:slot + 1], self.lens[slot:slot + 1]
        for i in range(self.layers):
            lay = self.w.layers[i]
            qkv = mxq.mxq_linear(h, *lay["qkv"], out_dtype=torch.bfloat16).view(1, rows, HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV_HEADS], qkv[:, :, HEADS + KV_HEADS:]      # slices, no copies
            mxq.mxq_kv_append(self.cache, i, k, v, tables, lens)
            a = mxq.mxq_kv_attention(q, self.cache, i, tables, lens, tree=tree, workspace=self.workspace)
            h = mxq.mxq_linear_residual(a.view(rows, HEADS * HEAD_DIM), *lay["out"], residual=h, workspace=self.linear_ws)
            act = mxq.mxq_linear_swiglu(h, *lay["gate_up"], workspace=self.linear_ws)
            h = mxq.mxq_linear_residual(act, *lay["down"], residual=h, workspace=self.linear_ws)
        return h

    def tokens(self, h, draft=None):
        """(the model's own token after every row, accepted proposals, next token)"""
        r = h.shape[0]
        if r not in self.head_ws:
            self.head_ws[r] = mxq.new_workspace(mxq.mxq_lm_head_accept_workspace_bytes(r, VOCAB, HIDDEN))
        d = None if draft is None else torch.tensor(draft, dtype=torch.int32, device="cuda")
        return mxq.mxq_lm_head_accept(h, *self.w.head, d, workspace=self.head_ws[r])

    # the interface of specdec.decode: `pos` tokens are settled, so whatever the cache holds behind them is rolled back
    def next(self, cur, pos):
        self.resize(0, pos + 1)
        return int(self.tokens(self.forward([cur]))[2])

    def verify(self, cur, pos, proposals):
        self.resize(0, pos + 1 + len(proposals))
        _, accepted, following = self.tokens(self.forward([cur] + list(proposals)), list(proposals))
        return int(accepted), int(following)


def branch(model):
    """Slot 0 forks into slots 1 to 3; every child takes another token and its own argmax; children 2 and 3 are freed."""
    n = int(model.lens[0])
    src, dst = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 0, 0], [1, 2, 3]))
    mxq.mxq_kv_fork(model.cache, model.tables, model.lens, src, dst)
    out = []
    for slot, token in ((1, 11), (2, 12), (3, 13)):
        model.resize(slot, n + 1)
        out.append(int(model.tokens(model.forward([token], slot))[2]))
    shared = int((model.cache.refs > 1).sum())
    for slot in (2, 3):
        model.resize(slot, 0)
    return out, shared


def tree(model, cur):
    """Root `cur` (the settled token) and two branches of two tokens, verified in one pass; the longer accepted path stays."""
    first = model.lens[0].clone()
    # row 0: root; rows 1, 2: first tokens of the branches; rows 3, 4: second tokens
    parent = [-1, 0, 0, 1, 2]
    n = int(first)
    model.resize(0, n + 1)
    own = int(model.tokens(model.forward([cur]))[2])                 # what the model itself says next: branch 0 starts with it
    model.resize(0, n)
    rows = [cur, own, (own + 1) % VOCAB, (own + 2) % VOCAB, (own + 3) % VOCAB]
    masks = []
    for i, p in enumerate(parent):
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
    model.resize(0, n + len(rows))
    hidden = model.forward(rows, tree=torch.tensor([masks], dtype=torch.int64, device="cuda"))
    said = model.tokens(hidden, [0] * (len(rows) - 1))[0].tolist()   # (only the token after every row is used, not the walk over a chain)
    path = [0]
    while True:                                                      # walk down as long as a child is what the model said
        step = [i for i in range(len(rows)) if parent[i] == path[-1] and rows[i] == said[path[-1]]]
        if not step:
            break
        path.append(step[0])
    keep = torch.tensor([path + [0] * (len(rows) - len(path))], dtype=torch.int32, device="cuda")
    kept = torch.tensor([len(path)], dtype=torch.int32, device="cuda")
    new = mxq.mxq_kv_compact(model.cache, model.tables[:1], model.lens[:1], None, keep, kept)
    model.resize(0, int(new))
    return [rows[i] for i in path], said[path[-1]]


def main(tokens=48):
    weights = Weights()
    target, draft = CachedModel(weights, LAYERS), CachedModel(weights, 1)
    stream, tally = specdec.decode([target, draft], [4], first_token=7, tokens=tokens)
    print("decoded %d tokens with %d target passes and %d draft steps, %d of %d proposals accepted" %
          (len(stream), tally.steps[0], tally.steps[1], tally.accepted[0], tally.proposed[0]))
    children, shared = branch(target)
    print("three children of one sequence go on with %s; %d pages were shared" % (children, shared))
    path, following = tree(target, stream[-1])
    print("a tree of five tokens: %d accepted, next token %d" % (len(path), following))
    free = [0] * SLOTS
    for m in (target, draft):
        mxq.mxq_kv_resize(m.cache, m.tables, m.lens, torch.tensor(free, dtype=torch.int32, device="cuda"))
        assert int(m.cache.refs.abs().sum()) == 0
    assert mxq.mxq_linear_device_status() == 0
    return stream, tally, shared, path


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 48)
