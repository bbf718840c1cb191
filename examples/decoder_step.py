"""A serving batch on a 4-bit decoder, with what stands between its linear layers and its cache: norms, rotary positions, one
adapter per request, and the requests' rules on the logits.

A small decoder with random weights.  Three requests with prompts of different lengths and adapters of their own (the last has none);
every layer is

    norm (with the residual's addition) -> q, k, v from one MXFP4 projection + adapters -> rotate + append to the 4-bit cache -> attention
    -> output projection -> norm (with the residual's addition) -> gated feed-forward block

and after the last one a norm, the vocabulary projection, and the verification of each request's proposals against the argmax of its
logits after penalties, biases and a grammar's mask.  Proposals come from the request's own history (the tokens that followed its
last token before).  What is accepted is counted, the rest is rolled back.

    python examples/decoder_step.py [rounds]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2503_13565_b200 as mxq

VOCAB, HIDDEN, HEADS, KV_HEADS, HEAD_DIM, FFN, LAYERS, RANK = 1000, 512, 8, 2, 64, 1024, 2, 16
REQUESTS, PROPOSALS, MAX_TOKENS, PAGE = 3, 3, 256, 32
ROWS = 1 + PROPOSALS


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Weights:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
        cast = lambda n, k, std: mxq.mxq_quantize((rn(n, k) * std).bfloat16())
        qkv = (HEADS + 2 * KV_HEADS) * HEAD_DIM
        self.embedding = rn(VOCAB, HIDDEN).bfloat16()
        self.layers = [dict(norm1=(1 + 0.1 * rn(HIDDEN)).bfloat16(), norm2=(1 + 0.1 * rn(HIDDEN)).bfloat16(), qkv=cast(qkv, HIDDEN, 0.05),
                            out=cast(HIDDEN, HEADS * HEAD_DIM, 0.04), gate_up=cast(2 * FFN, HIDDEN, 0.04), down=cast(HIDDEN, FFN, 0.03),
                            a=(rn(REQUESTS - 1, RANK, HIDDEN) * HIDDEN ** -0.5).bfloat16(), b=(rn(REQUESTS - 1, qkv, RANK) * 0.1).bfloat16())
                       for _ in range(LAYERS)]
        self.norm = (1 + 0.1 * rn(HIDDEN)).bfloat16()
        self.head = cast(VOCAB, HIDDEN, 0.08)
        self.scale = torch.tensor([1.0, 0.5], device="cuda")


class Server:
    """REQUESTS sequences with a cache, page tables and rules of their own."""

    def __init__(self, weights):
        self.w = weights
        self.cache = mxq.KVCache.new(LAYERS, 32, KV_HEADS, HEAD_DIM, PAGE)
        self.tables, self.lens = self.cache.new_sequences(REQUESTS, MAX_TOKENS)
        freq = 10000.0 ** (-torch.arange(HEAD_DIM // 2, dtype=torch.float64, device="cuda") * 2 / HEAD_DIM)
        self.rope = mxq.Rope(mxq.mxq_rope_table(freq, MAX_TOKENS))
        self.counts = torch.zeros(REQUESTS, VOCAB, dtype=torch.int32, device="cuda")
        penalties = torch.tensor([[1.0, 0.0, 0.0], [1.2, 0.3, 0.1], [1.0, 0.5, 0.2]], device="cuda")       # repetition, presence, frequency
        bias_tokens, bias_values = i32([[5, 6], [-1, -1], [7, 7]]), torch.tensor([[4.0, -9.0], [0.0, 0.0], [1.0, 2.0]], device="cuda")
        self.allowed = {}
        for rows in (1, ROWS):      # the grammar of the last request never allows odd tokens
            words = torch.full((REQUESTS, rows, (VOCAB + 31) // 32), -1, dtype=torch.int32, device="cuda")
            words[-1] = 0x55555555
            self.allowed[rows] = words
        self.rules = {r: mxq.LogitRules(self.counts, penalties, bias_tokens, bias_values, m) for r, m in self.allowed.items()}
        self.owner = {m: i32([0, 1, -1]).repeat_interleave(m) for m in (1, ROWS)}      # every row's adapter; the last request has none
        self.attention_ws = mxq.new_workspace(max(mxq.mxq_kv_attention_workspace_bytes(REQUESTS, m, HEADS, KV_HEADS, HEAD_DIM) for m in (1, ROWS)))
        self.accept_ws = mxq.new_workspace(mxq.mxq_greedy_accept_rules_workspace_bytes(REQUESTS, ROWS, VOCAB))
        self.linear_ws = mxq.new_workspace(max(mxq.mxq_linear_fused_workspace_bytes(16, n, k) for n, k in ((HIDDEN, HEADS * HEAD_DIM), (2 * FFN, HIDDEN), (HIDDEN, FFN))))

    def forward(self, tokens, rows=None):
        """Logits [REQUESTS, M, VOCAB] of the last rows[b] (None: all M) tokens of every sequence, whose room is there already."""
        b, m = tokens.shape
        h = self.w.embedding[tokens].view(b * m, HIDDEN)               # the residual stream
        update = torch.zeros_like(h)
        for i, lay in enumerate(self.w.layers):
            x = mxq.mxq_rmsnorm(update, lay["norm1"], residual=h, residual_out=h)
            qkv = mxq.mxq_linear_lora(x, *lay["qkv"], lay["a"], lay["b"], self.owner[m], scale=self.w.scale, out_dtype=torch.bfloat16)
            qkv = qkv.view(b, m, HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV_HEADS], qkv[:, :, HEADS + KV_HEADS:]     # slices, no copies
            q = mxq.mxq_kv_append_rope(self.cache, i, q, k, v, self.tables, self.lens, self.rope, rows=rows)
            a = mxq.mxq_kv_attention(q, self.cache, i, self.tables, self.lens, rows=rows, workspace=self.attention_ws)
            update = mxq.mxq_linear(a.view(b * m, HEADS * HEAD_DIM), *lay["out"])                             # FP32, straight into the norm
            x = mxq.mxq_rmsnorm(update, lay["norm2"], residual=h, residual_out=h)
            act = mxq.mxq_linear_swiglu(x, *lay["gate_up"], workspace=self.linear_ws)
            update = mxq.mxq_linear(act, *lay["down"])
        x = mxq.mxq_rmsnorm(update, self.w.norm, residual=h)
        return mxq.mxq_linear(x, *self.w.head).view(b, m, VOCAB)

    def grow(self, by):
        mxq.mxq_kv_resize(self.cache, self.tables, self.lens, self.lens + i32(by))

    def prefill(self, prompts):
        """All tokens of the prompts but the last, a few rows at a time; the prompts are marked in the counts."""
        longest = max(len(p) for p in prompts)
        padded = i32([list(p) + [0] * (longest - len(p)) for p in prompts])
        mxq.mxq_token_counts(self.counts, padded, i32([len(p) for p in prompts]), prompt=True)
        for at in range(0, longest - 1, ROWS):
            part = [list(p[at:min(at + ROWS, len(p) - 1)]) for p in prompts]
            self.grow([len(x) for x in part])
            self.forward(i32([x + [0] * (ROWS - len(x)) for x in part]), rows=i32([len(x) for x in part]))

    def step(self, last, proposals):
        """One verification: last [REQUESTS] and proposals [REQUESTS][PROPOSALS]; returns (accepted, next token) per request."""
        draft = i32(proposals)
        self.grow([ROWS] * REQUESTS)
        logits = self.forward(torch.cat([i32(last).view(-1, 1), draft], 1))
        _, accepted, following = mxq.mxq_greedy_accept_rules(logits, draft, self.rules[ROWS], workspace=self.accept_ws)
        mxq.mxq_token_counts(self.counts, draft, accepted, next_token=following)
        mxq.mxq_kv_resize(self.cache, self.tables, self.lens, self.lens - (PROPOSALS - accepted))
        return accepted.tolist(), following.tolist()


def propose(history):
    """What followed the last token before, or the last token again."""
    for i in range(len(history) - 2, -1, -1):
        if history[i] == history[-1]:
            return (history[i + 1:i + 1 + PROPOSALS] + [history[-1]] * PROPOSALS)[:PROPOSALS]
    return [history[-1]] * PROPOSALS


def main(rounds=12):
    server = Server(Weights())
    prompts = [[3, 14, 15, 9, 26, 5], [100, 200, 300], [42, 17, 42, 17, 42, 17, 42, 17, 42]]
    server.prefill(prompts)
    streams = [list(p) for p in prompts]
    taken = 0
    for _ in range(rounds):
        proposals = [propose(s) for s in streams]
        accepted, following = server.step([s[-1] for s in streams], proposals)
        for s, p, n, t in zip(streams, proposals, accepted, following):
            s += p[:n] + [t]
            taken += n
    torch.cuda.synchronize()
    assert mxq.mxq_linear_device_status() == 0
    made = [s[len(p):] for s, p in zip(streams, prompts)]
    assert all(t % 2 == 0 for t in made[-1]), "the grammar allows even tokens only"
    print("%d rounds: %s tokens, %d of %d proposals accepted" % (rounds, [len(m) for m in made], taken, rounds * REQUESTS * PROPOSALS))
    return server, prompts, streams


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 12)
