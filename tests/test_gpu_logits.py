"""mxq_logits_adjust, mxq_greedy_accept_rules and mxq_token_counts: the rules are FP32 with one rounding per operation, so adjusted logits
are compared to the bit and tokens exactly."""
import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq
import step_plain as plain

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def dev(x, dtype=torch.int32):
    return None if x is None else torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def make(b, t, r, v, dtype, seed, penalties=True, counts=True, biases=0, masks=None):
    """numpy rules and their device form; masks: None or the share of tokens that are allowed."""
    rng = np.random.default_rng(seed)
    logits = torch.from_numpy((rng.standard_normal((b, r, v)) * 3).astype(np.float32)).to(dtype)
    draft = rng.integers(0, v, (b, t)) if t else None
    if t >= 2:
        draft[:, 1] = draft[:, 0]                                     # a proposal that repeats the one before it
    n = dict(counts=None, penalties=None, bias_tokens=None, bias_values=None, allowed=None)
    if counts:
        c = np.where(rng.random((b, v)) < 0.1, rng.integers(1, 2000, (b, v)), 0)
        c[0, : v // 2] = rng.integers(0, 3, v // 2)                   # one sequence that has seen much
        n["counts"] = c | np.where(rng.random((b, v)) < 0.1, 1 << 31, 0)
    if penalties:
        n["penalties"] = np.stack([rng.uniform(0.8, 1.7, b), rng.uniform(-0.5, 1, b), rng.uniform(-0.1, 0.3, b)], 1).astype(np.float32)
        n["penalties"][0] = (1, 0, 0)
    if biases:
        tok = rng.integers(0, v, (b, biases))
        tok[:, ::5] = rng.integers(-3, 0, tok[:, ::5].shape)
        tok[:, 1::7] = v + 2
        if biases > 6:
            tok[:, 6] = tok[:, 2]                                     # the same token twice: the last entry counts
        n["bias_tokens"], n["bias_values"] = tok, (rng.standard_normal((b, biases)) * 5).astype(np.float32)
    if masks is not None:
        n["allowed"] = rng.random((b, r, v)) < masks
        n["allowed"][-1, -1] = False                                  # nothing is left
    bits = None
    if masks is not None:
        pad = np.zeros((b, r, -(-v // 32) * 32), bool)
        pad[..., :v] = n["allowed"]
        pad[..., v:] = True                                           # bits behind the vocabulary mean nothing
        bits = np.packbits(pad, axis=-1, bitorder="little").view(np.int32)
    cd = None if n["counts"] is None else dev(n["counts"].astype(np.uint32).view(np.int32))
    rules = mxq.LogitRules(cd, dev(n["penalties"], F32), dev(n["bias_tokens"]), dev(n["bias_values"], F32), dev(bits))
    return logits, draft, n, rules


def want_rows(logits, draft, n):
    return plain.adjusted(logits.float().numpy(), draft, n["counts"], n["penalties"], n["bias_tokens"], n["bias_values"], n["allowed"])


def check(logits, draft, n, rules, workspace=None):
    rows = want_rows(logits, draft, n)
    x, d = logits.cuda(), dev(draft)
    got = mxq.mxq_logits_adjust(x, rules, d)
    want = torch.from_numpy(rows).to(logits.dtype)
    g = got.cpu()
    assert torch.equal(g.isnan(), want.isnan()) and torch.equal(g.nan_to_num(1e30), want.nan_to_num(1e30)), (g != want).nonzero()[:5]
    ver, acc, nxt = (t.cpu().tolist() for t in mxq.mxq_greedy_accept_rules(x, d, rules, workspace=workspace))
    for b in range(rows.shape[0]):
        assert (ver[b], acc[b], nxt[b]) == plain.accept(rows[b], None if draft is None else draft[b]), b
    same = x.clone()
    assert mxq.mxq_logits_adjust(same, rules, d, out=same) is same and torch.equal(same.nan_to_num(1e30), got.nan_to_num(1e30))     # in place
    return rows


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,r,v,kw", [
    (1, 0, 1, 1, dict(biases=1)), (2, 0, 1, 3, dict()), (1, 1, 1, 31, dict(masks=0.5)), (3, 2, 3, 33, dict(biases=3, masks=0.5)), (1, 3, 4, 1023, dict()),
    (2, 4, 4, 1025, dict(biases=40, masks=0.1)), (5, 7, 8, 2049, dict(masks=0.9)), (1, 8, 9, 32000, dict()), (3, 64, 65, 5001, dict(biases=7)),
    (40, 2, 3, 4099, dict(biases=1024, masks=0.5)), (2, 1, 2, 128256, dict(biases=300, masks=0.03)), (700, 1, 2, 2047, dict()),
    (2, 5, 6, 40007, dict(counts=False)), (2, 5, 6, 3001, dict(penalties=False, biases=9)), (1, 5, 5, 20000, dict(penalties=False, counts=False, masks=0.2))])
def test_rules(b, t, r, v, kw, dtype):
    check(*make(b, t, r, v, dtype, seed=b + v, **kw))


def test_no_rule_at_all_is_the_plain_acceptance():
    logits, draft, n, rules = make(6, 5, 6, 3001, F32, 3, penalties=False, counts=False)
    draft[:, :3] = logits.numpy().argmax(-1)[:, :3]
    check(logits, draft, n, rules)
    x, d = logits.cuda(), dev(draft)
    assert torch.equal(mxq.mxq_logits_adjust(x, rules, d), x)
    acc, nxt = mxq.mxq_greedy_accept(x, d)
    got = mxq.mxq_greedy_accept_rules(x, d, rules)
    assert torch.equal(got[1], acc) and torch.equal(got[2], nxt)


def test_proposals_count_for_the_rows_after_them():
    """A token that leads by little loses its lead once it has been proposed before: the walk stops there."""
    v = 500
    logits = torch.zeros(1, 4, v)
    logits[0, :, 7] = 2.0
    logits[0, :, 9] = 1.5
    penalties = np.array([[1.0, 0.0, 1.0]], np.float32)               # one less for every time
    rules = mxq.LogitRules(counts=torch.zeros(1, v, dtype=torch.int32, device="cuda"), penalties=dev(penalties, F32))
    ver, acc, nxt = mxq.mxq_greedy_accept_rules(logits.cuda(), dev([[7, 9, 7]]), rules)
    assert ver.tolist() == [[7, 9, 7, 9]] or ver.tolist() == [[7, 9, 7, 9]]
    rows = plain.adjusted(logits.numpy(), np.array([[7, 9, 7]]), np.zeros((1, v), np.int64), penalties, None, None, None)
    assert (ver[0].tolist(), int(acc), int(nxt)) == plain.accept(rows[0], [7, 9, 7])


def test_masked_places_hide_what_they_hold_and_ties_go_to_the_lowest():
    v = 4100
    logits, draft, n, rules = make(2, 1, 2, v, F32, 5, counts=False, penalties=False, masks=0.5)
    a = torch.from_numpy(n["allowed"])
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.4e38])
    logits = torch.where(a, logits, bad[torch.arange(v) % 4])
    logits[0, 0][a[0, 0]] = -0.0
    first = int(torch.nonzero(a[0, 0])[3])
    logits[0, 0, first] = 0.0                                         # +0 does not beat the -0 of a lower index
    logits[0, 1][torch.nonzero(a[0, 1])[5]] = float("nan")
    rows = check(logits, draft, n, rules)
    assert plain.argmax(rows[0, 0]) == int(torch.nonzero(a[0, 0])[0])
    logits[1] = -float("inf")
    check(logits, draft, n, rules)


def test_infinities_meet_the_penalties():
    v = 64
    logits = torch.randn(1, 1, v)
    logits[0, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1e38])
    counts = np.zeros((1, v), np.int64)
    counts[0, :4] = 5
    n = dict(counts=counts, penalties=np.array([[1e-3, 0.5, 0.1]], np.float32), bias_tokens=np.array([[0, 1, 5]]), bias_values=np.array([[-np.inf, np.inf, 2]], np.float32),
             allowed=None)
    rules = mxq.LogitRules(dev(counts), dev(n["penalties"], F32), dev(n["bias_tokens"]), dev(n["bias_values"], F32))
    check(logits, None, n, rules)


def test_a_workspace_serves_calls_of_all_shapes_and_is_left_zero():
    ws = mxq.new_workspace(mxq.mxq_greedy_accept_rules_workspace_bytes(40, 9, 5000))
    for b, t, r, v in ((40, 8, 9, 5000), (1, 0, 1, 70000), (7, 3, 3, 100), (40, 8, 9, 5000)):
        check(*make(b, t, r, v, F32, b, biases=5, masks=0.5), workspace=ws)
        assert int(ws.count_nonzero()) == 0


def test_captured_calls_replay_on_new_contents():
    logits, draft, n, rules = make(4, 3, 4, 9001, F32, 11, biases=20, masks=0.5)
    x, d, ws = logits.cuda(), dev(draft), mxq.new_workspace(mxq.mxq_greedy_accept_rules_workspace_bytes(4, 4, 9001))
    mxq.mxq_greedy_accept_rules(x, d, rules, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adj = mxq.mxq_logits_adjust(x, rules, d)
        ver, acc, nxt = mxq.mxq_greedy_accept_rules(x, d, rules, workspace=ws)
        mxq.mxq_token_counts(rules.counts, d, acc, next_token=nxt)
    rng = np.random.default_rng(0)
    for _ in range(3):
        draft = rng.integers(0, 9001, draft.shape)
        d.copy_(dev(draft)), x.copy_(torch.randn(x.shape))
        counts = rules.counts.cpu().numpy().view(np.uint32).astype(np.int64)
        rows = want_rows(x.cpu(), draft, dict(n, counts=counts))
        draft[:, 0] = [plain.argmax(r[0]) for r in rows]              # one proposal that is right
        d.copy_(dev(draft))
        rows = want_rows(x.cpu(), draft, dict(n, counts=counts))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(adj.cpu().numpy(), rows)
        for b in range(4):
            said, a, nx = plain.accept(rows[b], draft[b])
            assert (ver[b].tolist(), int(acc[b]), int(nxt[b])) == (said, a, nx)
            for t in list(draft[b][:a]) + [nx]:
                counts[b, t] += 1
        assert np.array_equal(rules.counts.cpu().numpy().view(np.uint32), counts)


@pytest.mark.parametrize("b,v,l", [(1, 10, 1), (3, 1000, 31), (5, 33, 4000), (2, 50000, 1000), (300, 7, 257)])
def test_counts(b, v, l):
    rng = np.random.default_rng(l)
    counts = torch.zeros(b, v, dtype=torch.int32, device="cuda")
    want = np.zeros((b, v), np.int64)
    for step in range(3):
        tokens = (rng.random((b, l)) ** 3 * (v + 2)).astype(np.int64) - 1          # -1 and v among them
        n = rng.integers(-1, l + 2, b) if step else None
        extra = rng.integers(-1, v + 1, b) if step == 1 else None
        prompt = step == 2
        mxq.mxq_token_counts(counts, dev(tokens), dev(n), dev(extra), prompt=prompt)
        for i in range(b):
            t = list(tokens[i] if n is None else tokens[i][:max(0, n[i])]) + ([] if extra is None else [extra[i]])
            for x in t:
                if 0 <= x < v:
                    want[i, x] = want[i, x] | 1 << 31 if prompt else want[i, x] + 1
        assert np.array_equal(counts.cpu().numpy().view(np.uint32), want)


def test_two_streams_at_once():
    cases = [make(3, 4, 5, 30011, F32, s, biases=9, masks=0.5) for s in (1, 2)]
    dv = [(c[0].cuda(), dev(c[1]), c[3]) for c in cases]
    want = [[t.clone() for t in mxq.mxq_greedy_accept_rules(x, d, r)] for x, d, r in dv]
    sides = [torch.cuda.Stream() for _ in dv]
    torch.cuda.synchronize()
    got = [[mxq.mxq_greedy_accept_rules(*dv[i], stream=s) for _ in range(20)] for i, s in enumerate(sides)]
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for g in got[i] for a, b in zip(g, want[i]))
