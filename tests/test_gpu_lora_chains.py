"""mxq_lora calls one after another in a stream, without a synchronisation between them: what a call leaves for its own later kernels (the
plan of sorted rows, partial sums, fragments) is read only when it is there.  Every call has other rows and owners, and all share one
workspace, so that whatever is read too early belongs to another call and shows."""
import random

import pytest
import torch

import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu

N, K, RANK, COUNT, MOST = 136, 256, 24, 30, 1300


def rows_of_calls(seed, calls=200):
    """Mostly 17 to 511 rows; some few and some many between them, which write other things to the same places of the workspace."""
    rng = random.Random(seed)
    return [rng.choice([rng.randint(1, 16), rng.randint(512, MOST)]) if i % 5 == 4 else rng.randint(17, 511) for i in range(calls)]


def tensors(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, a, b = rn(MOST, K).bfloat16(), (rn(COUNT, RANK, K) / K ** 0.5).bfloat16(), rn(COUNT, N, RANK).bfloat16()
    return g, x, a, b, rn(MOST, N)


def workspace(rows, loaded):
    return torch.zeros(max(mxq.mxq_lora_workspace_bytes(m, N, K, RANK, n) for m in rows for n in loaded), dtype=torch.uint8, device="cuda")


def bits(t):
    return t.view(torch.int32)


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_calls_of_other_rows_and_owners_one_after_another(seed):
    rows = rows_of_calls(seed)
    g, x, a, b, base = tensors(seed)
    loaded = [random.Random(m).choice([1, 4, COUNT]) for m in rows]
    owners = [torch.randint(-1, n + 1, (m,), generator=g, device="cuda").int() for m, n in zip(rows, loaded)]
    ws = workspace(rows, set(loaded))
    out = [torch.empty(m, N, device="cuda") for m in rows]

    def call(i, y):
        m, n = rows[i], loaded[i]
        mxq.mxq_lora(x[:m], a[:n], b[:n], owners[i], base=base[:m], out=y, workspace=ws)

    want = [torch.empty_like(y) for y in out]
    for i, y in enumerate(want):
        torch.cuda.synchronize()
        call(i, y)
    torch.cuda.synchronize()
    for _ in range(3):
        for y in out:
            y.zero_()
        torch.cuda.synchronize()
        for i, y in enumerate(out):
            call(i, y)
        for i, (y, w) in enumerate(zip(out, want)):
            assert torch.equal(bits(y), bits(w)), (i, rows[i], loaded[i])
    assert mxq.mxq_linear_device_status() == 0


@pytest.mark.parametrize("m", [17, 64, 400, 511, 600])
def test_a_captured_chain(m):
    """Three calls of other owners in a graph, replayed with new rows and owners."""
    g, x, a, b, base = tensors(m)
    ws = workspace([m], [COUNT])
    x, base = x[:m].clone(), base[:m]
    ids = [torch.zeros(m, dtype=torch.int32, device="cuda") for _ in range(3)]
    out = [torch.empty(m, N, device="cuda") for _ in ids]
    run = lambda: [mxq.mxq_lora(x, a, b, i, base=base, out=y, workspace=ws) for i, y in zip(ids, out)]
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        x.copy_(torch.randn(m, K, generator=g, device="cuda"))
        for i in ids:
            i.copy_(torch.randint(-1, COUNT + 1, (m,), generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, y in zip(ids, out):
            assert torch.equal(bits(y), bits(mxq.mxq_lora(x, a, b, i, base=base)))
