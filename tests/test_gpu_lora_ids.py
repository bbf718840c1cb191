"""The owners of rows (ids) are a step's data: whatever ran before a call in its stream may have written them, a kernel of this library that
has let the next one start early among them."""
import pytest
import torch

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import synth

pytestmark = pytest.mark.gpu

N, K, RANK, COUNT, V = 520, 256, 24, 20, 60000


def bits(t):
    return t.view(torch.int32)


def tensors(m, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return g, rn(m, K).bfloat16(), (rn(COUNT, RANK, K) / K ** 0.5).bfloat16(), rn(COUNT, N, RANK).bfloat16(), rn(COUNT), rn(m, N)


def calls(m, seed):
    """mxq_lora, and for few rows mxq_linear_lora, as functions of (ids, out)."""
    g, x, a, b, scale, base = tensors(m, seed)
    ws = torch.zeros(mxq.mxq_lora_workspace_bytes(m, N, K, RANK, COUNT), dtype=torch.uint8, device="cuda")
    out = {"lora": lambda ids, y: mxq.mxq_lora(x, a, b, ids, scale=scale, base=base, out=y, workspace=ws)}
    if m <= 16:
        w = mxq.mxq_quantize(synth.normal_bf16((N, K), 0.05, seed).cuda())
        lws = torch.zeros(mxq.mxq_linear_lora_workspace_bytes(m, N, K, RANK, COUNT), dtype=torch.uint8, device="cuda")
        out["linear_lora"] = lambda ids, y: mxq.mxq_linear_lora(x, *w, a, b, ids, scale=scale, out=y, workspace=lws)
    return g, out


@pytest.mark.parametrize("loaded", [COUNT, 2])
@pytest.mark.parametrize("m", [1, 7, 16, 40, 130, 300, 700])
def test_owners_that_the_call_before_has_chosen(m, loaded):
    """The argmax of the logits under the rules is the owner: a long kernel, behind which the next one waits, writes it last."""
    g, run = calls(m, m)
    logits = torch.zeros(4, m, 1, V, device="cuda")
    owners = torch.randint(0, loaded, (4, m), generator=g, device="cuda")
    owners[torch.rand(4, m, generator=g, device="cuda") < 0.2] = V - 5                # no adapter
    logits.view(4, m, V).scatter_(2, owners.unsqueeze(-1), 1.0)
    rules = mxq.LogitRules()
    ids = torch.full((m,), -1, dtype=torch.int32, device="cuda")
    verdict = (ids.view(m, 1), torch.empty_like(ids), torch.empty_like(ids))
    ws = mxq.new_workspace(mxq.mxq_greedy_accept_rules_workspace_bytes(m, 1, V))
    for call in run.values():
        want = []
        for i in range(4):
            y = torch.empty(m, N, device="cuda")
            call(owners[i].int(), y)
            torch.cuda.synchronize()
            want.append(y)
        out = [torch.zeros(m, N, device="cuda") for _ in range(24)]
        torch.cuda.synchronize()
        for i, y in enumerate(out):
            mxq.mxq_greedy_accept_rules(logits[i % 4], None, rules, workspace=ws, out=verdict)
            call(ids, y)
        for i, y in enumerate(out):
            assert torch.equal(bits(y), bits(want[i % 4])), i
        ids.fill_(-1)
    assert mxq.mxq_linear_device_status() == 0


@pytest.mark.parametrize("between", [False, True])
@pytest.mark.parametrize("m", [1, 16, 64, 400, 511, 600, 1700])
def test_owners_from_an_operation_right_before_the_call(m, between):
    """... or right before a norm ahead of the call."""
    g, run = calls(m, m)
    owners = torch.randint(-1, COUNT + 1, (60, m), generator=g, device="cuda").int()
    h, weight, y8 = torch.randn(m, K, generator=g, device="cuda").bfloat16(), torch.ones(K, device="cuda"), torch.empty(m, K, device="cuda").bfloat16()
    for call in run.values():
        want = torch.empty(len(owners), m, N, device="cuda")
        for o, y in zip(owners, want):
            torch.cuda.synchronize()
            call(o, y)
        torch.cuda.synchronize()
        ids, out = torch.empty(m, dtype=torch.int32, device="cuda"), torch.zeros_like(want)
        for o, y in zip(owners, out):
            torch.add(o, 0, out=ids)
            if between:
                mxq.mxq_rmsnorm(h, weight, out=y8)
            call(ids, y)
        assert torch.equal(bits(out), bits(want))
