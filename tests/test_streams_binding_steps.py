"""What the binding allocates for the norm, the rotated append, the rules and the adapters on a given stream belongs to that stream (as in
tests/test_streams_binding.py; on the host, with the library and the stream context replaced by recorders)."""
import types

import pytest
import torch

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import binding
from test_streams_binding import STREAM, cache, record  # noqa: F401

BF, I = torch.bfloat16, torch.int32
RULES = types.SimpleNamespace(fit=lambda b, r, v: 0)


def rope(s):
    c, tables, lens = cache()
    mxq.mxq_kv_append_rope(c, 0, Q, KV, KV, tables, lens, types.SimpleNamespace(ptr=0), stream=s)


X, R, W = torch.ones(3, 64, dtype=BF), torch.ones(3, 64), torch.ones(64)
C8, S8, F64, LOGITS, BASE = torch.zeros(3, 64, dtype=torch.uint8), torch.zeros(3, 2, dtype=torch.uint8), torch.ones(8, dtype=torch.float64), torch.ones(2, 1, 50), torch.ones(3, 10)
W4 = (torch.zeros(10, 32, dtype=torch.uint8), torch.zeros(10, 2, dtype=torch.uint8))
Q, KV = torch.ones(3, 1, 4, 64, dtype=BF), torch.ones(3, 1, 2, 64)
AD = (torch.ones(2, 8, 64, dtype=BF), torch.ones(2, 10, 8, dtype=BF), torch.zeros(3, dtype=I))
CALLS = {
    "rmsnorm": lambda s: mxq.mxq_rmsnorm(X, W, stream=s),
    "rmsnorm of FP32 rows": lambda s: mxq.mxq_rmsnorm(R, W, residual=R, stream=s),
    "rmsnorm, both outputs": lambda s: mxq.mxq_rmsnorm(X, W, residual=X, mxfp8=True, stream=s),
    "dequantize_mxfp8": lambda s: mxq.mxq_dequantize_mxfp8(C8, S8, stream=s),
    "rope_table": lambda s: mxq.mxq_rope_table(F64, 5, stream=s),
    "kv_append_rope": rope,
    "logits_adjust": lambda s: mxq.mxq_logits_adjust(LOGITS, RULES, stream=s),
    "greedy_accept_rules": lambda s: mxq.mxq_greedy_accept_rules(LOGITS, None, RULES, stream=s),
    "lora": lambda s: mxq.mxq_lora(X, *AD, stream=s),
    "lora beside a base": lambda s: mxq.mxq_lora(X, *AD, base=BASE, stream=s),
    "linear_lora": lambda s: mxq.mxq_linear_lora(X, *W4, *AD, stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_calls_allocate_on_the_stream_they_run_on(name, record, monkeypatch):  # noqa: F811
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype, shape, what: t.data_ptr())
    for t in (X, R):
        monkeypatch.setattr(type(t), "is_cuda", property(lambda self: True), raising=False)
    CALLS[name](STREAM)
    assert record.launches == [77] and record.made and set(record.made) == {77}
    record.made.clear()
    CALLS[name](None)
    assert record.launches == [77, None] and record.made and set(record.made) == {None}
