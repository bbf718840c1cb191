"""What the binding allocates for a call on a given stream belongs to that stream: its zero fill runs there, before the call's kernel,
and its memory is not handed to work on another stream while the kernel runs.  On the host, with the library and the stream context
replaced by recorders; tests/test_gpu_streams.py runs the calls."""
import contextlib
import types

import pytest
import torch

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import binding

STREAM = types.SimpleNamespace(cuda_stream=77)


class FakeLibrary:
    def __init__(self, launches):
        self.launches = launches

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 4096
            self.launches.append(args[-1])
            return 0
        return call


@pytest.fixture()
def record(monkeypatch):
    """(allocations, launches): the stream each was made on (None: the current one)"""
    state = types.SimpleNamespace(on=None, made=[], launches=[])
    fake = FakeLibrary(state.launches)
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(binding, "_dev", lambda t, dtype, what: t.data_ptr())
    monkeypatch.setattr(binding, "_token_rows", lambda t, shape, what: (t.data_ptr(), 1))
    monkeypatch.setattr(binding, "_stream", lambda s=None: None if s is None else s.cuda_stream)
    monkeypatch.setattr(binding, "_default_ws", {})
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    @contextlib.contextmanager
    def stream(s):
        before, state.on = state.on, None if s is None else s.cuda_stream
        yield
        state.on = before

    monkeypatch.setattr(torch.cuda, "stream", stream)
    for name in ("empty", "zeros", "empty_like", "full"):
        def wrapped(*a, _make=getattr(torch, name), **kw):
            state.made.append(state.on)
            return _make(*a, **kw)
        monkeypatch.setattr(torch, name, wrapped)
    return state


def cache():
    c = types.SimpleNamespace(ptr=0, kv_heads=2, head_dim=64)
    tables, lens = torch.tensor([[0, 1]] * 3, dtype=torch.int32), torch.tensor([5, 6, 7], dtype=torch.int32)
    return c, tables, lens


def kv_attention(stream):
    c, tables, lens = cache()
    mxq.mxq_kv_attention(torch.ones(3, 1, 4, 64), c, 0, tables, lens, with_lse=True, stream=stream)


def kv_read(stream):
    c, tables, lens = cache()
    mxq.mxq_kv_read(c, 0, tables, lens, 2, stream=stream)


def kv_fork(stream):
    c, tables, lens = cache()
    mxq.mxq_kv_fork(c, tables, lens, lens[:1], lens[1:2], stream=stream)


def kv_compact(stream):
    c, tables, lens = cache()
    mxq.mxq_kv_compact(c, tables, lens, None, tables, lens, stream=stream)


KV = [kv_attention, kv_read, kv_fork, kv_compact]


@pytest.mark.parametrize("call", KV)
def test_cache_calls_allocate_on_the_stream_they_run_on(call, record):
    call(STREAM)
    assert record.launches == [77] and record.made and set(record.made) == {77}
    record.made.clear()
    call(None)
    assert record.launches == [77, None] and record.made and set(record.made) == {None}


W, X = (torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8)), torch.ones(3, 64, dtype=torch.bfloat16)
Y, BIG, LOGITS, DRAFT, TOKENS = torch.ones(3, 8), torch.ones(1000), torch.ones(2, 4, 100), torch.ones(2, 3), torch.ones(2, 4)
LAYERS = {
    "quantize": lambda s: mxq.mxq_quantize(X, stream=s),
    "dequantize": lambda s: mxq.mxq_dequantize(*W, stream=s),
    "linear": lambda s: mxq.mxq_linear(X, *W, stream=s),
    "linear_host": lambda s: mxq.mxq_linear_host(X, *W, Y, BIG, BIG, stream=s),
    "linear_bf16": lambda s: mxq.mxq_linear_bf16(X, torch.ones(8, 64), stream=s),
    "linear_residual": lambda s: mxq.mxq_linear_residual(X, *W, Y, stream=s),
    "linear_swiglu": lambda s: mxq.mxq_linear_swiglu(X, *W, stream=s),
    "linear_batch": lambda s: mxq.mxq_linear_batch([dict(x=X, codes=W[0], scales=W[1], out=Y)], stream=s),
    "greedy_accept": lambda s: mxq.mxq_greedy_accept(LOGITS, DRAFT, stream=s),
    "greedy_accept_tokens": lambda s: mxq.mxq_greedy_accept_tokens(DRAFT, TOKENS, stream=s),
    "lm_head_accept": lambda s: mxq.mxq_lm_head_accept(X, *W, stream=s),
}


@pytest.mark.parametrize("name", LAYERS)
def test_layer_calls_allocate_on_the_stream_they_run_on(name, record, monkeypatch):
    monkeypatch.setattr(binding, "_any_mem", lambda t, dtype, what: t.data_ptr())
    LAYERS[name](STREAM)
    assert record.launches == [77] and record.made and set(record.made) == {77}
    record.made.clear()
    LAYERS[name](None)
    assert record.launches == [77, None] and record.made and set(record.made) == {None}


def test_workspaces_kept_for_callers_that_pass_none_are_one_per_stream(record):
    for s in (None, STREAM, types.SimpleNamespace(cuda_stream=78), None, STREAM):
        LAYERS["linear"](s)
    assert sorted(str(k[2]) for k in binding._default_ws) == ["77", "78", "None"]
