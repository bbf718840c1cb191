"""Host threads with streams of their own that call the same operator on shapes whose kernels want different amounts of shared memory: no
call is refused on account of another thread's, and every result is what it is alone."""
import ctypes
import threading

import pytest
import torch

import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import binding

pytestmark = pytest.mark.gpu


def lora(m, n, k, r, count, dtype=torch.float32):
    """(a call of the C function on a stream, its outputs); what a caller in C would spend between two calls is little, and so is it here."""
    g = torch.Generator(device="cuda").manual_seed(k)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, a, b, base = rn(m, k).bfloat16(), (rn(count, r, k) / k ** 0.5).bfloat16(), rn(count, n, r).bfloat16(), rn(m, n).to(dtype)
    ids = torch.randint(0, count, (m,), generator=g, device="cuda").int()
    ws = torch.zeros(mxq.mxq_lora_workspace_bytes(m, n, k, r, count), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(base)
    ad, ip, _ = binding._adapters(a, b, None, ids, m, k)
    p, i64, f = ctypes.c_void_p, ctypes.c_int64, binding.lib().mxq_lora
    args = (p(x.data_ptr()), i64(m), p(ctypes.addressof(ad)), p(ip), i64(n), i64(k), p(base.data_ptr()), p(out.data_ptr()),
            ctypes.c_int(binding._DTYPES[dtype]), p(ws.data_ptr()), ctypes.c_size_t(ws.numel()))
    keep = (x, a, b, base, ids, ws, ad)

    def call(s, keep=keep):
        return f(*args, s)

    return call, (out,)


def rules(b, v, biases):
    g = torch.Generator(device="cuda").manual_seed(v)
    logits = torch.randn(b, 2, v, generator=g, device="cuda")
    draft = logits[:, 0].argmax(-1, keepdim=True).int()
    counts = torch.randint(0, 3, (b, v), generator=g, device="cuda").int()
    bias = (torch.randint(0, v, (b, biases), generator=g, device="cuda").int(), torch.randn(b, biases, generator=g, device="cuda")) if biases else (None, None)
    ru = mxq.LogitRules(counts, torch.tensor([[1.2, 0.1, 0.1]] * b, device="cuda"), *bias)
    ws = mxq.new_workspace(mxq.mxq_greedy_accept_rules_workspace_bytes(b, 2, v))
    i = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")
    out = (i(b, 2), i(b), i(b))
    p, f = ctypes.c_void_p, binding.lib().mxq_greedy_accept_rules
    args = (p(logits.data_ptr()), ctypes.c_int(0), ctypes.c_int64(b), ctypes.c_int(2), ctypes.c_int64(v), p(draft.data_ptr()), ctypes.c_int(1),
            p(ru.ptr), *(p(t.data_ptr()) for t in out), p(ws.data_ptr()), ctypes.c_size_t(ws.numel()))
    keep = (logits, draft, ru, ws)

    def call(s, keep=keep):
        return f(*args, s)

    return call, out


PAIRS = {
    "few rows": (lambda: lora(16, 64, 11008, 32, 16), lambda: lora(16, 64, 8192, 32, 16)),
    "windows": (lambda: lora(600, 40, 1312, 24, 20), lambda: lora(600, 40, 4128, 24, 20)),
    "many rows": (lambda: lora(3000, 64, 512, 64, 2), lambda: lora(1000, 64, 4096, 64, 2)),
    "many rows, BF16": (lambda: lora(3000, 4096, 96, 128, 2, torch.bfloat16), lambda: lora(2000, 4096, 96, 128, 2, torch.bfloat16)),
    "rules": (lambda: rules(64, 128000, 0), lambda: rules(64, 128000, 5)),
}


@pytest.mark.parametrize("name", PAIRS)
def test_threads(name):
    calls = [make() for make in PAIRS[name] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in calls]
    want = []
    for call, out in calls:
        assert call(ctypes.c_void_p(0)) == 0
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
    start, refused, wrong = threading.Barrier(len(calls)), [], []

    def work(call, out, stream, want):
        handle = ctypes.c_void_p(stream.cuda_stream)
        start.wait()
        for _ in range(30):
            bad = [rc for rc in [call(handle) for _ in range(100)] if rc]
            stream.synchronize()
            if bad:
                refused.append(bad)
            elif not all(torch.equal(g.cpu(), w.cpu()) for g, w in zip(out, want)):
                wrong.append(name)

    threads = [threading.Thread(target=work, args=(*c, s, w)) for c, s, w in zip(calls, streams, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refused and not wrong, (sum(map(len, refused)), wrong)
    assert mxq.mxq_linear_device_status() == 0
