"""mxq_lora and mxq_linear_lora against the definition in 64 bits, within the bound that include/mxq.h states."""
import numpy as np
import pytest
import torch

import oracle
import paper_2503_13565_b200 as mxq
import step_plain as plain
from paper_2503_13565_b200 import synth

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def make(m, n, k, r, count, seed=0, ids=None, scale=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = rn(m, k).bfloat16()
    a, b = (rn(count, r, k) / k ** 0.5).bfloat16(), (rn(count, n, r) * torch.exp(rn(count, n, 1))).bfloat16()
    if ids is None:
        ids = torch.randint(-2, count + 1, (m,), generator=g, device="cuda")          # -2, -1 and count: no adapter
    return x, a, b, torch.as_tensor(ids, device="cuda").int(), rn(count).contiguous() if scale else None


def tolerance(y, mag, k, r, dtype):
    # sums: K / 16 products' sums after one another, then warps, splits and 3 * r / 16 more, each within 2^-22 of the magnitude; BF16: A x
    # keeps 16 bits where it meets B (2^-17) and Y is rounded (2^-8)
    t = (k / 16 + 96) * 2.0 ** -22 * mag + 2.0 ** -23 * y.abs() + 1e-37
    return t if dtype == F32 else t + 2.0 ** -17 * mag + 2.0 ** -8 * (y.abs() + t)


def check(got, want, mag, k, r, extra=0.0):
    t = tolerance(want, mag, k, r, got.dtype) + extra
    err = (got.double().cpu() - want).abs()
    assert bool((err <= t).all()), (float((err / t).max()), np.argwhere((err > t).numpy())[:4])


SHAPES = [(1, 4096, 4096, 16, 8), (1, 1, 32, 8, 1), (2, 31, 64, 24, 3), (5, 33, 96, 40, 2), (16, 1025, 4096, 32, 24), (16, 256, 1312, 128, 5), (17, 100, 160, 64, 4),
          (64, 515, 768, 16, 40), (200, 72, 256, 72, 7), (511, 40, 64, 8, 3), (512, 136, 96, 104, 9), (700, 1000, 768, 64, 5), (1030, 33, 416, 16, 70), (513, 64, 64, 128, 2), (600, 40, 448, 24, 20), (2000, 264, 1024, 8, 3),
          (520, 48, 4096, 72, 5), (3001, 16, 128, 112, 40), (64, 40, 256, 24, 1), (64, 520, 96, 128, 1), (100, 136, 96, 16, 2), (191, 72, 320, 72, 3), (330, 33, 192, 128, 4)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k,r,count", SHAPES)
def test_adapters_of_many_rows(m, n, k, r, count, dtype):
    x, a, b, ids, scale = make(m, n, k, r, count, seed=m)
    base = torch.randn(m, n, device="cuda").to(dtype)
    want, mag = plain.lora(x, a, b, scale, ids, base)
    got = mxq.mxq_lora(x, a, b, ids, scale=scale, base=base)
    assert got.dtype == dtype
    check(got, want, mag, k, r)
    none = ((ids < 0) | (ids >= count)).cpu()
    assert torch.equal(got.cpu()[none], base.cpu()[none])
    own = base.clone()
    assert mxq.mxq_lora(x, a, b, ids, scale=scale, base=own, out=own) is own and torch.equal(own, got)           # in place
    alone = mxq.mxq_lora(x, a, b, ids, out_dtype=dtype)                                                          # no base, no scales
    want, mag = plain.lora(x, a, b, None, ids, None)
    check(alone, want, mag, k, r)
    assert bool((alone.cpu()[none] == 0).all()) and mxq.mxq_linear_device_status() == 0


def test_orders_and_neighbours_change_nothing():
    """A row's result does not depend on what the others have, nor on its place in the window (bit for bit)."""
    m, n, k, r, count = 130, 96, 256, 32, 6
    for m in (16, 130, 600):
        x, a, b, ids, scale = make(m, n, k, r, count, seed=2)
        got = mxq.mxq_lora(x, a, b, ids, scale=scale)
        order = torch.randperm(m, device="cuda")
        assert torch.equal(mxq.mxq_lora(x[order], a, b, ids[order], scale=scale), got[order])
        assert torch.equal(mxq.mxq_lora(x, a, b, ids, scale=scale), got)


@pytest.mark.parametrize("ids", [[0] * 16, [3] * 16, [-1] * 16, list(range(16)), [0, 1] * 8, [5] + [-1] * 15])
def test_owners(ids):
    x, a, b, ids, scale = make(16, 200, 512, 16, 16, ids=ids)
    base = torch.randn(16, 200, device="cuda")
    want, mag = plain.lora(x, a, b, scale, ids, base)
    check(mxq.mxq_lora(x, a, b, ids, scale=scale, base=base), want, mag, 512, 16)


def test_values_that_are_not_finite_stay_in_their_rows():
    for m, k in ((12, 96), (600, 96), (600, 128), (200, 128)):
        x, a, b, ids, scale = make(m, 72, k, 16, 4, seed=3, ids=[i % 4 for i in range(m)])
        base = torch.randn(m, 72, device="cuda")
        clean = mxq.mxq_lora(x, a, b, ids, scale=scale, base=base)
        a[1, 3, 5], b[2, 7, 2], x[3, 4], scale[1] = float("inf"), float("nan"), float("nan"), float("inf")
        got = mxq.mxq_lora(x, a, b, ids, scale=scale, base=base)
        fine = (ids == 0) | ((ids == 3) & (torch.arange(m, device="cuda") != 3))
        assert torch.equal(got[fine], clean[fine])
        assert not bool(got[ids == 1].isfinite().any()) and bool(got[3].isnan().all()) and bool(got[ids == 2][:, 7].isnan().all())
        keep = torch.arange(72, device="cuda") != 7
        assert torch.equal(got[ids == 2][:, keep], clean[ids == 2][:, keep])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k,r,count", [(1, 1000, 4096, 16, 3), (3, 33, 96, 8, 2), (8, 4096, 768, 64, 8), (16, 2000, 1312, 40, 20), (16, 11008, 4096, 32, 24)])
def test_beside_the_4_bit_layer(m, n, k, r, count, dtype):
    x, a, b, ids, scale = make(m, n, k, r, count, seed=n)
    w = synth.normal_bf16((n, k), 0.02, 9)
    codes, scales = mxq.mxq_quantize(w.cuda())
    y64, a64 = oracle.linear(synth.bits_of(x.cpu()), *oracle.quantize(synth.bits_of(w))[:2])
    want, mag = plain.lora(x, a, b, scale, ids, torch.from_numpy(y64))
    for ws in (None, torch.full((mxq.mxq_linear_lora_workspace_bytes(m, n, k, r, count),), 255, dtype=torch.uint8, device="cuda")):
        got = mxq.mxq_linear_lora(x, codes, scales, a, b, ids, scale=scale, out_dtype=dtype, workspace=ws)
        check(got, want, mag, k, r, extra=(2e-3 * torch.from_numpy(a64) + 1e-6) * (1 + 2.0 ** -8))
    if dtype == F32:                                      # without adapters it is the layer
        none = torch.full_like(ids, -1)
        ws = mxq.new_workspace(mxq.mxq_linear_workspace_bytes(m, n, k))
        assert torch.equal(mxq.mxq_linear_lora(x, codes, scales, a, b, none, scale=scale), mxq.mxq_linear(x, codes, scales, workspace=ws))
    assert mxq.mxq_linear_device_status() == 0


def test_chains_without_synchronisation():
    """Layers with adapters one after another through shared buffers and one workspace: as with a synchronisation after every call."""
    n, r, count = 768, 16, 5
    ws = torch.empty(mxq.mxq_linear_lora_workspace_bytes(16, n, n, r, count), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    layers = []
    for i in range(4):
        _, a, b, _, scale = make(1, n, n, r, count, seed=i)
        layers.append((mxq.mxq_quantize((torch.randn(n, n, generator=g, device="cuda") * 0.03).bfloat16()), a, (b * 0.1).bfloat16(), scale))
    for m in (1, 3, 16):
        x0 = torch.randn(m, n, generator=g, device="cuda").bfloat16()
        ids = torch.randint(-1, count, (m,), generator=g, device="cuda").int()

        def go(sync):
            x, y = x0.clone(), torch.empty_like(x0)
            for _ in range(3):
                for w, a, b, s in layers:
                    mxq.mxq_linear_lora(x, *w, a, b, ids, scale=s, out=y, workspace=ws)
                    if sync:
                        torch.cuda.synchronize()
                    x, y = y, x
            return x

        want = go(True)
        for _ in range(5):
            assert torch.equal(go(False), want)


def test_captured_and_on_a_stream_of_its_own():
    m, n, k, r, count = 9, 520, 256, 24, 3
    x, a, b, ids, scale = make(m, n, k, r, count)
    base = torch.randn(m, n, device="cuda")
    side = torch.cuda.Stream()
    want = mxq.mxq_lora(x, a, b, ids, scale=scale, base=base)
    torch.cuda.synchronize()
    got = [mxq.mxq_lora(x, a, b, ids, scale=scale, base=base, stream=side) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in got)
    ws = torch.empty(mxq.mxq_lora_workspace_bytes(m, n, k, r, count), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = mxq.mxq_lora(x, a, b, ids, scale=scale, base=base, workspace=ws)
    for s in (1, 2):
        x2, a2, _, ids2, _ = make(m, n, k, r, count, seed=s)
        x.copy_(x2), a.copy_(a2), ids.copy_(ids2)
        graph.replay()
        assert torch.equal(y, mxq.mxq_lora(x, a, b, ids, scale=scale, base=base))
