"""A workspace that is large enough for the largest call is large enough for the smaller ones."""
import pytest
import torch

import paper_2503_13565_b200 as mxq


@pytest.mark.parametrize("n,k", [(4096, 4096), (11008, 4096), (4096, 11008), (33, 96), (1000, 768), (520, 32), (64, 64)])
@pytest.mark.parametrize("rank", [8, 16, 64, 128])
def test_the_bytes_never_fall(n, k, rank):
    last = 0
    for m in list(range(1, 5000)) + [5120, 8191, 8192, 20000, 19000 * 3, 1 << 18, (1 << 20) - 1, 1 << 20]:
        now = [mxq.mxq_lora_workspace_bytes(m, n, k, rank, adapters) for adapters in (1, 6, 70, 65536)]
        assert len(set(now)) == 1 and now[0] >= last > (0 if m > 1 else -1), m
        last = now[0]
    last = [0] * 16
    for more in (0, 32, 320, 3200):
        now = [mxq.mxq_linear_lora_workspace_bytes(m, n + more, k + more, rank, 6) for m in range(1, 17)]
        assert now == sorted(now) and all(a >= b > -1 for a, b in zip(now, last))
        last = now


@pytest.mark.gpu
@pytest.mark.parametrize("k,rank,count", [(4096, 64, 6), (1312, 24, 40), (256, 128, 1)])
def test_small_batches_in_the_workspace_of_the_largest(k, rank, count):
    n, most, guard = 72, 2048, 4096
    g = torch.Generator(device="cuda").manual_seed(k)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, a, b = rn(most, k).bfloat16(), (rn(count, rank, k) / k ** 0.5).bfloat16(), rn(count, n, rank).bfloat16()
    need = mxq.mxq_lora_workspace_bytes(most, n, k, rank, count)
    held = torch.full((need + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
    for m in [1, 16, 17, 63, 64, 191, 192, 400, 511, 512, 900, 1152, 1153, 1500, most]:
        ids = torch.randint(-1, count, (m,), generator=g, device="cuda").int()
        got = mxq.mxq_lora(x[:m], a, b, ids, workspace=held[guard:guard + need])
        own = torch.full((mxq.mxq_lora_workspace_bytes(m, n, k, rank, count) + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
        assert torch.equal(got, mxq.mxq_lora(x[:m], a, b, ids, workspace=own[guard:-guard]))
        for t in (held, own):
            assert bool((t[:guard] == 0xA5).all()) and bool((t[-guard:] == 0xA5).all()), m
