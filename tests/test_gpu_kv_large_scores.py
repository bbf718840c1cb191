"""mxq_kv_attention where scores are large: a score is a sum in FP32, so its error grows with the sum of its terms' magnitudes S and goes
into every weight.  The bound of include/mxq.h, 2^-10 + (2 D + 8) * 2^-24 * S of sum w|v| / sum w, from ordinary scores to such of
thousands, against the 64-bit form of tests/kv_exact.py."""
import pytest
import torch

import kv_exact
import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,hq", [(1, 4), (3, 16)])
@pytest.mark.parametrize("size", [0.5, 4.0, 32.0, 256.0, 2048.0])
def test_scores_of_every_size(size, m, hq, d):
    """Keys in pairs that differ little, so that large scores lie close together and several tokens share the weight."""
    h, lens = 2, [400, 9001, 33]
    cache = mxq.KVCache.new(1, 300, h, d, 64)
    tables, t_lens = cache.new_sequences(3, max(lens))
    mxq.mxq_kv_resize(cache, tables, t_lens, i32(lens))
    gen = torch.Generator(device="cuda").manual_seed(int(size * 2) + d)
    for b, n in enumerate(lens):
        base = torch.randn(1, 1, h, d, generator=gen, device="cuda")
        k = base + torch.randn(1, n, h, d, generator=gen, device="cuda") * min(1.0, 2.0 / size)
        v = torch.randn(1, n, h, d, generator=gen, device="cuda")
        mxq.mxq_kv_append(cache, 0, k.bfloat16(), v.bfloat16(), tables[b:b + 1], t_lens[b:b + 1])
    q = (torch.randn(3, m, hq, d, generator=gen, device="cuda") * size).bfloat16()
    ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(3, m, hq, h, d))
    out, lse = mxq.mxq_kv_attention(q, cache, 0, tables, t_lens, workspace=ws, with_lse=True)
    exact = kv_exact.attention(cache, 0, q, tables, lens, [m] * 3, d ** -0.5)
    assert float(exact[3].max()) > 4 * size
    kv_exact.check(out, lse, exact, d, adds=512)
    assert bool(torch.isfinite(out).all())
