"""mxq_kv_fork at the edges: more layers than a grid has room for in one of its dimensions, and parents that lack a page."""
import pytest
import torch

import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("layers", [65535, 65536, 70000])
def test_fork_in_every_layer(layers):
    cache = mxq.KVCache.new(layers, 3, 1, 64, 32)
    cache.pages.copy_(torch.randint(0, 256, cache.pages.shape, dtype=torch.uint8, device="cuda"))
    tables, lens = cache.new_sequences(2, 64)
    mxq.mxq_kv_resize(cache, tables, lens, i32(37, 0))
    before = cache.pages.clone()
    mxq.mxq_kv_fork(cache, tables, lens, i32(0), i32(1))
    assert lens.tolist() == [37, 37] and tables.tolist() == [[0, 1], [0, 2]] and cache.refs.tolist() == [2, 1, 1]
    assert torch.equal(cache.pages[:, :2], before[:, :2]) and torch.equal(cache.pages[:, 2], before[:, 1])


@pytest.mark.parametrize("gone", [-1, 1 << 20])
def test_fork_of_a_parent_without_its_last_page(gone):
    """Tokens on an entry that is no page are left out by every call: a child has no more of them than its parent."""
    cache = mxq.KVCache.new(2, 8, 1, 64, 32)
    cache.pages.fill_(0x11)
    tables, lens = cache.new_sequences(4, 96)
    mxq.mxq_kv_resize(cache, tables, lens, i32(70, 40, 0, 0))
    tables[0, 2] = gone
    mxq.mxq_kv_fork(cache, tables, lens, i32(0, 1), i32(2, 3))
    assert lens.tolist() == [70, 40, 70, 40]
    assert tables[2].tolist() == [tables[0, 0], tables[0, 1], -1] and int(tables[3, 1]) >= 0
    q = torch.ones(4, 1, 1, 64, dtype=torch.bfloat16, device="cuda")
    _, lse = mxq.mxq_kv_attention(q, cache, 1, tables, lens, with_lse=True)
    assert torch.equal(lse[:2], lse[2:])
    held = (tables >= 0) & (tables < 8)
    assert int(cache.refs.sum()) == int(held.sum()) + 1          # (and the one that was taken out of the parent's table by hand)
