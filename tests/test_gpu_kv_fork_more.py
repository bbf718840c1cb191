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
