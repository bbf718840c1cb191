"""Sequences that share pages and go their own ways: after a fork, a sequence that rolls back behind it and grows again must not write
into its siblings' tokens.  Random programs of fork, rollback, append and release, with every sequence's tokens read back after every
step, and the bookkeeping against one page at a time."""
import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def plain_resize(tables, lens, refs, new, page):
    """The rule of include/mxq.h, one sequence after the other; returns the (sequence, old page, new page, tokens) copied."""
    up = lambda n: -(-int(n) // page)
    ok = [0 <= n <= tables.shape[1] * page for n in new]
    split = [int(tables[b, n // page]) if ok[b] and n < lens[b] and n % page and refs[tables[b, n // page]] > 1 else -1 for b, n in enumerate(new)]
    for b, n in enumerate(new):
        for w in range(up(n) if ok[b] else up(lens[b]), up(lens[b])):
            refs[tables[b, w]] -= 1
            tables[b, w] = -1
    free = [p for p in range(len(refs)) if refs[p] == 0]
    full, copies = False, []
    for b, n in enumerate(new):
        if not ok[b]:
            continue
        want = 1 if split[b] >= 0 else max(0, up(n) - up(lens[b]))
        if want and (full or want > len(free)):
            full = True
            if split[b] >= 0:
                lens[b] = min(lens[b], (n // page + 1) * page)
            continue
        if split[b] >= 0:
            tables[b, n // page] = free.pop(0)
            refs[tables[b, n // page]] = 1
            copies.append((b, split[b]))
        else:
            for w in range(up(lens[b]), up(n)):
                tables[b, w] = free.pop(0)
                refs[tables[b, w]] = 1
        lens[b] = n
    for _, old in copies:
        refs[old] -= 1
    return copies


class Server:
    """A cache and what it should hold: per sequence the tokens in order, a token being the values its rows were cast to."""

    def __init__(self, slots, width, pages, page, h, d, layers, seed):
        self.rng = np.random.default_rng(seed)
        self.page, self.h, self.d, self.layers, self.slots, self.width = page, h, d, layers, slots, width
        self.cache = mxq.KVCache.new(layers, pages, h, d, page)
        self.t_tables, self.t_lens = self.cache.new_sequences(slots, width * page)
        self.tables, self.lens, self.refs = np.full((slots, width), -1, np.int32), np.zeros(slots, np.int32), np.zeros(pages, np.int32)
        self.tokens = [torch.zeros(0, layers, 2, h, d, dtype=torch.bfloat16, device="cuda") for _ in range(slots)]
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def check_book(self):
        assert np.array_equal(self.t_lens.cpu().numpy(), self.lens)
        assert np.array_equal(self.t_tables.cpu().numpy(), self.tables)
        assert np.array_equal(self.cache.refs.cpu().numpy(), self.refs)
        for p in range(len(self.refs)):
            assert self.refs[p] == (self.tables == p).sum()

    def check_tokens(self):
        m = max(1, int(self.lens.max()))
        for layer in range(self.layers):
            k, v = mxq.mxq_kv_read(self.cache, layer, self.t_tables, self.t_lens, m, rows=self.t_lens)
            for b in range(self.slots):
                n = int(self.lens[b])
                for which, got in ((0, k), (1, v)):
                    bad = (got[b, :n] != self.tokens[b][:, layer, which]).flatten(1).any(1).nonzero()
                    assert bad.numel() == 0, "sequence %d, layer %d: token %d of %d is another's" % (b, layer, int(bad[0]), n)

    def resize(self, new):
        before = self.lens.copy()
        plain_resize(self.tables, self.lens, self.refs, [int(x) for x in new], self.page)
        mxq.mxq_kv_resize(self.cache, self.t_tables, self.t_lens, i32(new))
        self.check_book()
        for b in range(self.slots):
            self.tokens[b] = self.tokens[b][:self.lens[b]]
        return self.lens - np.minimum(before, self.lens)

    def grow(self, by):
        """Room for by[b] more tokens and their rows (of whoever got room)."""
        got = self.resize(np.minimum(self.lens + by, self.width * self.page))
        m = int(got.max())
        if m == 0:
            return
        # values that the cast keeps: the format's own, with a 4 in every block, so that its scale is 1
        own = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.bfloat16, device="cuda")
        x = own[torch.randint(0, 15, (self.slots, m, self.layers, 2, self.h, self.d), generator=self.gen, device="cuda")]
        x[..., ::32] = 4
        for layer in range(self.layers):
            mxq.mxq_kv_append(self.cache, layer, x[:, :, layer, 0].contiguous(), x[:, :, layer, 1].contiguous(), self.t_tables, self.t_lens, rows=i32(got))
        for b in range(self.slots):
            self.tokens[b] = torch.cat([self.tokens[b], x[b, :got[b]]])

    def fork(self, pairs):
        src, dst = [p[0] for p in pairs], [p[1] for p in pairs]
        mxq.mxq_kv_fork(self.cache, self.t_tables, self.t_lens, i32(src), i32(dst))
        lens = self.t_lens.cpu().numpy()
        for s, d in pairs:
            if lens[d]:
                self.tokens[d] = self.tokens[s].clone()
        self.lens, self.tables, self.refs = lens.copy(), self.t_tables.cpu().numpy().copy(), self.cache.refs.cpu().numpy().copy()


@pytest.mark.parametrize("seed,page,h,d,layers,pages", [(1, 32, 1, 64, 1, 100), (2, 32, 3, 128, 2, 60), (3, 64, 2, 64, 40, 50), (4, 128, 2, 128, 3, 24), (5, 256, 8, 64, 2, 30)])
def test_random_programs(seed, page, h, d, layers, pages):
    s = Server(7, 6, pages, page, h, d, layers, seed)
    rng = s.rng
    for step in range(40):
        what = rng.integers(0, 4)
        busy, idle = np.flatnonzero(s.lens), np.flatnonzero(s.lens == 0)
        if what == 0 or len(busy) == 0:
            by = rng.integers(0, 3 * page // 2, s.slots)
            by[rng.random(s.slots) < 0.4] = 0
            if rng.random() < 0.4:
                by = np.where(by > 0, -s.lens % page, 0)       # to a page's end: the next fork shares everything
            s.grow(by)
        elif what == 1 and len(idle):
            pick = rng.permutation(idle)[:rng.integers(1, 4)]
            s.fork([(int(rng.choice(busy)), int(x)) for x in pick])
        elif what == 2:
            new = np.where(rng.random(s.slots) < 0.5, s.lens, (s.lens * rng.random(s.slots)).astype(np.int64))
            s.resize(new)
        elif rng.random() < 0.4:
            s.resize(np.where(rng.random(s.slots) < 0.3, 0, s.lens))
        s.check_tokens()
    s.resize(np.zeros(s.slots))
    assert s.refs.sum() == 0


def test_rollback_behind_a_fork():
    """Parent and children share one full page; each rolls back into it and goes on by itself."""
    s = Server(4, 4, 12, 64, 2, 128, 33, 9)
    s.grow([128, 0, 0, 0])
    s.fork([(0, 1), (0, 2), (0, 3)])
    assert (s.refs == 4).sum() == 2
    s.resize([128, 100, 64, 33])          # one in the second page, one at its start (nothing to copy), one in the first
    s.check_tokens()
    assert s.refs[s.tables[0, 0]] == 3 and s.refs[s.tables[0, 1]] == 1
    s.grow([0, 40, 10, 20])
    s.check_tokens()
    s.resize([1, 1, 1, 1])                # all at once: everybody who shares the first page gets a copy, and the page is free again
    s.check_tokens()
    s.grow([70, 70, 70, 70])
    s.check_tokens()


def test_rollback_behind_a_fork_without_a_free_page():
    """The sequence goes back as far as it can without one: to the end of the shared page."""
    s = Server(3, 5, 4, 32, 1, 64, 2, 10)
    s.grow([64, 0, 0])
    s.fork([(0, 1)])
    s.grow([0, 32, 32])                   # the pool is full
    assert s.lens.tolist() == [64, 96, 32]
    s.resize([64, 40, 32])                # its own last page serves for the copy
    assert s.lens.tolist() == [64, 40, 32]
    s.check_tokens()
    s.resize([20, 40, 32])                # and here the page behind the shared one
    assert s.lens.tolist() == [20, 40, 32]
    s.check_tokens()
    s.grow([0, 0, 32])
    s.resize([20, 7, 32])
    s.check_tokens()


def test_rollback_with_no_page_at_all():
    s = Server(3, 5, 3, 32, 1, 64, 2, 11)
    s.grow([32, 0, 0])
    s.fork([(0, 1)])
    s.grow([0, 0, 64])
    assert s.lens.tolist() == [32, 32, 64] and (s.refs > 0).all()
    s.resize([32, 5, 64])
    assert s.lens.tolist() == [32, 32, 64]
    s.check_tokens()
    s.resize([32, 5, 0])
    assert s.lens.tolist() == [32, 5, 0]
    s.check_tokens()


def test_rollback_at_the_largest_lengths():
    """The end of a shared page that lies at 2^31 tokens, and no free page: the length stays what it was."""
    cache = mxq.KVCache.new(1, 1, 1, 64, 256)
    cache.refs.fill_(2)
    width, n = 1 << 23, (1 << 31) - 100
    tables = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    tables[0, width - 1] = 0
    lens = i32([n])
    mxq.mxq_kv_resize(cache, tables, lens, i32([n - 50]))
    assert lens.tolist() == [n] and cache.refs.tolist() == [2] and int(tables[0, -1]) == 0
