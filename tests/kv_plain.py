"""Plain 64-bit implementation of the 4-bit key/value cache's operators, for tests: numpy on the host, one step at a time,
written from the definitions in include/mxq.h.  The cast itself is the oracle's."""
import numpy as np

import oracle

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], np.float64)


def e8m0(b):
    b = np.asarray(b, np.int64)
    return np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))


class Cache:
    """Host copy of a pool: bytes [layers][pages][page bytes], with a view of one tile's parts."""

    def __init__(self, pool, kv_heads, head_dim, page_tokens):
        self.pool, self.h, self.d, self.p = pool, kv_heads, head_dim, page_tokens
        self.nb = head_dim // 32
        self.tile = 34 * head_dim
        assert pool.shape[2] == self.tile * kv_heads * (page_tokens // 32)

    def _base(self, page_slot, head):
        return ((page_slot // 32) * self.h + head) * self.tile

    def places(self, which, slot, head):
        """Byte offsets in a page of one token's row (in natural order) and of its scales; which: 0 = K, 1 = V."""
        t, nb, d = slot % 32, self.nb, self.d
        n = np.arange(d // 2)
        j, i = n // 16, n % 16
        if which == 0:
            row = (i // 4) * 4 * nb + 4 * j + i % 4
            sc = 32 * d + t * nb + np.arange(nb)
        else:
            row = (i // 2) * 2 * nb + 2 * j + i % 2
            u, tig, e, h = t // 16, t % 4, t % 8 // 4, t % 16 // 8
            sc = 32 * d + 32 * nb + 16 * nb * u + 4 * nb * tig + 2 * nb * h + 2 * np.arange(nb) + e
        base = self._base(slot, head)
        return base + which * 16 * d + t * (d // 2) + row, base + sc

    def put(self, which, layer, page, slot, head, codes, scales):
        row, sc = self.places(which, slot, head)
        self.pool[layer, page, row] = codes
        self.pool[layer, page, sc] = scales

    def get(self, which, layer, page, slot, head):
        row, sc = self.places(which, slot, head)
        return self.pool[layer, page, row], self.pool[layer, page, sc]

    def values(self, which, layer, table, n, head):
        """[n][d] float64 of tokens 0..n-1; rows on a missing page are None'd out by the second result."""
        out, there = np.zeros((n, self.d)), np.zeros(n, bool)
        for t in range(n):
            page = int(table[t // self.p])
            if not 0 <= page < self.pool.shape[1]:
                continue
            c, s = self.get(which, layer, page, t % self.p, head)
            v = np.stack([E2M1[c & 15], E2M1[c >> 4]], 1).reshape(-1)
            out[t] = v * np.repeat(e8m0(s), 32)
            there[t] = True
        return out, there


def append(cache, layer, k_bits, v_bits, tables, lens, rows):
    """k_bits, v_bits uint16 [B][M][H][D]"""
    for which, bits in ((0, k_bits), (1, v_bits)):
        b_, m, h_, d = bits.shape
        codes, scales, _ = oracle.quantize(np.ascontiguousarray(bits.reshape(-1, d)))
        codes, scales = codes.reshape(b_, m, h_, -1), scales.reshape(b_, m, h_, -1)
        for b in range(b_):
            for i in range(rows[b]):
                pos = lens[b] - rows[b] + i
                page = tables[b][pos // cache.p] if pos >= 0 else -1
                if 0 <= page < cache.pool.shape[1]:
                    for h in range(h_):
                        cache.put(which, layer, page, pos % cache.p, h, codes[b, i, h], scales[b, i, h])


def seen(n, r, i, tree):
    """Which of n tokens row i of the last r sees."""
    d = np.arange(n) - (n - r)
    if tree is None:
        return d <= i
    return (d < 0) | np.array([x >= 0 and (int(tree) >> int(x)) & 1 == 1 for x in d], bool)


def attention(cache, layer, q, tables, lens, rows, scale, trees=None):
    """q float64 [B][M][Hq][D] -> (o, lse, bound on what the rounding of the weights may do, bound on a score's error)"""
    b_, m, hq, d = q.shape
    g = hq // cache.h
    o, lse = np.zeros(q.shape), np.full((b_, m, hq), -np.inf)
    spread, smax = np.zeros(q.shape), np.zeros((b_, m, hq))
    for b in range(b_):
        n = int(lens[b])
        for h in range(cache.h):
            k, there = cache.values(0, layer, tables[b], n, h)
            v, _ = cache.values(1, layer, tables[b], n, h)
            for i in range(int(rows[b])):
                on = there & seen(n, int(rows[b]), i, None if trees is None else trees[b][i])
                if not on.any():
                    continue
                for a in range(g):
                    x = k[on] @ q[b, i, h * g + a] * scale
                    top = x.max() if not np.isnan(x).any() else np.nan
                    w = np.exp(x - top)
                    o[b, i, h * g + a] = w @ v[on] / w.sum()
                    spread[b, i, h * g + a] = w @ np.abs(v[on]) / w.sum()
                    lse[b, i, h * g + a] = top + np.log(w.sum())
                    smax[b, i, h * g + a] = (np.abs(k[on]) @ np.abs(q[b, i, h * g + a])).max() * abs(scale)
    return o, lse, spread, smax


def pages_for(n, p):
    return -(-int(n) // p)


def resize(tables, lens, refs, new, p):
    """One page at a time; tables, lens, refs are changed."""
    width = tables.shape[1]
    ok = [0 <= int(x) <= width * p for x in new]
    want = [pages_for(x, p) if y else pages_for(n, p) for x, y, n in zip(new, ok, lens)]
    for b in range(len(lens)):
        for w in range(want[b], pages_for(lens[b], p)):
            if 0 <= tables[b, w] < len(refs):
                refs[tables[b, w]] -= 1
            tables[b, w] = -1
    free = [i for i in range(len(refs)) if refs[i] == 0]
    full = False
    for b in range(len(lens)):
        have = pages_for(lens[b], p)
        grow = want[b] - have
        if grow > 0 and (full or grow > len(free)):
            full = True
            continue
        for w in range(have, want[b]):
            tables[b, w] = free.pop(0)
            refs[tables[b, w]] += 1
        if ok[b]:
            lens[b] = new[b]


def fork(cache, tables, lens, refs, src, dst, p):
    old = cache.pool.copy()
    before = lens.copy()
    free = [i for i in range(len(refs)) if refs[i] == 0]
    full = False
    for s, d in zip(src, dst):
        if not (0 <= s < len(lens) and 0 <= d < len(lens)) or s == d or before[d] != 0:
            continue
        n = int(before[s])
        part = n % p
        if part and (full or not free):
            full = True
            continue
        for w in range(n // p):
            tables[d, w] = tables[s, w]
            refs[tables[s, w]] += 1
        if part:
            q = free.pop(0)
            tables[d, n // p] = q
            refs[q] = 1
            filled = -(-part // 32) * cache.h * cache.tile
            cache.pool[:, q, :filled] = old[:, tables[s, n // p], :filled]
        lens[d] = n


def compact(cache, tables, lens, rows, keep, kept):
    out = []
    for b in range(len(lens)):
        first = int(lens[b]) - int(rows[b])
        for layer in range(cache.pool.shape[0]):
            for h in range(cache.h):
                for which in (0, 1):
                    moved = [cache.get(which, layer, tables[b][(first + x) // cache.p], (first + x) % cache.p, h) for x in keep[b][:kept[b]]]
                    moved = [(c.copy(), s.copy()) for c, s in moved]
                    for j, (c, s) in enumerate(moved):
                        cache.put(which, layer, tables[b][(first + j) // cache.p], (first + j) % cache.p, h, c, s)
        out.append(first + int(kept[b]))
    return np.array(out, np.int32)
