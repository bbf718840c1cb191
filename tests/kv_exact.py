"""Attention over a 4-bit cache in 64 bits on the GPU, for caches too long for the plain implementation on the host: written
from the layout and the formulas in include/mxq.h with elementary torch operations, one (sequence, kv head) at a time."""
import math

import torch

E2M1 = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]


def values(pages, which, table, n, head, heads, d, page):
    """[n][d] float64 of tokens 0..n-1 of a sequence (which: 0 = K, 1 = V), and which of them lie on a page of the pool.
    pages: uint8 [num_pages][bytes], one layer."""
    nb, dev = d // 32, pages.device
    t = torch.arange(n, device=dev)
    entry = table[t // page].long()
    there = (entry >= 0) & (entry < pages.shape[0])
    tile = entry.clamp(0, pages.shape[0] - 1) * pages.shape[1] + ((t % page // 32) * heads + head) * 34 * d
    s = t % 32
    b = torch.arange(d // 2, device=dev)           # natural byte of a row
    j, i = b // 16, b % 16
    if which == 0:
        row = (i // 4) * 4 * nb + 4 * j + i % 4
        scale = 32 * d + s.unsqueeze(1) * nb + torch.arange(nb, device=dev)
    else:
        row = (i // 2) * 2 * nb + 2 * j + i % 2
        at = 16 * nb * (s // 16) + 4 * nb * (s % 4) + 2 * nb * (s % 16 // 8) + s % 8 // 4
        scale = 32 * d + 32 * nb + at.unsqueeze(1) + 2 * torch.arange(nb, device=dev)
    flat = pages.reshape(-1)
    codes = flat[(tile + which * 16 * d + s * (d // 2)).unsqueeze(1) + row].long()
    table16 = torch.tensor(E2M1, dtype=torch.float64, device=dev)
    v = torch.stack((table16[codes & 15], table16[codes >> 4]), -1).view(n, nb, 32)
    e = flat[tile.unsqueeze(1) + scale].long()
    factor = torch.where(e == 255, math.nan, torch.ldexp(torch.ones_like(e, dtype=torch.float64), e - 127))
    return (v * factor.unsqueeze(-1)).view(n, d), there


def attention(cache, layer, q, tables, lens, rows, scale, trees=None):
    """q BF16 [B][M][Hq][D] on the GPU; lens, rows, trees: lists -> (o, lse, spread = sum w|v| / sum w, smax = the largest sum of
    magnitudes behind a visible score), all float64 on the GPU.  A row that sees nothing: o = 0, lse = -inf."""
    b_, m, hq, d = q.shape
    h, g, dev = cache.kv_heads, q.shape[2] // cache.kv_heads, q.device
    o, spread = (torch.zeros(q.shape, dtype=torch.float64, device=dev) for _ in range(2))
    lse = torch.full((b_, m, hq), -math.inf, dtype=torch.float64, device=dev)
    smax = torch.zeros((b_, m, hq), dtype=torch.float64, device=dev)
    for b in range(b_):
        n, r = int(lens[b]), int(rows[b])
        if n == 0 or r == 0:
            continue
        pos = torch.arange(n, device=dev) - (n - r)
        for head in range(h):
            k, there = values(cache.pages[layer], 0, tables[b], n, head, h, d, cache.page_tokens)
            v, _ = values(cache.pages[layer], 1, tables[b], n, head, h, d, cache.page_tokens)
            v = torch.where(there.unsqueeze(1), v, 0.0)
            for i in range(r):
                if trees is None:
                    see = pos <= i
                else:
                    bits = torch.tensor([(trees[b][i] >> x) & 1 == 1 for x in range(r)], device=dev)
                    see = (pos < 0) | bits[pos.clamp_min(0)]
                see = there & see
                if not bool(see.any()):
                    continue
                at = slice(head * g, head * g + g)
                x = (q[b, i, at].double() @ k.T * scale).masked_fill(~see, -math.inf)
                top = x.amax(-1, keepdim=True)         # (NaN if a visible score is)
                w = torch.exp(x - top)
                total = w.sum(-1, keepdim=True)
                dead = ~see if bool(torch.isnan(v).any()) else None
                vv = v if dead is None else torch.where(dead.unsqueeze(1), 0.0, v)
                o[b, i, at] = w @ vv / total
                spread[b, i, at] = w @ vv.abs() / total
                lse[b, i, at] = (top + torch.log(total)).squeeze(-1)
                smax[b, i, at] = ((q[b, i, at].double().abs() @ k.abs().T) * abs(scale)).masked_fill(~see, 0.0).amax(-1)
    return o, lse, spread, smax


def score_share(d, smax):
    """What the FP32 error of the scores may do to an output, in units of sum w|v| / sum w: a score is off by at most
    (D + 4) * 2^-24 of the sum of its terms' magnitudes (D products and sums, and the factor), every weight by that share of itself,
    and so is the sum that divides them."""
    return 2 * (d + 4) * 2.0 ** -24 * smax


def check(out, lse, exact, d, adds=0):
    """out BF16, lse FP32 against attention()'s result: the weights' rounding is 2^-10 of sum w|v| / sum w, the scores' error comes on
    top; rounding to BF16 is monotonic, so out lies between the roundings of both ends.  adds: length of the longest chain of FP32
    additions behind lse (2^-24 each)."""
    o, wl, spread, smax = exact
    nan, empty = torch.isnan(o).any(-1), torch.isneginf(wl)
    assert torch.equal(torch.isnan(out).any(-1), nan), "NaN in the wrong rows"
    assert torch.equal(torch.isneginf(lse), empty) and bool((out[empty] == 0).all())
    assert bool(torch.isnan(lse[torch.isnan(wl)]).all())
    bound = (2.0 ** -10 + score_share(d, smax)).unsqueeze(-1) * spread + 2.0 ** -133
    low, high, got = (o - bound).bfloat16().double(), (o + bound).bfloat16().double(), out.double()
    bad = ~nan.unsqueeze(-1) & ~((low <= got) & (got <= high))
    assert not bool(bad.any()), "%d outputs outside, first %s: %r not in %r .. %r" % (
        int(bad.sum()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(low[bad][0]), float(high[bad][0]))
    fine = ~empty & ~torch.isnan(wl)
    tol = (d + 4) * 2.0 ** -24 * smax + 2.0 ** -21 * wl.abs() + 2.0 ** -19 + adds * 2.0 ** -24
    off = (lse.double() - wl).abs()
    assert bool((off[fine] <= tol[fine]).all()), "lse error/tolerance %.3g" % float((off[fine] / tol[fine]).max())
