"""The operators of the 4-bit key/value cache as a user's program calls them, with their plain forms and their work.

A cache is a pool of pages, uint8 [layers][pages][P / 32][kv heads][tile], every tile holding 32 tokens of one head:

    K codes  [32][D/2]    byte c*(4*nb) + 4*j + i of a row = byte 16*j + 4*c + i of the row in natural order
    V codes  [32][D/2]    byte g*(2*nb) + 2*j + i of a row = byte 16*j + 2*g + i of the row in natural order
    K scales [32][nb]
    V scales [32*nb]      token t = 16*u + tig + 4*e + 8*h, block j at  16*nb*u + 4*nb*tig + 2*nb*h + 2*j + e

with nb = D / 32 blocks per row; natural byte b of a row holds elements 2b (low nibble) and 2b + 1, E2M1; scales E8M0.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"


# ---- cases --------------------------------------------------------------------------------------------------------------


def listed():
    return [
        # one draft step of a 7B-shaped model on one sequence: the smallest call, latency counts
        dict(name="attention_decode_1x2047_h32", op="attention", B=1, M=1, hq=32, hkv=32, d=128, page=64, layers=1,
             lo=2047, hi=2047, ragged=False, tree=False, shape_seed=1),
        # a serving batch of sequences of many lengths, grouped heads
        dict(name="attention_decode_32xragged_h32_8", op="attention", B=32, M=1, hq=32, hkv=8, d=128, page=64, layers=2,
             lo=257, hi=8193, ragged=False, tree=False, shape_seed=2),
        # verification of a token tree, several rows a sequence, small heads, fewer rows in some sequences
        dict(name="attention_tree_8x16_h32_8_d64", op="attention", B=8, M=16, hq=32, hkv=8, d=64, page=32, layers=1,
             lo=1001, hi=5003, ragged=True, tree=True, shape_seed=3),
        # long contexts, no grouping: the largest
        dict(name="attention_long_2x131071_h32", op="attention", B=2, M=1, hq=32, hkv=32, d=128, page=128, layers=1,
             lo=131071, hi=131071, ragged=False, tree=False, shape_seed=4),
        # the new row of every sequence of a decoding batch
        dict(name="append_decode_48x1_h8", op="append", B=48, M=1, hkv=8, d=128, page=64, layers=2, lo=100, hi=4000,
             ragged=False, shape_seed=5),
        # prompts of different lengths
        dict(name="append_prompt_4x4095_h32", op="append", B=4, M=4095, hkv=32, d=128, page=64, layers=1, lo=4095, hi=4400,
             ragged=True, shape_seed=6),
        # a speculative round's bookkeeping: room for the proposals, then back
        dict(name="resize_round_16_of_1024", op="resize", B=16, W=64, pages=1024, page=64, grow=8, lo=100, hi=3900, shape_seed=7),
        # a large server: some sequences take a whole prompt's pages
        dict(name="resize_prompts_256_of_65536", op="resize", B=256, W=512, pages=65536, page=64, grow=4096, lo=64, hi=24000, shape_seed=8),
        # one sequence branches into four
        dict(name="fork_1to4_layers32_h8", op="fork", B=1, children=4, W=64, hkv=8, d=128, page=64, layers=32, lo=1000, hi=3000, shape_seed=9),
        # a batch branches
        dict(name="fork_16to64_layers32_h8", op="fork", B=16, children=64, W=32, hkv=8, d=128, page=64, layers=32, lo=200, hi=1000, shape_seed=10),
        # accepted path of a token tree, one sequence
        dict(name="compact_1x16_layers32_h8", op="compact", B=1, M=16, hkv=8, d=128, page=64, layers=32, lo=500, hi=1500, shape_seed=11),
        # the same for a batch
        dict(name="compact_64x48_layers16_h8", op="compact", B=64, M=48, hkv=8, d=64, page=32, layers=16, lo=60, hi=600, shape_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "append", "resize", "fork", "compact"])
    seed = rng.randrange(1 << 30)
    page = rng.choice([32, 64, 128])
    d = rng.choice([64, 128, 128])
    if op == "attention":
        hq, hkv = rng.choice([(32, 32), (32, 8), (40, 40), (16, 2), (12, 12), (9, 3)])
        m = rng.choice([1, 1, 2, 5, 8, 16])
        hi = _log_int(rng, 64, 65536)
        b = max(1, min(_log_int(rng, 1, 64), 4000000 // (hi * hkv)))
        return dict(op=op, B=b, M=m, hq=hq, hkv=hkv, d=d, page=page, layers=rng.choice([1, 2]), lo=max(m, hi // rng.choice([1, 4, 30])),
                    hi=hi, ragged=m > 1 and rng.random() < 0.5, tree=m > 1 and rng.random() < 0.5, shape_seed=seed)
    if op == "append":
        m = rng.choice([1, 1, 5, 16, _log_int(rng, 17, 4000)])
        b = max(1, min(_log_int(rng, 1, 256), 16000 // m))
        return dict(op=op, B=b, M=m, hkv=rng.choice([2, 8, 32]), d=d, page=page, layers=rng.choice([1, 2]), lo=m, hi=m + _log_int(rng, 1, 500),
                    ragged=m > 1 and rng.random() < 0.5, shape_seed=seed)
    if op == "resize":
        b = _log_int(rng, 1, 256)
        w = _log_int(rng, 8, 400)
        return dict(op=op, B=b, W=w, pages=max(16, int(b * w * rng.uniform(0.6, 1.2))), page=page, grow=_log_int(rng, 1, w * page // 4),
                    lo=1, hi=w * page // 2, shape_seed=seed)
    layers = _log_int(rng, 1, 32)
    if op == "fork":
        b = _log_int(rng, 1, 16)
        w = rng.choice([8, 17, 32])
        return dict(op=op, B=b, children=b * rng.choice([1, 2, 4]), W=w, hkv=rng.choice([2, 8]), d=d, page=page, layers=layers,
                    lo=1, hi=min(w * page, 1500), shape_seed=seed)
    m = _log_int(rng, 4, 64)
    return dict(op=op, B=_log_int(rng, 1, 64), M=m, hkv=rng.choice([2, 8]), d=d, page=page, layers=min(layers, 16), lo=m, hi=m + 500, shape_seed=seed)


def _shapes(case):
    """Lengths and rows of a case's sequences, as its user's scheduler knows them on the host."""
    rng = random.Random(case["shape_seed"])
    lens = [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["B"])]
    m = case.get("M", 0)
    rows = [rng.randint(1, m) if case.get("ragged") else m for _ in lens]
    return lens, rows, rng


def _tile_bytes(d):
    return 32 * (d + d // 16)


def work(case):
    op = case["op"]
    lens, rows, rng = _shapes(case)
    if op == "attention":
        d, hq, hkv = case["d"], case["hq"], case["hkv"]
        trees = _trees(case, rows, rng) if case["tree"] else None
        pairs = 0
        for b, (n, r) in enumerate(zip(lens, rows)):
            for i in range(r):
                pairs += n - r + (bin(trees[b][i]).count("1") if trees else i + 1)
        io = sum(rows) * hq * (4 * d + 4)
        return {"bytes": sum(lens) * hkv * (d + d // 16) + io, "flops": 4 * pairs * hq * d}
    if op == "append":   # the new rows read, the cache written, the values it now stands for written
        n = sum(rows) * case["hkv"]
        return {"bytes": n * (4 * case["d"] + case["d"] + case["d"] // 16 + 4 * case["d"]), "flops": 4 * n * case["d"]}
    if op == "resize":
        return {"bytes": 4 * case["pages"] + 16 * case["B"], "flops": case["pages"]}
    if op == "fork":
        src = _fork_pairs(case)
        tiles = sum(-(-(lens[s] % case["page"]) // 32) for s in src)
        n = tiles * case["layers"] * case["hkv"] * _tile_bytes(case["d"])
        return {"bytes": 2 * n, "flops": 0}
    kept = sum(len(k) - 1 for k in _keeps(case, rows, rng))
    return {"bytes": 2 * kept * case["layers"] * case["hkv"] * (case["d"] + case["d"] // 16), "flops": 0}


def _trees(case, rows, rng):
    """Ancestor masks of random token trees: node 0 is the root, a node's parent is an earlier node."""
    out = []
    for r in rows:
        masks = []
        for i in range(r):
            masks.append((1 << i) | (masks[rng.randrange(max(0, i - 6), i)] if i else 0))
        out.append(masks + [0] * (case["M"] - r))
    return out


def _fork_pairs(case):
    return [i % case["B"] for i in range(case["children"])]


def _keeps(case, rows, rng):
    """Accepted paths: the root, then nodes behind the places they move to (a wide tree's deeper nodes)."""
    out = []
    for r in rows:
        n = rng.randint(2, max(2, min(6, r // 2)))
        out.append([0] + sorted(rng.sample(range(n, r), n - 1)))
    return out


# ---- layout and format (plain) ------------------------------------------------------------------------------------------


def _orders(d):
    """Natural byte of every stored byte of a K / V row, and the place of (token, block) among a tile's V scales."""
    nb = d // 32
    k = [16 * j + 4 * c + i for c in range(4) for j in range(nb) for i in range(4)]
    v = [16 * j + 2 * g + i for g in range(8) for j in range(nb) for i in range(2)]
    s = [[16 * nb * (t // 16) + 4 * nb * (t % 4) + 2 * nb * (t % 16 // 8) + 2 * j + t % 8 // 4 for j in range(nb)] for t in range(32)]
    return (torch.tensor(k, device=DEV), torch.tensor(v, device=DEV), torch.tensor(s, device=DEV))


def _power(e):
    """2^e in FP32 for whole e in -127..127, from the format's fields (a library's power function may be off by an ulp)."""
    bits = torch.where(e == -127, torch.full_like(e, 1 << 22), (e + 127) << 23)
    return bits.int().view(torch.float32)


def _cast(x):
    """Direct cast of [..., D] to (natural code bytes [..., D/2], scale bytes [..., D/32])."""
    blocks = x.float().unflatten(-1, (-1, 32))
    finite = torch.isfinite(blocks).all(-1)
    blocks = torch.where(finite.unsqueeze(-1), blocks, torch.zeros_like(blocks))
    top = blocks.abs().amax(-1)
    scale = ((top.view(torch.int32) >> 23) - 2).clamp_min(0)
    m = blocks.abs() * _power(127 - scale).unsqueeze(-1)
    code = ((m > 0.25).int() + (m >= 0.75).int() + (m > 1.25).int() + (m >= 1.75).int() + (m > 2.5).int() + (m >= 3.5).int() + (m > 5).int())
    code = (code + 8 * (torch.signbit(blocks) & finite.unsqueeze(-1)).int()).flatten(-2)
    scale = torch.where(finite, scale, torch.full_like(scale, 255))
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.to(torch.uint8)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _values(codes, scales):
    """FP32 values of natural code bytes [..., D/2] and scale bytes [..., D/32]."""
    table = torch.tensor([[_E2M1[b & 15], _E2M1[b >> 4]] for b in range(256)], device=DEV)
    x = table[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    s = scales.int()
    f = torch.where(s == 255, math.nan, _power(s.clamp_max(254) - 127))
    return (x * f.unsqueeze(-1)).flatten(-2)


def _encode_tiles(k, v):
    """K, V [n, 32, heads, D] -> tiles [n, heads, tile bytes]."""
    n, _, h, d = k.shape
    ok, ov, os_ = _orders(d)
    kc, ks = _cast(k.transpose(1, 2))
    vc, vs = _cast(v.transpose(1, 2))
    vst = torch.empty(n, h, 32 * d // 32, dtype=torch.uint8, device=DEV)
    vst[..., os_.flatten()] = vs.flatten(-2)
    return torch.cat([kc[..., ok].flatten(-2), vc[..., ov].flatten(-2), ks.flatten(-2), vst], -1)


def _decode_tiles(t, d):
    """Tiles [n, heads, tile bytes] -> FP32 K, V [heads, n * 32, D]."""
    ok, ov, os_ = _orders(d)
    nb, half = d // 32, 16 * d
    t = t.transpose(0, 1)
    kc = torch.empty_like(t[..., :half].unflatten(-1, (32, d // 2)))
    kc[..., ok] = t[..., :half].unflatten(-1, (32, d // 2))
    vc = torch.empty_like(kc)
    vc[..., ov] = t[..., half:2 * half].unflatten(-1, (32, d // 2))
    ks = t[..., 2 * half:2 * half + 32 * nb].unflatten(-1, (32, nb))
    vs = t[..., 2 * half + 32 * nb:][..., os_.flatten()].unflatten(-1, (32, nb))
    return _values(kc, ks).flatten(1, 2), _values(vc, vs).flatten(1, 2)


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _place(lens, page, pages, width, rng):
    """Page tables as a server's history leaves them: pages scattered over the pool."""
    order = list(range(pages))
    rng.shuffle(order)
    tables = np.full((len(lens), width), -1, np.int32)
    refs = np.zeros(pages, np.int32)
    at = 0
    for b, n in enumerate(lens):
        m = -(-n // page)
        tables[b, :m] = order[at:at + m]
        refs[order[at:at + m]] = 1
        at += m
    return tables, refs


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device=DEV)


def _finish(st, case, pages):
    st["pages"] = pages
    if own:
        import paper_2503_13565_b200 as mxq
        st["cache"] = mxq.KVCache(pages, st["refs"], kv_heads=case.get("hkv", 1), head_dim=case.get("d", 64), page_tokens=case["page"])
    return st


def prepare(case, seed):
    op, page = case["op"], case["page"]
    lens, rows, rng = _shapes(case)
    extra = _trees(case, rows, rng) if op == "attention" and case["tree"] else _keeps(case, rows, rng) if op == "compact" else None
    g = _generator(seed)
    place = random.Random(seed)
    st = dict(case=case, lens_host=lens, rows_host=rows, page=page)
    need = [-(-n // page) for n in lens]
    if op == "resize":
        # lengths as they are; the sequences that ask for room (as many as fit into half of what is free), and how much
        room = case["pages"]
        fit = []
        for b, m in enumerate(need):
            fit.append(lens[b] if m <= room else 0)
            room -= m if fit[b] else 0
        lens = st["lens_host"] = fit
        tables, refs = _place(lens, page, case["pages"], case["W"], place)
        grown = [min(n + place.randint(1, case["grow"]), case["W"] * page) for n in lens]
        st.update(tables=_i32(tables), refs=_i32(refs), lens=_i32(lens), lens_back=_i32(lens), lens_new=_i32(grown))
        # the pool's pages are not touched: a token's worth of bytes per page stands for them
        return _finish(st, dict(case, hkv=1, d=64), torch.zeros(1, case["pages"], page // 32 * _tile_bytes(64), dtype=torch.uint8, device=DEV))
    d, hkv, layers = case["d"], case["hkv"], case["layers"]
    if op == "fork":
        src = _fork_pairs(case)
        pages = sum(need) + len(src) + 7
        tables, refs = _place(lens, page, pages, case["W"], place)
        tables = np.concatenate([tables, np.full((len(src), case["W"]), -1, np.int32)])
        both = lens + [0] * len(src)
        st.update(tables=_i32(tables), refs=_i32(refs), lens=_i32(both), lens_back=_i32(both), src=_i32(src),
                  dst=_i32([len(lens) + i for i in range(len(src))]), src_host=src)
    else:
        width = max(need) + 1
        pages = sum(need) + 3
        tables, refs = _place(lens, page, pages, width, place)
        st.update(tables=_i32(tables), refs=_i32(refs), lens=_i32(lens))
    if op == "attention":
        m, hq = case["M"], case["hq"]
        pool = torch.zeros(layers, pages, page // 32, hkv, _tile_bytes(d), dtype=torch.uint8, device=DEV)
        # keys around a direction per head, so that weights are spread over a few orders of magnitude; a first token that
        # draws weight and carries little; values with a spread of sizes from token to token
        mean = torch.randn(hkv, d, generator=g, device=DEV)
        for b, n in enumerate(lens):
            ids = st["tables"][b, :need[b]].long()
            for a in range(0, need[b], max(1, 65536 // page)):
                part = ids[a:a + max(1, 65536 // page)]
                shape = (part.numel() * (page // 32), 32, hkv, d)
                k = (torch.randn(shape, generator=g, device=DEV) + 0.5 * mean).bfloat16()
                v = (torch.randn(shape, generator=g, device=DEV) * torch.exp(torch.randn(shape[:3] + (1,), generator=g, device=DEV))).bfloat16()
                if a == 0:
                    k[0, 0], v[0, 0] = (mean * 2).bfloat16(), v[0, 0] * 0.01
                tiles = _encode_tiles(k, v).view(part.numel(), page // 32, hkv, -1)
                pool[layers - 1, part] = tiles
        q = ((torch.randn(case["B"], m, hq, d, generator=g, device=DEV) + 0.3 * mean.repeat_interleave(hq // hkv, 0)) * 2).bfloat16()
        st.update(q=q, rows=_i32(rows) if case["ragged"] else None, scale=d ** -0.5)
        st["tree"] = torch.tensor(extra, dtype=torch.int64, device=DEV) if extra else None
        _finish(st, case, pool.view(layers, pages, -1))
        if own:
            import paper_2503_13565_b200 as mxq
            st["workspace"] = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(case["B"], m, hq, hkv, d))
        return st
    if op == "append":
        m = case["M"]
        k, v = (torch.randn(case["B"], m, hkv, d, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(d, generator=g, device=DEV)) for _ in range(2))
        st.update(k=k.bfloat16(), v=v.bfloat16(), rows=_i32(rows) if case["ragged"] else None)
        return _finish(st, case, torch.zeros(layers, pages, page // 32 * hkv * _tile_bytes(d), dtype=torch.uint8, device=DEV))
    pool = torch.randint(0, 256, (layers, pages, page // 32 * hkv * _tile_bytes(d)), generator=g, dtype=torch.uint8, device=DEV)
    if op == "compact":
        keep = np.zeros((case["B"], case["M"]), np.int32)
        for b, ks in enumerate(extra):
            keep[b, :len(ks)] = ks
        st.update(rows=_i32(rows), keep=_i32(keep), kept=_i32([len(x) for x in extra]), keep_host=extra)
    _finish(st, case, pool)
    if own and op == "fork":
        import paper_2503_13565_b200 as mxq
        st["workspace"] = mxq.new_workspace(mxq.mxq_kv_fork_workspace_bytes(case["children"]))
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


# the calls of a user's program


def _own_attention(st):
    import paper_2503_13565_b200 as mxq
    out, lse = mxq.mxq_kv_attention(st["q"], st["cache"], st["case"]["layers"] - 1, st["tables"], st["lens"], rows=st["rows"], tree=st["tree"],
                                    scale=st["scale"], workspace=st["workspace"], with_lse=True)
    return {"out": out, "lse": lse}


def _own_append(st):
    import paper_2503_13565_b200 as mxq
    layer = st["case"]["layers"] - 1
    mxq.mxq_kv_append(st["cache"], layer, st["k"], st["v"], st["tables"], st["lens"], rows=st["rows"])
    k, v = mxq.mxq_kv_read(st["cache"], layer, st["tables"], st["lens"], st["case"]["M"], rows=st["rows"])
    return {"k": k, "v": v}


def _own_resize(st):
    import paper_2503_13565_b200 as mxq
    mxq.mxq_kv_resize(st["cache"], st["tables"], st["lens"], st["lens_new"])
    out = {"tables": st["tables"].clone(), "lens": st["lens"].clone(), "refs": st["refs"].clone()}
    mxq.mxq_kv_resize(st["cache"], st["tables"], st["lens"], st["lens_back"])
    return dict(out, refs_back=st["refs"])


def _own_fork(st):
    import paper_2503_13565_b200 as mxq
    mxq.mxq_kv_fork(st["cache"], st["tables"], st["lens"], st["src"], st["dst"], workspace=st["workspace"])
    out = {"tables": st["tables"].clone(), "lens": st["lens"].clone(), "refs": st["refs"].clone(), "pages": st["pages"]}
    mxq.mxq_kv_resize(st["cache"], st["tables"], st["lens"], st["lens_back"])
    return dict(out, refs_back=st["refs"])


def _own_compact(st):
    import paper_2503_13565_b200 as mxq
    lens = mxq.mxq_kv_compact(st["cache"], st["tables"], st["lens"], st["rows"], st["keep"], st["kept"])
    return {"lens": lens, "pages": st["pages"]}


# the plain forms


def _plain_attention(st):
    c = st["case"]
    d, hkv, m, hq, page = c["d"], c["hkv"], c["M"], c["hq"], c["page"]
    pool = st["pages"][c["layers"] - 1].view(-1, page // 32, hkv, _tile_bytes(d))
    out = torch.zeros(c["B"], m, hq, d, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((c["B"], m, hq), -math.inf, device=DEV)
    for b, (n, r) in enumerate(zip(st["lens_host"], st["rows_host"])):
        ids = st["tables"][b, :-(-n // page)].long()
        k, v = _decode_tiles(pool[ids].flatten(0, 1), d)
        k, v = k[:, :n], v[:, :n]
        q = st["q"][b, :r].float().transpose(0, 1).reshape(hkv, -1, d)            # [kv head, group * row, D]
        s = (q * st["scale"]) @ k.transpose(1, 2)
        j = torch.arange(n, device=DEV) - (n - r)
        if st["tree"] is None:
            seen = j <= torch.arange(r, device=DEV).unsqueeze(1)
        else:
            seen = (j < 0) | ((st["tree"][b, :r].unsqueeze(1) >> j.clamp_min(0)) & 1).bool()
        s = s.view(hkv, hq // hkv, r, n).masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = (p.flatten(1, 2) @ v).view(hkv, hq // hkv, r, d) / torch.where(total == 0, torch.ones_like(total), total)
        out[b, :r] = o.flatten(0, 1).transpose(0, 1).to(torch.bfloat16)
        lse[b, :r] = (torch.log(total) + top).squeeze(-1).flatten(0, 1).transpose(0, 1)
    return {"out": out, "lse": lse}


def _token_bytes(d):
    """Offsets in a tile of the bytes of every token: [32, D/2] K codes, [32, D/2] V codes, [32, nb] K and V scales."""
    nb = d // 32
    t = torch.arange(32, device=DEV).unsqueeze(1)
    codes = torch.arange(d // 2, device=DEV)
    return (t * (d // 2) + codes, 16 * d + t * (d // 2) + codes, 32 * d + t * nb + torch.arange(nb, device=DEV), 32 * d + 32 * nb + _orders(d)[2])


def _token_base(st, seq, pos):
    """Offset in a layer of the tiles (one per head) that hold position pos[i] of sequence seq[i], and the slots in them."""
    c = st["case"]
    page, hkv, size = c["page"], c["hkv"], _tile_bytes(c["d"])
    at = st["tables"][seq, pos // page].long() * (page // 32) + pos % page // 32
    return ((at.unsqueeze(1) * hkv) + torch.arange(hkv, device=DEV)) * size, pos % 32


def _plain_append(st):
    c = st["case"]
    ok, ov, _ = _orders(c["d"])
    off = _token_bytes(c["d"])
    flat = st["pages"][c["layers"] - 1].view(-1)
    row = torch.arange(c["M"], device=DEV)
    rows = torch.full_like(st["lens"], c["M"]) if st["rows"] is None else st["rows"]
    seq, i = torch.nonzero(row < rows.unsqueeze(1), as_tuple=True)
    base, slot = _token_base(st, seq, (st["lens"] - rows).long()[seq] + i)
    at = [base.unsqueeze(-1) + o[slot].unsqueeze(1) for o in off]
    for n, (x, order) in enumerate(((st["k"], ok), (st["v"], ov))):
        codes, scales = _cast(x[seq, i])
        flat[at[n]] = codes[..., order]
        flat[at[2 + n]] = scales
    out = [torch.zeros_like(st["k"]), torch.zeros_like(st["v"])]
    for n, order in enumerate((ok, ov)):
        stored = flat[at[n]]
        codes = torch.empty_like(stored)
        codes[..., order] = stored
        out[n][seq, i] = _values(codes, flat[at[2 + n]]).to(torch.bfloat16)
    return {"k": out[0], "v": out[1]}


def _resize_plain(tables, lens, refs, new, page):
    width = tables.shape[1]
    valid = (new >= 0) & (new <= width * page)
    col = torch.arange(width, device=DEV)
    have = (lens + page - 1) // page
    want = torch.where(valid, (new + page - 1) // page, have)
    drop = (col >= want.unsqueeze(1)) & (col < have.unsqueeze(1))
    refs.index_add_(0, tables.clamp_min(0).flatten().long(), -drop.int().flatten())
    tables[:] = torch.where(drop, torch.full_like(tables, -1), tables)
    need = (want - have).clamp_min(0)
    upto = need.cumsum(0)
    free = torch.sort((refs != 0).int(), stable=True).indices
    fits = valid & ((need == 0) | (upto <= (refs == 0).sum()))
    take = (col >= have.unsqueeze(1)) & (col < want.unsqueeze(1)) & fits.unsqueeze(1)
    rank = (upto - need - have).unsqueeze(1) + col
    page_of = free[rank.clamp(0, refs.numel() - 1).long()].int()
    tables[:] = torch.where(take, page_of, tables)
    refs.index_add_(0, tables.clamp_min(0).flatten().long(), take.int().flatten())
    lens[:] = torch.where(fits, new, lens)


def _plain_resize(st):
    _resize_plain(st["tables"], st["lens"], st["refs"], st["lens_new"], st["page"])
    out = {"tables": st["tables"].clone(), "lens": st["lens"].clone(), "refs": st["refs"].clone()}
    _resize_plain(st["tables"], st["lens"], st["refs"], st["lens_back"], st["page"])
    return dict(out, refs_back=st["refs"])


def _plain_fork(st):
    c = st["case"]
    page, tables, lens, refs = st["page"], st["tables"], st["lens"], st["refs"]
    src, dst = st["src"].long(), st["dst"].long()
    n = lens[src]
    whole, part = n // page, n % page
    need = (part > 0).int()
    upto = need.cumsum(0)
    free = torch.sort((refs != 0).int(), stable=True).indices
    fits = (need == 0) | (upto <= (refs == 0).sum())
    col = torch.arange(tables.shape[1], device=DEV)
    share = (col < whole.unsqueeze(1)) & fits.unsqueeze(1)
    fresh = free[(upto - 1).clamp(0, refs.numel() - 1).long()].int()
    rows = torch.where(share, tables[src], torch.full_like(tables[src], -1))
    last = (col == whole.unsqueeze(1)) & (fits & (part > 0)).unsqueeze(1)
    old = torch.gather(tables[src], 1, whole.clamp_max(tables.shape[1] - 1).long().unsqueeze(1)).squeeze(1)
    rows = torch.where(last, fresh.unsqueeze(1), rows)
    tables[dst] = rows
    lens[dst] = torch.where(fits, n, torch.zeros_like(n))
    refs.index_add_(0, rows.clamp_min(0).flatten().long(), (share | last).int().flatten())
    tiles = c["hkv"] * _tile_bytes(c["d"])
    pool = st["pages"].view(c["layers"], -1, page // 32, tiles)
    for i, s in enumerate(st["src_host"]):
        filled = -(-(st["lens_host"][s] % page) // 32)
        if filled:
            pool[:, fresh[i], :filled] = pool[:, old[i], :filled]
    out = {"tables": tables.clone(), "lens": lens.clone(), "refs": refs.clone(), "pages": st["pages"]}
    _resize_plain(tables, lens, refs, st["lens_back"], page)
    return dict(out, refs_back=refs)


def _plain_compact(st):
    c = st["case"]
    flat = st["pages"].view(c["layers"], -1)
    off = torch.cat(_token_bytes(c["d"]), 1)
    seq, to = torch.nonzero(torch.arange(c["M"], device=DEV) < st["kept"].unsqueeze(1), as_tuple=True)
    first = (st["lens"] - st["rows"]).long()[seq]
    base, slot = _token_base(st, seq, first + st["keep"].long()[seq, to])
    moved = flat[:, base.unsqueeze(-1) + off[slot].unsqueeze(1)]
    base, slot = _token_base(st, seq, first + to)
    flat[:, base.unsqueeze(-1) + off[slot].unsqueeze(1)] = moved
    return {"lens": st["lens"] - st["rows"] + st["kept"], "pages": st["pages"]}


_own = {"attention": _own_attention, "append": _own_append, "resize": _own_resize, "fork": _own_fork, "compact": _own_compact}
_plain = {"attention": _plain_attention, "append": _plain_append, "resize": _plain_resize, "fork": _plain_fork, "compact": _plain_compact}


# ---- from the definition, in 64 bits ------------------------------------------------------------------------------------


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_value(code, scale):
    """Value of an E2M1 nibble under an E8M0 scale, from the format's fields (sign, two exponent bits, one of mantissa)."""
    e, m = (code >> 1) & 3, (code & 1).double()
    mag = torch.where(e == 0, m * 0.5, (1 + m * 0.5) * _exact_power(e - 1))
    val = torch.where((code & 8) != 0, -mag, mag) * _exact_power(scale - 127)
    return torch.where(scale == 255, torch.full_like(val, math.nan), val)


def _exact_rows(tiles, d, which):
    """tiles [n, bytes] of one head -> [n * 32, D] in 64 bits; which = 0 for K, 1 for V."""
    nb, half = d // 32, 16 * d
    e = torch.arange(d, device=DEV)
    j, inside = e // 32, (e % 32) // 2
    if which == 0:
        byte = (inside // 4) * 4 * nb + 4 * j + inside % 4
    else:
        byte = (inside // 2) * 2 * nb + 2 * j + inside % 2
    t = torch.arange(32, device=DEV).unsqueeze(1)
    code = tiles[:, which * half + t * (d // 2) + byte].int()
    code = torch.where(e % 2 == 1, code >> 4, code & 15)
    if which == 0:
        place = 2 * half + t * nb + j
    else:
        place = 2 * half + 32 * nb + (t // 16) * 16 * nb + (t & 3) * 4 * nb + ((t >> 3) & 1) * 2 * nb + 2 * j + ((t >> 2) & 1)
    return _exact_value(code, tiles[:, place].int()).flatten(0, 1)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op, page = case["op"], case["page"]
    lens, rows = st["lens_host"], st["rows_host"]
    if op == "attention":
        return _exact_attention(case, st, lens, rows)
    if op == "append":
        out = {}
        for name in ("k", "v"):
            x = st[name].double().unflatten(-1, (-1, 32))
            top = x.abs().amax(-1, keepdim=True)
            unit = _exact_power((torch.frexp(top).exponent - 3).clamp_min(-127))     # top = mantissa in [1/2, 1) times 2^exponent
            m = (x.abs() / unit).clamp_max(6)
            step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
            val = torch.round(m / step) * step * unit * torch.sign(x)      # ties to even multiples, which are the even codes
            val = val.flatten(-2)
            for b, r in enumerate(rows):
                val[b, r:] = 0
            out[name] = val
        return out
    tables, refs = st["tables"].cpu().numpy().copy(), st["refs"].cpu().numpy().copy()
    if op == "resize":
        cur, new = list(lens), st["lens_new"].tolist()
        free = [p for p in range(case["pages"]) if refs[p] == 0]
        full = False
        for b, n in enumerate(new):
            have, want = -(-cur[b] // page), -(-n // page)
            if want > have and (full or want - have > len(free)):
                full = True
                continue
            for w in range(have, want):
                tables[b, w] = free.pop(0)
                refs[tables[b, w]] += 1
            cur[b] = n
        as64 = lambda x: torch.tensor(np.asarray(x, np.int64))
        return {"tables": as64(tables), "lens": as64(cur), "refs": as64(refs), "refs_back": st["refs"].long().cpu()}
    if op == "fork":
        pool, cur = st["pages"].clone(), lens + [0] * len(st["src_host"])
        size = case["hkv"] * _tile_bytes(case["d"])
        for i, s in enumerate(st["src_host"]):
            child, n = len(lens) + i, lens[s]
            for w in range(-(-n // page)):
                p = int(tables[s, w])
                if (w + 1) * page > n:
                    q = int(np.flatnonzero(refs == 0)[0])
                    filled = -(-(n % page) // 32) * size
                    pool[:, q, :filled] = st["pages"][:, p, :filled]
                    p = q
                tables[child, w] = p
                refs[p] += 1
            cur[child] = n
        as64 = lambda x: torch.tensor(np.asarray(x, np.int64))
        return {"tables": as64(tables), "lens": as64(cur), "refs": as64(refs), "pages": pool, "refs_back": st["refs"].long().cpu()}
    # compact: token by token
    d, nb, hkv = case["d"], case["d"] // 32, case["hkv"]
    old = st["pages"].view(case["layers"], -1, page // 32, hkv, _tile_bytes(d))
    new = old.clone()
    for b, ks in enumerate(st["keep_host"]):
        first = lens[b] - rows[b]
        for to, ki in enumerate(ks):
            for base in (0, 16 * d):
                _move(new, old, tables[b], page, first + to, first + ki, lambda t: slice(base + t * (d // 2), base + (t + 1) * (d // 2)))
            _move(new, old, tables[b], page, first + to, first + ki, lambda t: slice(32 * d + t * nb, 32 * d + (t + 1) * nb))
            v0 = 32 * d + 32 * nb
            _move(new, old, tables[b], page, first + to, first + ki,
                  lambda t: [v0 + (t // 16) * 16 * nb + (t & 3) * 4 * nb + ((t >> 3) & 1) * 2 * nb + 2 * j + ((t >> 2) & 1) for j in range(nb)])
    return {"lens": torch.tensor([n - r + len(k) for n, r, k in zip(lens, rows, st["keep_host"])]), "pages": new.view_as(st["pages"])}


def _move(new, old, table, page, to, at, where):
    new[:, int(table[to // page]), to % page // 32, :, where(to % 32)] = old[:, int(table[at // page]), at % page // 32, :, where(at % 32)]


def _exact_attention(case, st, lens, rows):
    d, hkv, m, hq, page = case["d"], case["hkv"], case["M"], case["hq"], case["page"]
    group = hq // hkv
    pool = st["pages"][case["layers"] - 1].view(-1, page // 32, hkv, _tile_bytes(d))
    out = torch.zeros(case["B"], m, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((case["B"], m, hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, r) in enumerate(zip(lens, rows)):
        ids = st["tables"][b, :-(-n // page)].long()
        pos = torch.arange(n, device=DEV).expand(r, n)
        row = torch.arange(r, device=DEV).unsqueeze(1)
        drafted = pos - (n - r)
        if st["tree"] is None:
            hidden = drafted > row
        else:
            bits = st["tree"][b, :r].unsqueeze(1).expand(r, n)
            hidden = (drafted >= 0) & (torch.bitwise_right_shift(bits, drafted.clamp_min(0)) % 2 == 0)
        for h in range(hkv):
            tiles = pool[ids, :, h].flatten(0, 1)
            k, v = _exact_rows(tiles, d, 0)[:n], _exact_rows(tiles, d, 1)[:n]
            for a in range(group):
                s = st["q"][b, :r, h * group + a].double() @ k.T * st["scale"]
                s[hidden] = -math.inf
                z = torch.logsumexp(s, -1)
                w = torch.exp(s - torch.where(torch.isinf(z), torch.zeros_like(z), z).unsqueeze(1))
                out[b, :r, h * group + a] = w @ v
                lse[b, :r, h * group + a] = z
    return {"out": out, "lse": lse}
