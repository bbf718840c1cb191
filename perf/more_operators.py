"""What a decoder step needs beside its 4-bit linear layers and its 4-bit cache, as a user's program calls it: the norm with the
residual's addition, rotated queries and keys on their way into the cache, low-rank adapters beside the shared weights, and the rules
that a server applies to logits before it takes their argmax.  Plain forms, work, and definitions in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"


# ---- cases --------------------------------------------------------------------------------------------------------------


def listed():
    return [
        # the norm ahead of a draft step's projections, one token: latency counts
        dict(name="norm_decode_1x4096", op="norm", M=1, K=4096, x="bf16", residual="bf16", weight="bf16", y=True, pair=False),
        # after a projection that returns FP32 sums, rows of a verification; a consumer that takes 8 bits
        dict(name="norm_verify_16x5120_pair", op="norm", M=16, K=5120, x="f32", residual="bf16", weight="f32", y=False, pair=True),
        # long prompts, both outputs: the largest
        dict(name="norm_prompt_8191x8192_both", op="norm", M=8191, K=8192, x="bf16", residual="bf16", weight="bf16", y=True, pair=True),
        # one draft step's new row of one sequence, grouped heads
        dict(name="rope_decode_1x1_h32_8", op="rope", B=1, M=1, hq=32, hkv=8, d=128, rot=128, style="halves", page=64, lo=1900, hi=2100,
             table=4096, ragged=False, tree=False, shape_seed=1),
        # proposals of a batch as trees: positions by depth, part of the head rotated, neighbouring pairs, fewer rows in some sequences
        dict(name="rope_tree_61x9_h16_4_d64", op="rope", B=61, M=9, hq=16, hkv=4, d=64, rot=32, style="pairs", page=32, lo=100, hi=6000,
             table=8192, ragged=True, tree=True, shape_seed=2),
        # prompts of different lengths
        dict(name="rope_prompt_3x8191_h32_8", op="rope", B=3, M=8191, hq=32, hkv=8, d=128, rot=128, style="halves", page=64, lo=8191, hi=9000,
             table=131072, ragged=True, tree=False, shape_seed=3),
        # verification of eight proposals of one sequence, penalties only
        dict(name="accept_1x8_v32000", op="accept", B=1, T=8, extra=1, V=32000, dtype="f32", history=700, bias=0, masks=False, shape_seed=4),
        # a batch under grammars, with biases; BF16 logits of a large vocabulary
        dict(name="accept_24x7_v128256_masks", op="accept", B=24, T=7, extra=1, V=128256, dtype="bf16", history=5000, bias=200, masks=True, shape_seed=5),
        # the first token after prompts: counts are built, the adjusted logits go to a sampler; an odd vocabulary
        dict(name="first_token_48_v32001", op="first", B=48, V=32001, dtype="f32", prompt=20000, bias=30, masks=True, shape_seed=6),
        # one token through a shared 4-bit projection with its adapter
        dict(name="lora_decode_1_r16_4096x4096", op="lora", M=1, N=4096, K=4096, r=16, L=8, shared=True, out="f32", none=False, shape_seed=7),
        # a decoding batch of many adapters
        dict(name="lora_decode_16_r32_11008x4096", op="lora", M=16, N=11008, K=4096, r=32, L=24, shared=True, out="bf16", none=True, shape_seed=8),
        # prompts of several requests, beside a projection computed elsewhere
        dict(name="lora_prompt_4095_r64_4096x4096", op="lora", M=4095, N=4096, K=4096, r=64, L=6, shared=False, out="bf16", none=True, shape_seed=9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "rope", "rope", "accept", "accept", "first", "lora", "lora", "lora"])
    seed = rng.randrange(1 << 30)
    if op == "norm":
        k = 32 * _log_int(rng, 8, 512)
        m = min(_log_int(rng, 1, 12000), (1 << 26) // k)
        y = rng.random() < 0.7
        return dict(op=op, M=m, K=k, x=rng.choice(["bf16", "f32"]), residual=rng.choice(["none", "bf16", "bf16", "f32"]),
                    weight=rng.choice(["bf16", "f32"]), y=y, pair=not y or rng.random() < 0.4)
    if op == "rope":
        hq, hkv = rng.choice([(32, 32), (32, 8), (12, 4), (9, 3), (16, 1), (8, 8)])
        d = rng.choice([64, 128, 128])
        rot = rng.choice([d, d, d // 2, d // 4])
        m = rng.choice([1, 1, 3, 9, 16, _log_int(rng, 17, 6000)])
        b = max(1, min(_log_int(rng, 1, 256), 20000 * 48 // (m * (hq + 2 * hkv))))
        hi = m + _log_int(rng, 1, 4000)
        return dict(op=op, B=b, M=m, hq=hq, hkv=hkv, d=d, rot=rot, style=rng.choice(["halves", "halves", "pairs"]), page=rng.choice([32, 64, 128]),
                    lo=m, hi=hi, table=hi + _log_int(rng, 1, 100000), ragged=m > 1 and rng.random() < 0.5, tree=1 < m <= 16 and rng.random() < 0.5,
                    shape_seed=seed)
    if op == "accept":
        v = _log_int(rng, 1000, 200000)
        t = rng.choice([0, 1, 2, 4, 7, 8, 16])
        b = max(1, min(_log_int(rng, 1, 128), 24 * 8 * 128256 // (v * (t + 1))))
        return dict(op=op, B=b, T=t, extra=1 if t == 0 else rng.choice([1, 1, 0]), V=v, dtype=rng.choice(["f32", "bf16"]),
                    history=_log_int(rng, 1, 20000), bias=rng.choice([0, 1, 300]), masks=rng.random() < 0.5, shape_seed=seed)
    if op == "first":
        v = _log_int(rng, 1000, 200000)
        b = max(1, min(_log_int(rng, 1, 96), 48 * 100000 // v))
        return dict(op=op, B=b, V=v, dtype=rng.choice(["f32", "bf16"]), prompt=_log_int(rng, 1, 20000), bias=rng.choice([0, 10, 300]),
                    masks=rng.random() < 0.5, shape_seed=seed)
    r = rng.choice([8, 16, 16, 24, 32, 64, 128])
    n, k = rng.choice([(4096, 4096), (768, 768), (11008, 4096), (4096, 11008), (5120, 5120), (1025, 96), (2000, 1312)])
    shared = rng.random() < 0.6
    m = rng.randint(1, 16) if shared else _log_int(rng, 1, 4095)
    return dict(op=op, M=m, N=n, K=k, r=r, L=_log_int(rng, 1, 32) if m * r < 65536 else _log_int(rng, 1, 6), shared=shared,
                out=rng.choice(["f32", "bf16"]), none=rng.random() < 0.5, shape_seed=seed)


def _kind(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _size(name):
    return {"none": 0, "bf16": 2, "f32": 4}[name]


def _lengths(case):
    """Tokens and rows of a case's sequences, as its user's scheduler knows them on the host."""
    rng = random.Random(case["shape_seed"])
    lens = [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["B"])]
    rows = [rng.randint(1, case["M"]) if case["ragged"] else case["M"] for _ in lens]
    return lens, rows


def _depths(case, rows):
    """Depths of the nodes of token trees; the root is node 0 and has depth 0."""
    rng = random.Random(case["shape_seed"] + 1)
    out = []
    for n in rows:
        d = [0]
        for i in range(1, n):
            d.append(d[rng.randrange(max(0, i - 5), i)] + 1)
        out.append(d + [0] * (case["M"] - n))
    return out


def _histories(case):
    """How many tokens every sequence has: from a hundredth of the longest to all of it."""
    rng = random.Random(case["shape_seed"])
    top = case["history"] if case["op"] == "accept" else case["prompt"]
    return [_log_int(rng, max(1, top // 100), top) for _ in range(case["B"])]


def _owners(case):
    """The adapter of every row: rows of a prompt lie together, decoding rows come as they come; -1 is none."""
    rng = random.Random(case["shape_seed"])
    if case["M"] <= 64:
        ids = [rng.randrange(case["L"]) for _ in range(case["M"])]
    else:
        cuts = sorted(rng.randrange(case["M"]) for _ in range(case["L"] - 1))
        ids = [a for a, (lo, hi) in enumerate(zip([0] + cuts, cuts + [case["M"]])) for _ in range(hi - lo)]
    if case["none"]:
        for i in rng.sample(range(case["M"]), case["M"] // 8):
            ids[i] = -1
    return ids


def work(case):
    op = case["op"]
    if op == "norm":
        m, k = case["M"], case["K"]
        each = _size(case["x"]) + 2 * _size(case["residual"]) + 2 * case["y"]
        # the pair is written, read again, and the values that it stands for are written
        return {"bytes": m * k * each + k * _size(case["weight"]) + (m * k * (2 + 2 / 32 + 2) if case["pair"] else 0), "flops": 6 * m * k}
    if op == "rope":
        _, rows = _lengths(case)
        n, d = sum(rows), case["d"]
        kv = case["hkv"] * d
        cache = 2 * kv * 17 / 32
        # rotated queries read and written; keys and values read, their 4-bit form written, read again and returned
        return {"bytes": n * (4 * case["hq"] * d + 4 * kv + 2 * cache + 4 * case["rot"]) + 4 * case["B"] * case["M"] * kv,
                "flops": 3 * n * (case["hq"] + case["hkv"]) * case["rot"] + 4 * n * kv}
    if op in ("accept", "first"):
        b, v = case["B"], case["V"]
        rows = case["T"] + case["extra"] if op == "accept" else 1
        n = b * rows * v
        each = _size(case["dtype"]) * (1 if op == "accept" else 2) + (1 / 8 if case["masks"] else 0)
        return {"bytes": int(n * each) + 4 * b * v + 8 * b * case["bias"] + (sum(_histories(case)) * 4 if op == "first" else 0), "flops": 4 * n}
    m, n, k, r = case["M"], case["N"], case["K"], case["r"]
    ids = [a for a in _owners(case) if a >= 0]
    out = _size(case["out"])
    return {"bytes": 2 * m * k + 2 * len(set(ids)) * r * (n + k) + m * n * out + (n * k * 17 // 32 if case["shared"] else m * n * out),
            "flops": 2 * len(ids) * r * (n + k) + (2 * m * n * k if case["shared"] else 0)}


# ---- formats (plain) ----------------------------------------------------------------------------------------------------


def _power(e):
    """2^e in FP32 for whole e in -127..127, from the format's fields."""
    bits = torch.where(e == -127, torch.full_like(e, 1 << 22), (e + 127) << 23)
    return bits.int().view(torch.float32)


def _blocks(x, below):
    """FP32 blocks of 32 and the exponent of their scale: 2^(floor(log2 max) - below), at least 2^-127; and which blocks are finite."""
    x = x.unflatten(-1, (-1, 32))
    finite = torch.isfinite(x).all(-1, keepdim=True)
    x = torch.where(finite, x, torch.zeros_like(x))
    top = x.abs().amax(-1, keepdim=True)
    return x, ((top.view(torch.int32) >> 23) - below).clamp_min(0) - 127, finite


def _through_fp4(x):
    """The values that FP32 [..., D] has after the direct cast to MXFP4."""
    x, e, finite = _blocks(x, 2)
    a = x.abs() * _power(-e)
    code = (a > 0.25).float() * 0.5 + (a >= 0.75).float() * 0.5 + (a > 1.25).float() * 0.5 + (a >= 1.75).float() * 0.5 + \
        (a > 2.5).float() + (a >= 3.5).float() + (a > 5).float() * 2
    value = torch.copysign(code, x) * _power(e)
    return torch.where(finite, value, torch.full_like(value, math.nan)).flatten(-2)


def _through_fp8(x):
    """The values that FP32 [..., K] has after the cast to MXFP8 (E4M3)."""
    x, e, finite = _blocks(x, 8)
    a = x.abs() * _power(-e)
    step = _power(((a.view(torch.int32) >> 23) - 127).clamp_min(-6) - 3)
    value = torch.copysign((torch.round(a / step) * step).clamp_max(448), x) * _power(e)
    return torch.where(finite, value, torch.full_like(value, math.nan)).flatten(-2)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _weights(codes, scales):
    """FP32 [N, K] of an MXFP4 pair."""
    table = torch.tensor([[_E2M1[b & 15], _E2M1[b >> 4]] for b in range(256)], device=DEV)
    return (table[codes.int()].flatten(-2).unflatten(-1, (-1, 32)) * _power(scales.int() - 127).unsqueeze(-1)).flatten(-2)


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prepare_norm(case, g):
    m, k = case["M"], case["K"]
    # a residual stream: a few channels carry large values, rows differ in size
    channel = torch.exp(1.2 * torch.randn(k, generator=g, device=DEV))
    x = torch.randn(m, k, generator=g, device=DEV) * channel
    x = (x * torch.exp(0.5 * torch.randn(m, 1, generator=g, device=DEV))).to(_kind(case["x"]))
    st = dict(x=x, residual=None, weight=(1 + 0.3 * torch.randn(k, generator=g, device=DEV)).to(_kind(case["weight"])), eps=1e-5)
    if case["residual"] != "none":
        st["residual"] = (torch.randn(m, k, generator=g, device=DEV) * channel * 3).to(_kind(case["residual"]))
        st["sum"] = torch.empty_like(st["residual"])
    return st


def _prepare_rope(case, g):
    b, m, d, hkv, page = case["B"], case["M"], case["d"], case["hkv"], case["page"]
    lens, rows = _lengths(case)
    i = torch.arange(case["rot"] // 2, device=DEV, dtype=torch.float64)
    angle = torch.arange(case["table"], device=DEV, dtype=torch.float64).unsqueeze(1) * 10000.0 ** (-2 * i / case["rot"])
    st = dict(table=torch.cat([torch.cos(angle), torch.sin(angle)], 1).float(), lens=_i32(lens), rows=_i32(rows) if case["ragged"] else None,
              positions=None)
    if case["tree"]:
        depth = _i32(_depths(case, rows))
        st["positions"] = (st["lens"] - _i32(rows)).unsqueeze(1) + depth
    # one fused projection's output, of which queries, keys and values are slices
    channel = torch.exp(0.7 * torch.randn((case["hq"] + 2 * hkv), d, generator=g, device=DEV))
    qkv = (torch.randn(b, m, case["hq"] + 2 * hkv, d, generator=g, device=DEV) * channel).bfloat16()
    st.update(q=qkv[:, :, :case["hq"]], k=qkv[:, :, case["hq"]:case["hq"] + hkv], v=qkv[:, :, case["hq"] + hkv:])
    if own:
        import paper_2503_13565_b200 as mxq
        need = [-(-n // page) for n in lens]
        at = torch.randperm(sum(need), generator=g, device=DEV).int()
        tables = torch.full((b, max(need)), -1, dtype=torch.int32, device=DEV)
        tables[torch.arange(max(need), device=DEV) < _i32(need).unsqueeze(1)] = at
        cache = mxq.KVCache.new(1, sum(need), hkv, d, page)
        cache.refs.fill_(1)
        st.update(cache=cache, tables=tables, rope=mxq.Rope(st["table"], case["style"]))
    return st


def _prepare_logits(case, g):
    b, v = case["B"], case["V"]
    r = case["T"] + case["extra"] if case["op"] == "accept" else 1
    rng = random.Random(case["shape_seed"] + 1)
    n = _i32(_histories(case))
    # histories that repeat themselves: frequent tokens are much more frequent
    longest = max(_histories(case))
    tokens = (v * torch.rand(b, longest, generator=g, device=DEV) ** 6).int().clamp_max(v - 1)
    logits = 2.5 * torch.randn(b, r, v, generator=g, device=DEV)
    penalties = torch.stack([1 + 0.4 * torch.rand(b, generator=g, device=DEV), 0.8 * torch.rand(b, generator=g, device=DEV),
                             0.3 * torch.rand(b, generator=g, device=DEV)], 1)
    penalties[0] = torch.tensor([1.0, 0.0, 0.0], device=DEV)                    # a request without penalties
    st = dict(tokens=tokens, n=n, penalties=penalties, bias_tokens=None, bias_values=None, allowed=None, draft=None)
    chosen = torch.randint(0, v, (b, r), generator=g, device=DEV)
    logits.scatter_(2, chosen.unsqueeze(-1), 40.0)                              # what the model is sure of
    if case["bias"]:
        st["bias_tokens"] = torch.randint(-1, v, (b, case["bias"]), generator=g, device=DEV, dtype=torch.int32)
        st["bias_values"] = 3 * torch.randn(b, case["bias"], generator=g, device=DEV)
    if case["masks"]:
        words = -(-v // 32)
        few = torch.randint(-2 ** 31, 2 ** 31, (4, b, r, words), generator=g, device=DEV).int()
        some = few[0] & few[1] & few[2] & few[3]                                # one token of sixteen is allowed
        word = some.gather(2, (chosen // 32).unsqueeze(-1))
        bit = (torch.ones_like(chosen) << (chosen % 32)).unsqueeze(-1)
        some.scatter_(2, (chosen // 32).unsqueeze(-1), (word.long() | torch.where(bit >= 2 ** 31, bit - 2 ** 32, bit)).int())
        free = torch.rand(b, 1, 1, generator=g, device=DEV) < 0.3               # inside a string everything is allowed
        some = torch.where(free, torch.full_like(some, -1), some)
        if rng.random() < 0.5:
            some[b - 1, r - 1] = 0                                              # a grammar that has ended allows nothing
        st["allowed"] = some
        hidden = ((some[..., 0] & 1) == 0)
        logits[..., 0] = torch.where(hidden, torch.full_like(logits[..., 0], math.nan), logits[..., 0])
    st["logits"] = logits.to(_kind(case["dtype"]))
    st["counts"] = torch.zeros(b, v, dtype=torch.int32, device=DEV)
    if case["op"] == "accept":
        if case["T"]:
            stop = torch.randint(0, case["T"] + 1, (b, 1), generator=g, device=DEV)
            other = torch.randint(0, v, (b, case["T"]), generator=g, device=DEV)
            st["draft"] = torch.where(torch.arange(case["T"], device=DEV) < stop, chosen[:, :case["T"]], other).int()
        part = torch.arange(longest, device=DEV) < n.unsqueeze(1)
        prompt = torch.arange(longest, device=DEV) < (n // 2).unsqueeze(1)
        made = torch.zeros(b, v, dtype=torch.int32, device=DEV).scatter_add_(1, tokens.long(), (part & ~prompt).int())
        seen = torch.zeros(b, v, dtype=torch.int32, device=DEV).scatter_add_(1, tokens.long(), prompt.int())
        st["counts"] = torch.where(seen > 0, made.long() - 2 ** 31, made.long()).int()
    if own:
        import paper_2503_13565_b200 as mxq
        st["rules"] = mxq.LogitRules(counts=st["counts"], penalties=penalties, bias_tokens=st["bias_tokens"], bias_values=st["bias_values"],
                                     allowed=st["allowed"])
        if case["op"] == "accept":
            st["workspace"] = mxq.new_workspace(mxq.mxq_greedy_accept_rules_workspace_bytes(b, r, v))
    return st


def _prepare_lora(case, g):
    m, n, k, r, count = case["M"], case["N"], case["K"], case["r"], case["L"]
    st = dict(x=torch.randn(m, k, generator=g, device=DEV).bfloat16(), a=(torch.randn(count, r, k, generator=g, device=DEV) / k ** 0.5).bfloat16(),
              b=(0.02 * torch.randn(count, n, r, generator=g, device=DEV)).bfloat16(), scale=1 + torch.rand(count, generator=g, device=DEV),
              ids=_i32(_owners(case)))
    if case["shared"]:
        st["codes"] = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
        st["scales"] = torch.randint(117, 121, (n, k // 32), generator=g, device=DEV, dtype=torch.uint8)
    else:
        st["base"] = torch.randn(m, n, generator=g, device=DEV).to(_kind(case["out"]))
    if own:
        import paper_2503_13565_b200 as mxq
        size = mxq.mxq_linear_lora_workspace_bytes(m, n, k, r, count) if case["shared"] else mxq.mxq_lora_workspace_bytes(m, n, k, r, count)
        st["workspace"] = mxq.new_workspace(size)
    return st


def prepare(case, seed):
    g = _generator(seed)
    st = {"norm": _prepare_norm, "rope": _prepare_rope, "accept": _prepare_logits, "first": _prepare_logits, "lora": _prepare_lora}[case["op"]](case, g)
    return dict(st, case=case)


# ---- one pass -----------------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


# the calls of a user's program


def _own_norm(st):
    import paper_2503_13565_b200 as mxq
    c, out = st["case"], {}
    got = mxq.mxq_rmsnorm(st["x"], st["weight"], st["eps"], residual=st["residual"], residual_out=st.get("sum"), bf16=c["y"], mxfp8=c["pair"])
    got = got if isinstance(got, tuple) else (got,)
    if c["y"]:
        out["y"] = got[0]
    if c["pair"]:
        out["v8"] = mxq.mxq_dequantize_mxfp8(*got[-2:])
    if st["residual"] is not None:
        out["sum"] = st["sum"]
    return out


def _own_rope(st):
    import paper_2503_13565_b200 as mxq
    q = mxq.mxq_kv_append_rope(st["cache"], 0, st["q"], st["k"], st["v"], st["tables"], st["lens"], st["rope"], rows=st["rows"],
                               positions=st["positions"])
    k, v = mxq.mxq_kv_read(st["cache"], 0, st["tables"], st["lens"], st["case"]["M"], rows=st["rows"])
    return {"q": q, "k": k, "v": v}


def _own_accept(st):
    import paper_2503_13565_b200 as mxq
    verifier, accepted, following = mxq.mxq_greedy_accept_rules(st["logits"], st["draft"], st["rules"], workspace=st["workspace"])
    return {"verifier": verifier, "accepted": accepted, "next": following}


def _own_first(st):
    import paper_2503_13565_b200 as mxq
    st["counts"].zero_()
    mxq.mxq_token_counts(st["counts"], st["tokens"], st["n"], prompt=True)
    return {"logits": mxq.mxq_logits_adjust(st["logits"], st["rules"]), "counts": st["counts"]}


def _own_lora(st):
    import paper_2503_13565_b200 as mxq
    kind = _kind(st["case"]["out"])
    if st["case"]["shared"]:
        return mxq.mxq_linear_lora(st["x"], st["codes"], st["scales"], st["a"], st["b"], st["ids"], scale=st["scale"], out_dtype=kind,
                                   workspace=st["workspace"])
    return mxq.mxq_lora(st["x"], st["a"], st["b"], st["ids"], scale=st["scale"], base=st["base"], out_dtype=kind, workspace=st["workspace"])


# the plain forms


def _plain_norm(st):
    c, out = st["case"], {}
    h = st["x"].float()
    if st["residual"] is not None:
        h = h + st["residual"].float()
        out["sum"] = h.to(st["residual"].dtype)
    y = h * (1 / torch.sqrt(h.square().mean(-1, keepdim=True) + st["eps"])) * st["weight"].float()
    if c["y"]:
        out["y"] = y.bfloat16()
    if c["pair"]:
        out["v8"] = _through_fp8(y).bfloat16()
    return out


def _row_positions(st):
    """Position of every row, and which rows there are."""
    m = st["case"]["M"]
    rows = torch.full_like(st["lens"], m) if st["rows"] is None else st["rows"]
    i = torch.arange(m, device=DEV)
    at = (st["lens"] - rows).unsqueeze(1) + i if st["positions"] is None else st["positions"]
    return at, i < rows.unsqueeze(1)


def _rotate(x, cos, sin, style):
    half = cos.shape[-1]
    x = x.float()
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    one, two = (turned[..., :half], turned[..., half:]) if style == "halves" else (turned[..., 0::2], turned[..., 1::2])
    first, second = one * cos - two * sin, two * cos + one * sin
    turned = torch.cat([first, second], -1) if style == "halves" else torch.stack([first, second], -1).flatten(-2)
    return torch.cat([turned, rest], -1)


def _plain_rope(st):
    c = st["case"]
    at, there = _row_positions(st)
    row = st["table"][at.clamp(0, c["table"] - 1).long()].unsqueeze(2)
    cos, sin = row[..., :c["rot"] // 2], row[..., c["rot"] // 2:]
    q, k = _rotate(st["q"], cos, sin, c["style"]), _through_fp4(_rotate(st["k"], cos, sin, c["style"]))
    v = _through_fp4(st["v"].float())
    there = there.unsqueeze(-1).unsqueeze(-1)
    return {n: torch.where(there, x, torch.zeros_like(x)).bfloat16() for n, x in (("q", q), ("k", k), ("v", v))}


def _adjusted(st, counts):
    """Logits after the rules, FP32 [B, R, V]; `counts` int32 [B, V]."""
    b, r, v = st["logits"].shape
    x = st["logits"].float()
    made = (counts & 0x7FFFFFFF).unsqueeze(1).expand(b, r, v)
    if st["draft"] is not None:          # row i also counts the proposals before it
        t = st["draft"].shape[1]
        each = torch.zeros(b, t, v, dtype=torch.int32, device=DEV).scatter_(2, st["draft"].long().unsqueeze(-1), 1)
        made = made + torch.cat([torch.zeros_like(each[:, :1]), each.cumsum(1, dtype=torch.int32)], 1)[:, :r]
    repetition, presence, frequency = (st["penalties"][:, i].view(b, 1, 1) for i in range(3))
    again = (counts < 0).unsqueeze(1) | (made > 0)
    x = torch.where(again, torch.where(x > 0, x / repetition, x * repetition), x)
    x = torch.where(made > 0, x - frequency * made.float() - presence, x)
    if st["bias_tokens"] is not None:    # of entries with the same token the last one counts
        j = torch.arange(st["bias_tokens"].shape[1], device=DEV).expand_as(st["bias_tokens"])
        token = torch.where(st["bias_tokens"] < 0, v, st["bias_tokens"]).long()
        last = torch.full((b, v + 1), -1, dtype=torch.int64, device=DEV).scatter_reduce(1, token, j, "amax")[:, :v]
        x = torch.where((last >= 0).unsqueeze(1), x + st["bias_values"].gather(1, last.clamp_min(0)).unsqueeze(1), x)
    if st["allowed"] is not None:
        i = torch.arange(v, device=DEV)
        x = torch.where((st["allowed"][..., i // 32] >> (i % 32).int()) & 1 == 0, torch.full_like(x, -math.inf), x)
    return x


def _plain_accept(st):
    b, r, v = st["logits"].shape
    x = _adjusted(st, st["counts"])
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top = x.amax(-1, keepdim=True)
    i = torch.arange(v, device=DEV, dtype=torch.int32)
    said = torch.where((x == top) & (top > -math.inf), i, torch.full_like(i, v)).amin(-1)
    said = torch.where(said == v, torch.zeros_like(said), said)
    if st["draft"] is None:
        return {"verifier": said, "accepted": torch.zeros(b, dtype=torch.int32, device=DEV), "next": said[:, 0]}
    t = st["draft"].shape[1]
    right = (said[:, :t] == st["draft"]).int()
    accepted = right.cumprod(1).sum(1).int()
    following = torch.where(accepted < r, said.gather(1, accepted.clamp_max(r - 1).long().unsqueeze(1)).squeeze(1), torch.full_like(accepted, -1))
    return {"verifier": said, "accepted": accepted, "next": following}


def _plain_first(st):
    part = torch.arange(st["tokens"].shape[1], device=DEV) < st["n"].unsqueeze(1)
    seen = torch.zeros_like(st["counts"]).scatter_add_(1, st["tokens"].long(), part.int())
    counts = torch.where(seen > 0, torch.full_like(seen, -2 ** 31), torch.zeros_like(seen))
    return {"logits": _adjusted(st, counts).to(st["logits"].dtype), "counts": counts}


def _plain_lora(st):
    c = st["case"]
    x, count = st["x"].float(), st["a"].shape[0]
    t = (x @ st["a"].float().flatten(0, 1).T).view(c["M"], count, c["r"])
    mine = st["ids"].unsqueeze(1) == torch.arange(count, device=DEV)
    t = (t * (mine.float() * st["scale"]).unsqueeze(-1)).flatten(1)
    y = t @ st["b"].float().transpose(1, 2).flatten(0, 1)
    y = y + (x @ _weights(st["codes"], st["scales"]).T if c["shared"] else st["base"].float())
    return y.to(_kind(c["out"]))


_own = {"norm": _own_norm, "rope": _own_rope, "accept": _own_accept, "first": _own_first, "lora": _own_lora}
_plain = {"norm": _plain_norm, "rope": _plain_rope, "accept": _plain_accept, "first": _plain_first, "lora": _plain_lora}


# ---- from the definition, in 64 bits ------------------------------------------------------------------------------------


def _exact_cast(x, mantissa, lowest, most):
    """FP64 [..., n * 32] -> the values of a block format whose elements have `mantissa` bits, exponents from `lowest` on and at most `most`."""
    shape = x.shape
    x = x.reshape(-1, 32)
    top = x.abs().max(1, keepdim=True).values
    share = torch.frexp(top).exponent - 1                       # floor(log2 top)
    share = (share - math.floor(math.log2(most))).clamp_min(-127)
    share = torch.where(top == 0, torch.full_like(share, -127), share)
    a = torch.ldexp(x, -share)
    e = (torch.frexp(a).exponent - 1).clamp_min(lowest) - mantissa
    a = torch.ldexp(torch.round(torch.ldexp(a, -e)), e).clamp(-most, most)
    return torch.ldexp(a, share).reshape(shape)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "rope": _exact_rope, "accept": _exact_rules, "first": _exact_rules, "lora": _exact_lora}[case["op"]](case, st)


def _exact_norm(case, st):
    out = {}
    h = st["x"].double()
    if st["residual"] is not None:
        h += st["residual"].double()
        out["sum"] = h.clone()
    rms = torch.linalg.vector_norm(h, dim=1).square_().div_(case["K"]).add_(st["eps"]).sqrt_()
    y = h.div_(rms.unsqueeze(1)).mul_(st["weight"].double())
    if case["pair"]:
        out["v8"] = _exact_cast(y, 3, -6, 448.0)
    if case["y"]:
        out["y"] = y
    return out


def _exact_rope(case, st):
    half = case["rot"] // 2
    lens, rows = _lengths(case)
    b, m = case["B"], case["M"]
    keep = torch.tensor([[i < n for i in range(m)] for n in rows], device=DEV).view(b, m, 1)
    place = st["positions"].long() if st["positions"] is not None else torch.tensor([[n - r + i for i in range(m)] for n, r in zip(lens, rows)], device=DEV)
    place = place.clamp(0, case["table"] - 1)
    out = {}
    for name in ("q", "k", "v"):
        heads = []
        for h in range(st[name].shape[2]):
            x = st[name][:, :, h].double()
            if name != "v":
                c, s = (st["table"].double()[:, :half][place], st["table"].double()[:, half:][place])
                z = torch.complex(c, s)
                i = torch.arange(half, device=DEV)
                re, im = (i, i + half) if case["style"] == "halves" else (2 * i, 2 * i + 1)
                w = torch.complex(x[..., re], x[..., im]) * z
                x[..., re], x[..., im] = w.real, w.imag
            if name != "q":
                x = _exact_cast(x, 1, 0, 6.0)
            heads.append(torch.where(keep, x, torch.zeros_like(x)))
        out[name] = torch.stack(heads, 2)
    return out


def _exact_rules(case, st):
    b, r, v = st["logits"].shape
    counts = st["counts"].long()
    made, old = counts % 2 ** 31, counts < 0
    if case["op"] == "first":
        old = torch.zeros(b, v, dtype=torch.bool, device=DEV)
        for i, n in enumerate(_histories(case)):
            old[i, st["tokens"][i, :n].long()] = True
        made = torch.zeros_like(counts)
    logits, said = [], []
    for i in range(b):
        rep, pres, freq = st["penalties"][i].double().tolist()
        for j in range(r):
            x, k = st["logits"][i, j].double(), made[i].clone()
            if st["draft"] is not None and j:
                k += torch.bincount(st["draft"][i, :j].long(), minlength=v)
            again = old[i] | (k > 0)
            x[again] = torch.where(x[again] > 0, x[again] / rep, x[again] * rep)
            x[k > 0] -= freq * k[k > 0] + pres
            if st["bias_tokens"] is not None:
                entries = {t: z for t, z in zip(st["bias_tokens"][i].tolist(), st["bias_values"][i].tolist()) if t >= 0}
                x[torch.tensor(list(entries), dtype=torch.int64, device=DEV)] += torch.tensor(list(entries.values()), dtype=torch.float64, device=DEV)
            if st["allowed"] is not None:
                bits = st["allowed"][i, j].view(torch.uint8).unsqueeze(1) >> torch.arange(8, device=DEV, dtype=torch.uint8)
                x[(bits & 1).flatten()[:v] == 0] = -math.inf
            if case["op"] == "first":
                logits.append(x)
            else:
                z = torch.nan_to_num(x, nan=-math.inf, posinf=math.inf, neginf=-math.inf)
                top = z.max()
                said.append(0 if top == -math.inf else int(torch.nonzero(z == top)[0]))
    if case["op"] == "first":
        return {"logits": torch.stack(logits).view(b, r, v), "counts": torch.where(old, -2 ** 31, 0)}
    accepted, following = [], []
    for i in range(b):
        mine = said[i * r:(i + 1) * r]
        draft = st["draft"][i].tolist() if st["draft"] is not None else []
        n = next((j for j, t in enumerate(draft) if mine[j] != t), len(draft))
        accepted.append(n)
        following.append(mine[n] if n < r else -1)
    return {"verifier": torch.tensor(said).view(b, r), "accepted": torch.tensor(accepted), "next": torch.tensor(following)}


def _exact_lora(case, st):
    x, out = st["x"].double(), []
    if case["shared"]:
        low, high = st["codes"].long() & 15, st["codes"].long() >> 4
        nibble = torch.stack([low, high], -1).flatten(1)
        e, f = (nibble >> 1) & 3, (nibble & 1).double()
        w = torch.where(e == 0, f / 2, torch.ldexp(1 + f / 2, e - 1)) * torch.where(nibble >= 8, -1.0, 1.0)
        w = torch.ldexp(w.unflatten(1, (-1, 32)), st["scales"].long().unsqueeze(-1) - 127).flatten(1)
        y = x @ w.T
    else:
        y = st["base"].double()
    ids = st["ids"].tolist()
    for a in sorted(set(ids) - {-1}):
        mine = torch.tensor([i for i, j in enumerate(ids) if j == a], device=DEV)
        y[mine] += float(st["scale"][a]) * ((x[mine] @ st["a"][a].double().T) @ st["b"][a].double().T)
    return y
