"""Plain implementations, for tests, of what a decoder step needs between its linear layers and its cache: written from the definitions
in include/mxq.h, in 64 bits where the result has a tolerance, in FP32 step by step where it is defined to the bit."""
import numpy as np
import torch

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def rmsnorm(x, residual, weight, eps):
    """(h, y) in 64 bits."""
    h = x.double() + (0 if residual is None else residual.double())
    return h, h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()


def mxfp8_values(codes, scales):
    """64-bit values of an MXFP8 pair, from the formats' fields."""
    c = codes.cpu().numpy().astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7)) * np.where(c & 128, -1.0, 1.0)
    s = scales.cpu().numpy().astype(np.int64)
    return v * np.repeat(np.where(s == 255, np.nan, np.ldexp(1.0, s - 127)), 32, axis=-1)


def cast_fp4(x):
    """The values [..., D] (float64) that FP32 x has after the direct cast to MXFP4."""
    b = np.asarray(x, np.float64).reshape(-1, 32)
    top = np.abs(b).max(1)
    fine = np.isfinite(b).all(1)
    with np.errstate(all="ignore"):
        e = np.where(top > 0, np.frexp(np.where(fine, top, 1))[1] - 1, -1000)
        scale = np.ldexp(1.0, np.maximum(e - 2, -127))[:, None]
        a = np.minimum(np.abs(b) / scale, 6)
    code = np.abs(a[..., None] - E2M1).argmin(-1)
    tie = np.abs(a - E2M1[code]) == np.abs(E2M1[np.minimum(code + 1, 7)] - a)
    code = code + (tie & (code % 2 == 1) & (code < 7))           # (argmin takes the lower of two; a tie goes to the even code)
    v = np.copysign(E2M1[code], b) * scale
    return np.where(fine[:, None], v, np.nan).reshape(np.shape(x))


def rotate(x, cos, sin, rotary, style):
    """FP32 step by step: x [..., D] float32, cos / sin [..., rotary / 2] float32."""
    x, half = x.copy(), rotary // 2
    a, b = (slice(0, half), slice(half, rotary)) if style == "halves" else (slice(0, rotary, 2), slice(1, rotary, 2))
    one, two = x[..., a].copy(), x[..., b].copy()
    x[..., a] = (one * cos).astype(np.float32) - (two * sin).astype(np.float32)
    x[..., b] = (two * cos).astype(np.float32) + (one * sin).astype(np.float32)
    return x


def bf16(x):
    """FP32 array -> the nearest BF16 values, as FP32."""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().float().numpy()


def adjusted(logits, draft, counts, penalties, bias_tokens, bias_values, allowed):
    """FP32 [B, R, V], one rounding per operation; counts as int64 with bit 31, allowed bool [B, R, V]; None: no such rule."""
    f = np.float32
    out = logits.astype(f).copy()
    b_, r_, v_ = out.shape
    for b in range(b_):
        for r in range(r_):
            x = out[b, r]
            if penalties is not None:
                rep, pres, freq = (f(z) for z in penalties[b])
                n = np.zeros(v_, np.int64) if counts is None else counts[b] & 0x7FFFFFFF
                old = np.zeros(v_, bool) if counts is None else (counts[b] >> 31) & 1 == 1
                n = n.copy()
                for t in (draft[b][:r] if draft is not None else []):
                    if 0 <= t < v_:
                        n[t] += 1
                with np.errstate(all="ignore"):
                    x = np.where(old | (n > 0), np.where(x > 0, x / rep, x * rep), x).astype(f)
                    x = np.where(n > 0, (x - (freq * n.astype(f)).astype(f)).astype(f) - pres, x).astype(f)
            if bias_tokens is not None:
                for t, z in {int(t): z for t, z in zip(bias_tokens[b], bias_values[b]) if 0 <= t < v_}.items():
                    with np.errstate(invalid="ignore"):
                        x[t] = f(x[t]) + f(z)
            if allowed is not None:
                x = np.where(allowed[b, r], x, f(-np.inf))
            out[b, r] = x
    return out


def argmax(row):
    best, at = -np.inf, 0
    for i in np.flatnonzero(row > -np.inf):
        if row[i] > best:
            best, at = row[i], i
    return int(at)


def accept(rows, draft):
    """(verifier [R], accepted, next) of one sequence's adjusted rows."""
    said = [argmax(r) for r in rows]
    draft = [] if draft is None else list(draft)
    n = next((i for i, t in enumerate(draft) if said[i] != t), len(draft))
    return said, n, said[n] if n < len(said) else -1


def lora(x, a, b, scale, ids, base):
    """(y, magnitude) in 64 bits: the magnitude is |s| sum |B| sum |A x|."""
    m, n = x.shape[0], b.shape[1]
    y = torch.zeros(m, n, dtype=torch.float64) if base is None else base.double().cpu().clone()
    mag = torch.zeros(m, n, dtype=torch.float64)
    x, a, b = x.double().cpu(), a.double().cpu(), b.double().cpu()
    for i, o in enumerate(ids.tolist()):
        if 0 <= o < a.shape[0]:
            s = 1.0 if scale is None else float(scale[o])
            y[i] += s * (b[o] @ (a[o] @ x[i]))
            mag[i] = abs(s) * (b[o].abs() @ (a[o].abs() @ x[i].abs()))
    return y, mag
