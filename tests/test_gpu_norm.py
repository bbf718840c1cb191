"""mxq_rmsnorm and mxq_dequantize_mxfp8 against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2503_13565_b200 as mxq
import step_plain as plain

pytestmark = pytest.mark.gpu

# The kernel's y before rounding: the sum of squares is a chain of at most 32 additions per lane, 5 in a warp and 5 over the warps, each
# 2^-24 of the sum, halved by the root; division, root, two products and h itself some 2^-24 each: below 2^-18 in all.
Y_REL = 2.0 ** -18
BF16, F32 = torch.bfloat16, torch.float32


def data(m, k, x, res, w, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    channel = torch.exp(1.5 * r(k))
    return (r(m, k) * channel).to(x), None if res is None else (3 * r(m, k) * channel).to(res), (1 + 0.3 * r(k)).to(w)


def near(got, want, rel, floor=0.0):
    got, want = got.double(), want.double()
    assert bool(((got - want).abs() <= rel * want.abs() + floor).all()), float(((got - want).abs() / want.abs().clamp_min(1e-300)).max())


def check_pair(codes, scales, y):
    v = torch.from_numpy(plain.mxfp8_values(codes, scales)).cuda()
    b, u = y.view(-1, 32), v.view(-1, 32)
    s = 2.0 ** (scales.view(-1, 1).double() - 127)
    top = b.abs().amax(1, keepdim=True)
    low = s == 2.0 ** -127
    assert bool(((s * 256 <= top * (1 + Y_REL)) | low).all()) and bool((top < s * 512 * (1 + Y_REL)).all())
    want = torch.minimum(torch.maximum(b, -448 * s), 448 * s)
    assert bool(((u - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * s + 2 * Y_REL * b.abs()).all())


@pytest.mark.parametrize("m,k,x,res,w", [
    (1, 32, BF16, BF16, BF16), (1, 4096, BF16, BF16, BF16), (3, 96, F32, None, F32), (16, 5120, F32, BF16, F32), (7, 8192, BF16, F32, BF16),
    (5, 8224, F32, F32, BF16), (2, 16416, BF16, None, F32), (2, 32768, F32, F32, F32), (1000, 768, BF16, BF16, F32), (3, 11008, BF16, BF16, BF16)])
def test_against_the_definition(m, k, x, res, w):
    xs, r, wt = data(m, k, x, res, w)
    out = None if r is None else torch.empty_like(r)
    y, codes, scales = mxq.mxq_rmsnorm(xs, wt, 1e-5, residual=r, residual_out=out, mxfp8=True)
    h, want = plain.rmsnorm(xs, r, wt, 1e-5)
    if r is not None:
        near(out, h, 2.0 ** -24 if res == F32 else 2.0 ** -8, 1e-38)
    near(y, want, 2.0 ** -8 + 2 * Y_REL, 1e-38)
    check_pair(codes, scales, want)
    # each output alone, and without the sum, is the same
    assert torch.equal(mxq.mxq_rmsnorm(xs, wt, 1e-5, residual=r), y)
    c2, s2 = mxq.mxq_rmsnorm(xs, wt, 1e-5, residual=r, bf16=False, mxfp8=True)
    assert torch.equal(c2, codes) and torch.equal(s2, scales)
    # the pair's inverse
    v = plain.mxfp8_values(codes, scales)
    assert np.array_equal(mxq.mxq_dequantize_mxfp8(codes, scales, out_dtype=F32).cpu().numpy().astype(np.float64), v)
    assert torch.equal(mxq.mxq_dequantize_mxfp8(codes, scales).cpu(), torch.from_numpy(v).bfloat16())


def test_rows_that_are_zero_tiny_huge_or_not_finite():
    k = 256
    x = torch.randn(8, k, device="cuda")
    x[0] = 0
    x[1] *= 1e-30
    x[2] *= 1e15
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    x[5] = 0
    x[5, 33] = 1e-42                     # subnormal: the row's mean square vanishes beside eps
    w = torch.ones(k, device="cuda")
    y, codes, scales = mxq.mxq_rmsnorm(x, w, 1e-6, mxfp8=True)
    _, want = plain.rmsnorm(x, None, w, 1e-6)
    for row in (0, 1, 2, 5, 6, 7):
        near(y[row], want[row], 2.0 ** -8 + 2 * Y_REL, 2.0 ** -134)
    assert bool((scales[0] == 0).all()) and bool(((codes[0] & 127) == 0).all())
    assert bool(y[3].isnan().all()) and bool((scales[3] == 255).all()) and bool((codes[3] == 0).all())
    inf = y[4].float()                   # 1 / inf = 0: the others are zero, the infinite one is no number
    assert bool(inf[7].isnan()) and bool((inf[torch.arange(k, device="cuda") != 7] == 0).all())
    assert int(scales[4, 0]) == 255 and bool((scales[4, 1:] == 0).all())
    check_pair(codes[[1, 2, 6, 7]], scales[[1, 2, 6, 7]], want[[1, 2, 6, 7]])


def test_every_e4m3_code_and_rounding():
    """Blocks whose largest element is 256 (scale 1): all values near every border of the format; ties go to the even code."""
    grid = e4m3_values()
    mid = (grid[1:] + grid[:-1]) / 2
    v = np.concatenate([grid, mid, np.nextafter(mid.astype(np.float32), 0), np.nextafter(mid.astype(np.float32), 1e9)]).astype(np.float32)
    v = v[v < 300]
    v = np.concatenate([v, -v])
    v = np.concatenate([v, np.zeros((-len(v)) % 31, np.float32)]).reshape(-1, 31)
    v = np.concatenate([np.full((len(v), 1), 256, np.float32), v], 1)
    x = torch.from_numpy(v).cuda()
    # weight 1 and rows scaled so that the norm changes nothing: eps makes the mean square exactly 2^44
    sq = (x.double() ** 2).mean(1)
    k = x.shape[1]
    codes, scales = [], []
    for i in range(len(v)):
        # one row at a time: y = h * (1 / sqrt(mean + eps)) with mean + eps rounded to 2^44, so that y = h * 2^-22 exactly
        c, s = mxq.mxq_rmsnorm(x[i:i + 1], torch.ones(k, device="cuda"), float(2.0 ** 44), bf16=False, mxfp8=True)
        codes.append(c), scales.append(s)
    assert float(sq.max()) < 2.0 ** 20          # (below half a step of 2^44 in FP32: it leaves eps as it is)
    codes, scales = torch.cat(codes), torch.cat(scales)
    assert bool((scales == 127 - 22).all())
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).float()
    assert torch.equal(mxq.mxq_dequantize_mxfp8(codes, scales, out_dtype=F32), want * 2.0 ** -22)


def e4m3_values():
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7))


def test_strided_rows_in_place_sum_and_aliases():
    m, k = 37, 768
    wide = torch.randn(m, 3 * k, device="cuda").bfloat16()
    r = torch.randn(m, k, device="cuda").bfloat16()
    w = torch.rand(k, device="cuda").bfloat16()
    x = wide[:, k:2 * k]
    want_h = torch.empty_like(r)
    want = mxq.mxq_rmsnorm(x.contiguous(), w, residual=r, residual_out=want_h)
    before = wide.clone()
    stream = r.clone()
    assert torch.equal(mxq.mxq_rmsnorm(x, w, residual=stream, residual_out=stream), want) and torch.equal(stream, want_h) and torch.equal(wide, before)
    a = x.contiguous()
    assert torch.equal(mxq.mxq_rmsnorm(a, w, residual=r, out=a), want) and torch.equal(a, want)       # y over x
    with pytest.raises(TypeError):
        mxq.mxq_rmsnorm(wide.t()[:m], w)
    with pytest.raises(mxq.MxqError):
        mxq.mxq_rmsnorm(wide[:, 4:4 + k], w)                                                          # rows not 16-byte aligned
    with pytest.raises(TypeError):
        mxq.mxq_rmsnorm(x, w, residual=r, residual_out=torch.empty(m, k, device="cuda"))
