"""The 4-bit key/value cache on the GPU (mxq_kv_append, _read, _attention, _resize, _fork, _compact) against the plain 64-bit
implementation of tests/kv_plain.py.

Bytes, tables, lengths and counts must be equal.  For attention the bounds are derived, not fitted: a weight is rounded to 11
bits (2^-12 of itself) and the sum it is divided by is not, the scores carry FP32 errors far below that, so the documented
bound of 2^-10 * sum w|v| / sum w on the FP32 result covers them with a factor of four to spare.  Rounding to BF16 is monotonic, so the
output must lie between the roundings of the exact result minus and plus that bound.
A score is a sum of D products in FP32: at most (D + 2) * 2^-24 of the sum of its terms' magnitudes, which bounds lse too;
its own exp2 / log2 and the sum of the weights add less than 2^-19, and its rounding 2^-23 of its size (2^-21 is asked)."""

import numpy as np
import pytest
import torch

import kv_plain
import paper_2503_13565_b200 as mxq
from paper_2503_13565_b200 import synth

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def bits_of(x):
    return synth.bits_of(x)


class Setup:
    """A pool whose every byte is set, scattered page tables, and the same on the host."""

    def __init__(self, seed, lens, d, h, page, layers=1, spare=2, width=None, fill=None):
        self.rng = np.random.default_rng(seed)
        need = [kv_plain.pages_for(n, page) for n in lens]
        self.lens, self.page = np.array(lens, np.int32), page
        pages = sum(need) + spare
        nbytes = 34 * d * h * (page // 32)
        pool = self.rng.integers(0, 256, (layers, pages, nbytes), dtype=np.uint8) if fill is None else np.full((layers, pages, nbytes), fill, np.uint8)
        width = width or max(1, max(need))
        self.tables = np.full((len(lens), width), -1, np.int32)
        order = self.rng.permutation(pages)
        self.refs = np.zeros(pages, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.tables[b, :n] = order[at:at + n]
            self.refs[order[at:at + n]] = 1
            at += n
        self.host = kv_plain.Cache(pool, h, d, page)
        self.upload()

    def upload(self):
        self.t_pages = torch.from_numpy(self.host.pool.copy()).cuda()
        self.t_refs, self.t_tables, self.t_lens = i32(self.refs), i32(self.tables), i32(self.lens)
        self.cache = mxq.KVCache(self.t_pages, self.t_refs, self.host.h, self.host.d, self.page)

    def random_rows(self, m, scale=1.0):
        """K, V [B][M][H][D] BF16 (host)"""
        shape = (len(self.lens), m, self.host.h, self.host.d)
        make = lambda: torch.from_numpy((self.rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)
        return make(), make()

    def fill_cache(self, layer, big=None):
        """Every token of every sequence from random rows (host side, then uploaded)."""
        for b, n in enumerate(self.lens):
            if n == 0:
                continue
            one = Setup.__new__(Setup)
            one.rng, one.lens, one.host = self.rng, self.lens[b:b + 1], self.host
            k, v = one.random_rows(int(n))
            if big is not None:
                k, v = big(b, k, v)
            kv_plain.append(self.host, layer, bits_of(k), bits_of(v), self.tables[b:b + 1], self.lens[b:b + 1], [int(n)])
        self.upload()

    def check_pool(self):
        got = self.t_pages.cpu().numpy()
        bad = np.argwhere(got != self.host.pool)
        assert bad.size == 0, "%d bytes differ, first at %s" % (len(bad), bad[:3])


# ---- append and read ------------------------------------------------------------------------------------------------------

APPEND = [  # lens, M, rows, d, heads, page, layers
    ([1], 1, None, 128, 1, 32, 1), ([1, 33, 64], 1, None, 64, 2, 64, 2), ([40, 17, 200], 17, None, 128, 3, 32, 1),
    ([300, 299], 299, [299, 1], 64, 8, 256, 1), ([7, 5, 9, 33], 5, [5, 0, 3, 2], 128, 4, 128, 3), ([129], 129, None, 128, 5, 64, 1)]


@pytest.mark.parametrize("lens,m,rows,d,h,page,layers", APPEND)
def test_append_writes_the_cast_and_nothing_else(lens, m, rows, d, h, page, layers):
    s = Setup(1, lens, d, h, page, layers)
    k, v = s.random_rows(m)
    r = [m] * len(lens) if rows is None else rows
    for layer in range(layers):
        mxq.mxq_kv_append(s.cache, layer, k.cuda(), v.cuda(), s.t_tables, s.t_lens, rows=None if rows is None else i32(rows))
        kv_plain.append(s.host, layer, bits_of(k), bits_of(v), s.tables, s.lens, r)
        s.check_pool()
        gk, gv = mxq.mxq_kv_read(s.cache, layer, s.t_tables, s.t_lens, m, rows=None if rows is None else i32(rows))
        for b in range(len(lens)):
            for h_ in range(h):
                for which, got in ((0, gk), (1, gv)):
                    want, _ = s.host.values(which, layer, s.tables[b], lens[b], h_)
                    got_b = got[b, :, h_].float().cpu().numpy().astype(np.float64)
                    assert np.array_equal(got_b[:r[b]], want[lens[b] - r[b]:])
                    assert (got_b[r[b]:] == 0).all()


@pytest.mark.parametrize("d,h,lens,rows", [(128, 32, [4900, 60], [4800, 37]), (64, 33, [4700], None)])
def test_append_of_a_prompt(d, h, lens, rows):
    """Large enough for the prompt kernel; heads that do not fill its groups; rows that are not there; slices of a fused tensor."""
    s = Setup(5, lens, d, h, 64, layers=2)
    m = 4800 if rows else 4700
    fused = torch.from_numpy(s.rng.standard_normal((len(lens), m, (2 * h + 1) * d)).astype(np.float32)).to(torch.bfloat16)
    fused[0, 7, 5] = float("inf")
    fused[0, 8] = 0
    g = fused.cuda()
    k, v = (x[..., d:(h + 1) * d].unflatten(-1, (h, d)) for x in (fused, g)), (x[..., (h + 1) * d:].unflatten(-1, (h, d)) for x in (fused, g))
    (k, gk), (v, gv) = tuple(k), tuple(v)
    r = rows or [m]
    mxq.mxq_kv_append(s.cache, 1, gk, gv, s.t_tables, s.t_lens, rows=None if rows is None else i32(rows))
    kv_plain.append(s.host, 1, bits_of(k.contiguous()), bits_of(v.contiguous()), s.tables, s.lens, r)
    s.check_pool()
    rk, rv = mxq.mxq_kv_read(s.cache, 1, s.t_tables, s.t_lens, m, rows=None if rows is None else i32(rows))
    for b in range(len(lens)):
        for head in (0, 1, h // 2, h - 1):
            for which, got in ((0, rk), (1, rv)):
                want, _ = s.host.values(which, 1, s.tables[b], lens[b], head)
                x = got[b, :, head].float().cpu().numpy().astype(np.float64)
                assert np.array_equal(x[:r[b]], want[lens[b] - r[b]:], equal_nan=True) and (x[r[b]:] == 0).all()


def test_append_of_special_values():
    s = Setup(2, [64], 128, 2, 64)
    k, v = s.random_rows(64)
    for x in (k, v):
        x[0, 0, 0, 5] = float("inf")
        x[0, 1, 0, 40] = float("nan")
        x[0, 2] = 0
        x[0, 3, 1, :32] = -0.0
        x[0, 4] *= 2.0 ** -126
        x[0, 5] = x[0, 5] * 2.0 ** 120
        x[0, 6, 0, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    mxq.mxq_kv_append(s.cache, 0, k.cuda(), v.cuda(), s.t_tables, s.t_lens)
    kv_plain.append(s.host, 0, bits_of(k), bits_of(v), s.tables, s.lens, [64])
    s.check_pool()
    gk, _ = mxq.mxq_kv_read(s.cache, 0, s.t_tables, s.t_lens, 64)
    want, _ = s.host.values(0, 0, s.tables[0], 64, 0)
    assert np.array_equal(gk[0, :, 0].float().cpu().numpy().astype(np.float64), want, equal_nan=True)


def test_append_takes_slices_of_a_fused_projection():
    d, h, hq, m = 128, 2, 6, 7
    s = Setup(3, [20, 7], d, h, 32)
    fused = torch.from_numpy(s.rng.standard_normal((2, m, (hq + 2 * h) * d)).astype(np.float32)).to(torch.bfloat16).cuda()
    k = fused[..., hq * d:(hq + h) * d].unflatten(-1, (h, d))
    v = fused[..., (hq + h) * d:].unflatten(-1, (h, d))
    assert not k.is_contiguous()
    mxq.mxq_kv_append(s.cache, 0, k, v, s.t_tables, s.t_lens)
    kv_plain.append(s.host, 0, bits_of(k.cpu().contiguous()), bits_of(v.cpu().contiguous()), s.tables, s.lens, [m, m])
    s.check_pool()


def test_rows_without_a_page_are_left_out():
    """Entries that are no page of the pool, positions before the start, rows beyond rows[b]."""
    s = Setup(4, [100, 3], 64, 2, 32)
    s.tables[0, 3] = -1
    s.tables[0, 2] = 1 << 20
    s.lens[1] = 2   # two tokens, five rows: the first three would be at negative positions
    s.upload()
    k, v = s.random_rows(5)
    mxq.mxq_kv_append(s.cache, 0, k.cuda(), v.cuda(), s.t_tables, s.t_lens)
    kv_plain.append(s.host, 0, bits_of(k), bits_of(v), s.tables, s.lens, [5, 5])
    s.check_pool()
    gk, _ = mxq.mxq_kv_read(s.cache, 0, s.t_tables, s.t_lens, 5)
    assert (gk[0] == 0).all() and (gk[1, :3] == 0).all() and not (gk[1, 3:] == 0).all()


# ---- attention ------------------------------------------------------------------------------------------------------------


def between_roundings(o, want, bound):
    """BF16 outputs o against exact - bound .. exact + bound, both ends rounded to BF16 (NaN where the exact result is)."""
    low, high = (torch.from_numpy(x).to(torch.bfloat16).double().numpy() for x in (want - bound, want + bound))
    fine = ~np.isnan(want)
    bad = fine & ~((low <= o) & (o <= high))
    assert not bad.any(), "%d outside, first %s: %r not in %r .. %r" % (bad.sum(), np.argwhere(bad)[0], o[bad][0], low[bad][0], high[bad][0])
    return True


def check_attention(s, layer, q, rows=None, trees=None, scale=None, q_gpu=None, **kw):
    b, m, hq, d = q.shape
    r = [m] * b if rows is None else rows
    sc = d ** -0.5 if scale is None else scale
    q_gpu = q.cuda() if q_gpu is None else q_gpu
    t = None if trees is None else torch.from_numpy(np.asarray(trees, np.uint64).view(np.int64)).cuda()
    ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(b, m, hq, s.host.h, d))
    args = dict(rows=None if rows is None else i32(rows), tree=t, scale=scale, workspace=ws, with_lse=True, **kw)
    out, lse = mxq.mxq_kv_attention(q_gpu, s.cache, layer, s.t_tables, s.t_lens, **args)
    again, lse2 = mxq.mxq_kv_attention(q_gpu, s.cache, layer, s.t_tables, s.t_lens, **args)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))
    assert int(ws[:4096].sum()) == 0
    want, wl, spread, smax = kv_plain.attention(s.host, layer, q.double().numpy(), s.tables, s.lens, r, sc, trees)
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(o), nan), "NaN in the wrong places: %d, expected %d" % (np.isnan(o).sum(), nan.sum())
    assert between_roundings(o, want, 2.0 ** -10 * spread + 2.0 ** -133)
    empty = np.isneginf(wl)
    assert np.array_equal(np.isneginf(l), empty)
    assert (o[empty] == 0).all()
    fine = ~empty & ~np.isnan(wl)
    assert np.isnan(l[np.isnan(wl)]).all()
    tl = (d + 2) * 2.0 ** -24 * smax + 2.0 ** -21 * np.abs(np.where(fine, wl, 0)) + 2.0 ** -19
    assert (np.abs(l[fine] - wl[fine]) <= tl[fine]).all(), "lse error/tolerance %.3g" % (np.abs(l[fine] - wl[fine]) / tl[fine]).max()
    return out, lse


def queries(s, m, hq, scale=1.0):
    shape = (len(s.lens), m, hq, s.host.d)
    return torch.from_numpy((s.rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)


LENGTHS = [[1], [2, 31], [32], [33, 64, 63], [65, 1, 127], [128], [129, 7], [255, 257], [500], [1000, 3, 400]]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 256])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda x: "x".join(map(str, x)))
def test_attention_single_token(lens, page, d):
    s = Setup(10, lens, d, 2, page)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, 1, 2, 2.0))


HEADS = [(1, 1), (4, 4), (8, 2), (6, 3), (9, 1), (16, 1), (17, 1), (40, 1), (5, 5)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 2, 5, 16])
@pytest.mark.parametrize("hq,h", HEADS)
def test_attention_heads_and_rows(hq, h, m, d):
    s = Setup(11, [77, 200, m], d, h, 64, layers=2)
    s.fill_cache(1)
    check_attention(s, 1, queries(s, m, hq, 2.0))


@pytest.mark.parametrize("d,m", [(128, 64), (64, 64), (128, 100), (64, 33)])
def test_attention_many_rows(d, m):
    s = Setup(12, [300, m, m + 40], d, 2, 128)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, m, 4, 1.5))


@pytest.mark.parametrize("d", [64, 128])
def test_attention_ragged_rows_and_empty_sequences(d):
    s = Setup(13, [90, 40, 0, 6, 64], d, 3, 32)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, 6, 6), rows=[6, 0, 4, 6, 1])


@pytest.mark.parametrize("rows", [[0], [0, 2], [3, 0, 0, 1]])
def test_attention_long_sequences_without_rows(rows):
    lens = [9000, 5000, 7777, 100][:len(rows)]
    s = Setup(29, lens, 64, 2, 64)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, max(max(rows), 1), 8), rows=rows)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 5, 16, 48, 64])
def test_attention_token_trees(m, d):
    """Random ancestor masks, rows that see only what came before, and rows that see nothing at all."""
    s = Setup(14, [m, m + 100, m + 31, 200], d, 2, 64)
    s.fill_cache(0)
    trees = np.zeros((4, m), np.uint64)
    for b in range(4):
        for i in range(m):
            parent = int(s.rng.integers(0, i)) if i else -1
            trees[b, i] = (trees[b, parent] if parent >= 0 else np.uint64(0)) | np.uint64(1 << i)
    trees[0, m - 1] = 0      # nothing before the rows and none of the rows: an empty row
    trees[1, 0] = 0          # only what came before
    trees[2] = s.rng.integers(0, 1 << 63, m, dtype=np.uint64)   # anything goes (bits beyond the rows are ignored)
    check_attention(s, 0, queries(s, m, 6, 2.0), rows=None if m == 1 else [m, m, m, m // 2], trees=trees)


def test_attention_query_slices_and_given_outputs():
    d, h, hq, m = 128, 2, 4, 3
    s = Setup(15, [50, 130], d, h, 64)
    s.fill_cache(0)
    fused = torch.randn(2, m, (hq + 2 * h) * d, device="cuda").to(torch.bfloat16)
    q = fused[..., :hq * d].unflatten(-1, (hq, d))
    out = torch.full((2, m, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    got, _ = check_attention(s, 0, q.cpu().contiguous(), q_gpu=q, out=out)
    assert got.data_ptr() == out.data_ptr()


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 5.0])
def test_attention_scales(scale):
    s = Setup(16, [150, 20], 64, 2, 32)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, 2, 4, 3.0), scale=scale)


@pytest.mark.parametrize("power", [-60, -20, 20, 60])
def test_attention_sizes_of_queries(power):
    """Large and small queries against keys of the opposite size: the scores are ordinary, the factors are not."""
    s = Setup(17, [140], 128, 2, 64)
    s.fill_cache(0, big=lambda b, k, v: (k * 2.0 ** -power, v))
    q = queries(s, 2, 4) * 2.0 ** power
    q[0, 1, 0, :64] *= 2.0 ** -30      # and a row whose elements span a wide range
    check_attention(s, 0, q)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shift", [10, 25, 60, 100])
def test_attention_values_of_very_different_size(shift, d):
    """Tokens whose values are 2^shift larger than the others' but carry next to no weight, and the other way round: every
    row's result must be right to its own size."""
    s = Setup(18, [200, 333], d, 2, 64)
    target = torch.zeros(d)
    target[0] = 40.0

    def big(b, k, v):
        k[..., 0] = 0
        k[0, 7:11, :, 0] = 8.0            # what the first query looks at: small values
        k[0, 60:64, :, 0] = -8.0          # what the second looks at: large ones
        v[0, 60:64] *= 2.0 ** (shift / 2)
        v[0, 7:11] *= 2.0 ** (-shift / 2)
        v[0, 20] = 0
        return k, v

    s.fill_cache(0, big=big)
    q = torch.zeros(2, 2, 4, d)
    q[:, :, 0::2], q[:, :, 1::2] = target, -target
    check_attention(s, 0, q.to(torch.bfloat16))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.5, 1.0, 7 / 6, 4 / 3, 1.5, 2.0, 4.0])
def test_attention_small_weights_where_the_large_ones_meet_zeros(scale, d):
    """One token takes nearly all the weight, but holds zeros in half of the elements: there the result is the others', whose
    weights are e^-6 .. e^-48 of the largest, and must be right to its own size."""
    s = Setup(30, [96, 700], d, 2, 32)

    def big(b, k, v):
        k[:] = 0
        k[..., 0] = -12.0
        k[0, 3] = 0
        v[..., 31::32] = 6.0             # every block has the same scale
        v[0, 3] = 4.0
        v[0, 3].view(2, d // 32, 32)[:, :, :16] = 0
        return k, v

    s.fill_cache(0, big=big)
    q = torch.zeros(2, 1, 4, d)
    q[..., 0] = 1.0
    check_attention(s, 0, q.to(torch.bfloat16), scale=scale)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [0xFF, 0xFE, 0xF0])
def test_what_a_row_does_not_see_does_not_touch_it(bad, d):
    """The pool outside the sequences, the tokens behind a sequence's end on its last page, and the drafted tokens a row
    must not see hold NaN scales, or the largest ones."""
    m = 5
    s = Setup(19, [m + 40, m + 3, 96], d, 2, 64, fill=bad)
    s.fill_cache(0)
    for b in range(3):                       # drafted tokens 2 and 4: NaN, or values of 2^126 and 2^112
        n = int(s.lens[b])
        for j in (2, 4):
            pos = n - m + j
            for h in range(2):
                for which in (0, 1):
                    s.host.put(which, 0, s.tables[b][pos // 64], pos % 64, h, np.full(d // 2, 0x11, np.uint8), np.full(d // 32, bad, np.uint8))
    s.upload()
    trees = np.array([[0b00001, 0b00011, 0b00001, 0b01011, 0b00000]] * 3, np.uint64)
    q = queries(s, m, 4)
    check_attention(s, 0, q, trees=trees)
    # causally, rows 0 and 1 are clean and the rows from 2 on see the bad token: NaN scales give NaN there and only there
    if bad == 0xFF:
        check_attention(s, 0, q)


def test_attention_rows_of_nan_and_infinity():
    s = Setup(20, [100], 128, 2, 32)
    s.fill_cache(0)
    q = queries(s, 3, 4)
    q[0, 1, 2, 17] = float("nan")
    ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(1, 3, 4, 2, 128))
    out = mxq.mxq_kv_attention(q.cuda(), s.cache, 0, s.t_tables, s.t_lens, workspace=ws).cpu()
    assert torch.isnan(out[0, 1, 2].float()).all()
    out[0, 1, 2] = 0
    assert torch.isfinite(out.float()).all()


def test_attention_tokens_without_a_page():
    s = Setup(21, [200, 64], 128, 2, 32)
    s.fill_cache(0)
    s.tables[0, 2] = -1
    s.tables[0, 4] = 1 << 24
    s.tables[1, :] = -1        # nothing left of the second sequence: empty rows
    s.upload()
    check_attention(s, 0, queries(s, 2, 4))


def test_attention_long_and_many():
    """Segments that are cut over many CTAs, and more sequences than CTAs."""
    s = Setup(22, [9000], 128, 1, 256)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, 1, 4, 2.0))
    s = Setup(23, [int(x) for x in np.random.default_rng(5).integers(1, 70, 700)], 64, 1, 32)
    s.fill_cache(0)
    check_attention(s, 0, queries(s, 1, 2, 2.0))


def test_attention_calls_of_all_shapes_share_a_workspace():
    """Small and large batches, both head dimensions, few and many rows, cut and whole segments, in turn on one workspace."""
    shapes = [(64, 1, 2, 2, [40]), (128, 5, 8, 2, [700, 90]), (64, 1, 4, 1, [2000] * 3), (128, 1, 1, 1, [5000]), (64, 16, 8, 1, [300] * 40),
              (128, 1, 8, 8, [64] * 100)]
    cases = []
    for i, (d, m, hq, h, lens) in enumerate(shapes):
        s = Setup(80 + i, lens, d, h, 64)
        s.fill_cache(0)
        cases.append((s, queries(s, m, hq).cuda()))
    ws = mxq.new_workspace(max(mxq.mxq_kv_attention_workspace_bytes(len(lens), m, hq, h, d) for d, m, hq, h, lens in shapes))
    run = lambda s, q, w: mxq.mxq_kv_attention(q, s.cache, 0, s.t_tables, s.t_lens, workspace=w)
    alone = [run(s, q, None) for s, q in cases]
    for order in (range(6), reversed(range(6)), (3, 0, 5, 1, 4, 2, 3, 3)):
        for i in order:
            assert torch.equal(run(*cases[i], ws), alone[i]), shapes[i]
    assert mxq.mxq_linear_device_status() == 0


def test_attention_lengths_beyond_the_table_count_as_its_end():
    s = Setup(24, [64, 64], 64, 1, 32)
    s.fill_cache(0)
    s.t_lens = i32([1000, -5])
    s.lens = np.array([64, 0], np.int32)
    check_attention(s, 0, queries(s, 1, 2))


@pytest.mark.parametrize("d", [64, 128])
def test_offsets_beyond_32_bits(d):
    """The pages in use lie behind the first 5 GB of the pool, in its last layer."""
    h, page, layers = 8, 64, 2
    nbytes = 34 * d * h * 2
    pages = (5 << 30) // nbytes // layers * 2
    s = Setup(25, [150, 70], d, h, page, layers=1, spare=0)
    s.fill_cache(0)
    small = s.t_pages
    used = small.shape[1]
    pool = torch.empty((layers, pages, nbytes), dtype=torch.uint8, device="cuda")
    pool[layers - 1, pages - used:] = small[0]
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    s.cache = mxq.KVCache(pool, refs, h, d, page)
    q = queries(s, 2, 8)
    s.t_tables = torch.where(s.t_tables >= 0, s.t_tables + (pages - used), s.t_tables)
    host = s.tables
    want, _, spread, _ = kv_plain.attention(s.host, 0, q.double().numpy(), host, s.lens, [2, 2], d ** -0.5)
    out = mxq.mxq_kv_attention(q.cuda(), s.cache, layers - 1, s.t_tables, s.t_lens).double().cpu().numpy()
    assert between_roundings(out, want, 2.0 ** -10 * spread)
    k, v = s.random_rows(3)
    mxq.mxq_kv_append(s.cache, layers - 1, k.cuda(), v.cuda(), s.t_tables, s.t_lens)
    kv_plain.append(s.host, 0, bits_of(k), bits_of(v), host, s.lens, [3, 3])
    assert np.array_equal(pool[layers - 1, pages - used:].cpu().numpy(), s.host.pool[0])


def test_streams_and_graph_replay():
    """append + attention on a side stream, then captured and replayed with other inputs in the same buffers."""
    d, h, hq = 128, 2, 8
    s = Setup(26, [120, 77], d, h, 32)
    s.fill_cache(0)
    side = torch.cuda.Stream()
    q, out = queries(s, 1, hq).cuda(), torch.empty(2, 1, hq, d, dtype=torch.bfloat16, device="cuda")
    k, v = (x.cuda() for x in s.random_rows(1))
    ws = mxq.new_workspace(mxq.mxq_kv_attention_workspace_bytes(2, 1, hq, h, d))
    torch.cuda.synchronize()

    def step():
        mxq.mxq_kv_append(s.cache, 0, k, v, s.t_tables, s.t_lens)
        mxq.mxq_kv_attention(q, s.cache, 0, s.t_tables, s.t_lens, out=out, workspace=ws)

    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        nk, nv = s.random_rows(1)
        nq = queries(s, 1, hq)
        k.copy_(nk), v.copy_(nv), q.copy_(nq)
        graph.replay()
        torch.cuda.synchronize()
        kv_plain.append(s.host, 0, bits_of(nk), bits_of(nv), s.tables, s.lens, [1, 1])
        s.check_pool()
        want, _, spread, _ = kv_plain.attention(s.host, 0, nq.double().numpy(), s.tables, s.lens, [1, 1], d ** -0.5)
        assert between_roundings(out.double().cpu().numpy(), want, 2.0 ** -10 * spread)


# ---- pages ----------------------------------------------------------------------------------------------------------------


def check_book(s):
    assert np.array_equal(s.t_lens.cpu().numpy(), s.lens)
    assert np.array_equal(s.t_tables.cpu().numpy(), s.tables)
    assert np.array_equal(s.t_refs.cpu().numpy(), s.refs)


@pytest.mark.parametrize("seed,b,page,width,spare", [(1, 1, 32, 4, 9), (2, 5, 64, 7, 3), (3, 40, 32, 9, 0), (4, 300, 32, 5, 200), (5, 1500, 32, 3, 900),
                                                     (6, 64, 32, 40, 40000)])
def test_resize_random_walk(seed, b, page, width, spare):
    """Growth, rollback, release and calls that run out of pages, against one page at a time."""
    rng = np.random.default_rng(seed)
    s = Setup(30 + seed, [int(x) for x in rng.integers(0, width * page // 2, b)], 64, 1, page, spare=spare, width=width, fill=0)
    for step in range(6):
        new = rng.integers(0, width * page + 1, b) if step % 2 else np.minimum(s.lens + rng.integers(0, 40, b), width * page)
        new[rng.random(b) < 0.2] = 0
        if step == 3:
            new[rng.integers(0, b)] = width * page + 1      # not a length the table can hold
            new[rng.integers(0, b)] = -3
        mxq.mxq_kv_resize(s.cache, s.t_tables, s.t_lens, i32(new))
        kv_plain.resize(s.tables, s.lens, s.refs, new, page)
        check_book(s)
    mxq.mxq_kv_resize(s.cache, s.t_tables, s.t_lens, i32(np.zeros(b)))
    assert int(s.t_refs.abs().sum()) == 0 and bool((s.t_tables == -1).all())


def test_resize_gives_back_what_does_not_fit():
    s = Setup(40, [32, 32, 32], 64, 1, 32, spare=4, width=8, fill=0)
    mxq.mxq_kv_resize(s.cache, s.t_tables, s.t_lens, i32([64, 192, 64]))   # 1 + 5 + 1 pages wanted, 4 free
    kv_plain.resize(s.tables, s.lens, s.refs, [64, 192, 64], 32)
    assert s.lens.tolist() == [64, 32, 32]
    check_book(s)
    mxq.mxq_kv_resize(s.cache, s.t_tables, s.t_lens, i32([10, 31, 0]))
    kv_plain.resize(s.tables, s.lens, s.refs, [10, 31, 0], 32)
    check_book(s)


FORKS = [([40], [0], [1], 2, 64, 1, 3), ([100, 33, 64, 0], [0, 0, 1, 2, 3], [4, 5, 6, 7, 8], 9, 32, 2, 10), ([129, 60], [0, 1, 0, 1], [2, 3, 4, 5], 6, 128, 3, 2),
         ([200], [0, 0, 0], [1, 2, 3], 4, 64, 2, 3)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,src,dst,b,page,layers,spare", FORKS)
def test_fork(lens, src, dst, b, page, layers, spare, d):
    s = Setup(50, lens + [0] * (b - len(lens)), d, 3, page, layers=layers, spare=spare)
    mxq.mxq_kv_fork(s.cache, s.t_tables, s.t_lens, i32(src), i32(dst))
    kv_plain.fork(s.host, s.tables, s.lens, s.refs, src, dst, page)
    check_book(s)
    s.check_pool()
    # shared pages live until their last holder lets go
    for new in (np.where(np.arange(b) < len(lens), 0, s.lens), np.zeros(b)):
        mxq.mxq_kv_resize(s.cache, s.t_tables, s.t_lens, i32(new))
        kv_plain.resize(s.tables, s.lens, s.refs, new.astype(int), page)
        check_book(s)
    assert s.refs.sum() == 0


def test_fork_leaves_out_pairs_that_make_no_sense():
    s = Setup(51, [40, 50, 0, 0], 64, 2, 32, spare=5, width=4)
    src, dst = [0, 7, 1, 0, 1], [2, 3, 0, -1, 1]     # good; no such source; occupied; no such slot; itself
    mxq.mxq_kv_fork(s.cache, s.t_tables, s.t_lens, i32(src), i32(dst))
    kv_plain.fork(s.host, s.tables, s.lens, s.refs, src, dst, 32)
    assert s.lens.tolist() == [40, 50, 40, 0]
    check_book(s)
    s.check_pool()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,page,h,layers", [(1, 32, 1, 1), (5, 32, 2, 2), (16, 64, 8, 3), (64, 32, 2, 1), (64, 256, 3, 2)])
def test_compact(m, page, h, layers, d):
    """Paths whose sources lie among their destinations, paths kept as they are, empty ones, rows across pages."""
    s = Setup(60, [m, m + 30, m + 31, m + 200, 70 + m, m + 5], d, h, page, layers=layers)
    rows = np.array([m, m, max(1, m // 2), m, m, m], np.int32)
    keep, kept = np.zeros((6, m), np.int32), np.zeros(6, np.int32)
    for b in range(6):
        n = int(s.rng.integers(0, rows[b] + 1)) if b < 4 else (0 if b == 4 else rows[b])
        keep[b, :n] = np.sort(s.rng.choice(rows[b], n, replace=False))
        kept[b] = n
    got = mxq.mxq_kv_compact(s.cache, s.t_tables, s.t_lens, i32(rows), i32(keep), i32(kept))
    want = kv_plain.compact(s.host, s.tables, s.lens, rows, keep, kept)
    assert np.array_equal(got.cpu().numpy(), want)
    s.check_pool()
    mxq.mxq_kv_resize(s.cache, s.t_tables, s.t_lens, got)
    kv_plain.resize(s.tables, s.lens, s.refs, want, page)
    check_book(s)


# ---- refusals of the binding ----------------------------------------------------------------------------------------------


def test_wrong_tensors_are_refused():
    s = Setup(70, [40, 50], 64, 2, 32)
    k, v = (x.cuda() for x in s.random_rows(2))
    q = queries(s, 2, 4).cuda()
    with pytest.raises(ValueError):
        mxq.mxq_kv_append(s.cache, 0, k[:, :1], v, s.t_tables, s.t_lens)
    with pytest.raises(TypeError):
        mxq.mxq_kv_append(s.cache, 0, k.float(), v, s.t_tables, s.t_lens)
    with pytest.raises(TypeError):
        mxq.mxq_kv_append(s.cache, 0, k.transpose(1, 2).contiguous().transpose(1, 2), v, s.t_tables, s.t_lens)
    with pytest.raises(ValueError):
        mxq.mxq_kv_append(s.cache, 0, k, v, s.t_tables, s.t_lens[:1])
    with pytest.raises(TypeError):
        mxq.mxq_kv_append(s.cache, 0, k, v, s.t_tables.long(), s.t_lens)
    with pytest.raises(mxq.MxqError):
        mxq.mxq_kv_append(s.cache, 1, k, v, s.t_tables, s.t_lens)
    with pytest.raises(mxq.MxqError):
        mxq.mxq_kv_attention(q[:, :, :3], s.cache, 0, s.t_tables, s.t_lens)     # 3 query heads over 2
    with pytest.raises(ValueError):
        mxq.mxq_kv_attention(q, s.cache, 0, s.t_tables, s.t_lens, tree=torch.zeros(2, 3, dtype=torch.int64, device="cuda"))
    with pytest.raises(mxq.MxqError):
        mxq.mxq_kv_attention(q, s.cache, 0, s.t_tables, s.t_lens, workspace=mxq.new_workspace(16))
    with pytest.raises(mxq.MxqError):
        mxq.mxq_kv_compact(s.cache, s.t_tables, s.t_lens, None, torch.zeros(2, 65, dtype=torch.int32, device="cuda"), i32([0, 0]))
    with pytest.raises(mxq.MxqError):
        mxq.mxq_kv_compact(s.cache, s.t_tables, s.t_lens, None, i32(np.zeros((2, 2))), i32([0, 0]), lens_out=s.t_lens)
    with pytest.raises(ValueError):
        mxq.KVCache(s.t_pages[:, :, :-16], s.t_refs, 2, 64, 32)
    with pytest.raises(ValueError):
        mxq.KVCache.new(1, 4, 2, 80)
    s.check_pool()
