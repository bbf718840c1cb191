// mxq_kv_append / mxq_kv_read: the direct cast of new K and V rows into the pages of a 4-bit cache, and its inverse.
//
// Both are streams: 2 bytes of BF16 against 0.53 bytes of codes and scales per element, in opposite directions; a decode
// step's few rows are a launch's latency.  In the append of a few rows and in the read four
// lanes share a row: lane c takes elements 8c..8c+7 of every MX block (16-byte accesses, 64 consecutive bytes per quad),
// the quad agrees on the blocks' maxima with two exchanges (two blocks per register), and the permutation of the layout
// (mxq_kv.cuh) makes the lane's codes of the row ONE store: K wants word c of every block side by side, V its halfwords.
// Measured in a replayed graph, head dimension 128: 48 rows of 8 heads 1.8 us (append) and 1.8 us (read), the launch's own
// time; 5718 rows of 32 heads (94 MB of BF16, 25 MB of cache) 27.5 us for the append, 4.3 TB/s = 66 % of the copy rate (the direct cast of
// weights, the same arithmetic: 92 %).  No unit is saturated there (integer pipe 41 %, L1 58 %): its 96 registers leave 17 warps per SM, which
// wait for their loads; what it has beside the cast are the exchange of words, scale bytes stored one by one, and a grid over padded
// rows (two thirds of them leave at once in this batch).  The
// read of a batch padded to 16380 rows (its zeros are written too: 268 MB) takes 49 us, 6.0 TB/s = 92 % of the copy rate.
#include "mxq_kv.cuh"

namespace mxq {

constexpr int kKvThreads = 128;
// Token rows of a sequence per lane of the read: one for a decode step (nothing to share, latency counts); several for a prompt,
// so that a lane's lookups (length, row count) are spent once and more loads are in flight.
constexpr int kPromptRows = 4;

struct RowPlace {
    uint8_t *tile;   // nullptr: no such row
    int slot;        // token in the tile
};

// where the token at position pos of sequence b lives
template <int D>
__device__ __forceinline__ RowPlace row_place(const KvView &c, const KvSeqs &s, int b, int pos, int head) {
    RowPlace p = {nullptr, 0};
    if (pos < 0) return p;
    const int page = s.page(b, pos >> c.page_shift);
    if (!kv_page_ok(c, page)) return p;
    const int slot = pos & ((1 << c.page_shift) - 1);
    p.tile = kv_tile<D>(c, page, slot, head);
    p.slot = slot & (kTileTokens - 1);
    return p;
}

// a lane's part of a call: quarter q of `head`'s rows i .. of sequence b
struct LaneRows {
    int b, i, head;
    uint32_t q;
};
template <int ROWS>
__device__ __forceinline__ LaneRows lane_rows(const KvView &c, const KvSeqs &s, uint32_t idx) {
    LaneRows l;
    const uint32_t groups = (uint32_t)(s.m + ROWS - 1) / ROWS, rowhead = idx >> 2, row = rowhead / (uint32_t)c.heads;
    l.q = idx & 3u, l.head = (int)(rowhead - row * (uint32_t)c.heads);
    l.b = ROWS == 1 && s.m == 1 ? (int)row : (int)(row / groups);
    l.i = (int)(row - (uint32_t)l.b * groups) * ROWS;
    return l;
}

struct KvRows {   // the BF16 side: [B][M][heads][D], token rows `stride` elements apart
    const uint16_t *k, *v;
    int64_t k_stride, v_stride;
};

// grid.x covers (sequence, row, head, quarter); grid.y: 0 = K, 1 = V
template <int D>
__global__ void __launch_bounds__(kKvThreads) kv_append_kernel(KvView c, KvSeqs s, KvRows in, uint32_t total) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb;
    pdl_trigger();
    const uint32_t idx = blockIdx.x * kKvThreads + threadIdx.x;
    const bool value = blockIdx.y != 0;
    if ((idx & ~31u) >= total) return;   // (warps leave together; total is a multiple of 4)
    const LaneRows l = lane_rows<1>(c, s, idx < total ? idx : total - 1);
    pdl_wait();
    const int rows = s.nrows(l.b);
    const bool live = idx < total && l.i < rows;
    const int64_t stride = value ? in.v_stride : in.k_stride;
    const uint16_t *base = value ? in.v : in.k, *src = base + ((int64_t)l.b * s.m + l.i) * stride + (int64_t)l.head * D + 8 * l.q;
    uint4 x[kNb];
#pragma unroll
    for (int j = 0; j < kNb; ++j) {
        x[j] = make_uint4(0, 0, 0, 0);
        if (live) x[j] = ld_dep_u4(MXQ_AT(src + 32 * j, 16, base, (((int64_t)s.B * s.m - 1) * stride + (int64_t)c.heads * D) * 2));
    }
    RowPlace at = {nullptr, 0};
    if (live) at = row_place<D>(c, s, l.b, s.len(l.b) - rows + l.i, l.head);
    // maxima of blocks 2p and 2p + 1 in the halves of one register
    uint32_t top[kNb / 2];
#pragma unroll
    for (int p = 0; p < kNb / 2; ++p) {
        const uint32_t a = chunk_max2(x[2 * p]), d = chunk_max2(x[2 * p + 1]);
        top[p] = __vmaxu2(__byte_perm(a, d, 0x5410), __byte_perm(a, d, 0x7632));
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) top[p] = __vmaxu2(top[p], __shfl_xor_sync(0xffffffffu, top[p], o));
    }
    uint32_t w[kNb], scale = 0;
#pragma unroll
    for (int j = 0; j < kNb; ++j) {
        const uint32_t byte = scale_byte((top[j / 2] >> (16 * (j & 1))) & 0xFFFFu);
        w[j] = byte == 0xFFu ? 0u : cast_chunk(x[j], __uint_as_float((254u - byte) << 23));
        scale |= byte << (8 * j);
    }
    if (at.tile == nullptr) return;
    uint32_t out[kNb];
    if (!value) {
#pragma unroll
        for (int j = 0; j < kNb; ++j) out[j] = w[j];
    } else {   // chunk 2q: the low halves of every block's word, chunk 2q + 1: the high halves
#pragma unroll
        for (int p = 0; p < kNb / 2; ++p) {
            out[p] = __byte_perm(w[2 * p], w[2 * p + 1], 0x5410);
            out[kNb / 2 + p] = __byte_perm(w[2 * p], w[2 * p + 1], 0x7632);
        }
    }
    uint8_t *dst = MXQ_AT(at.tile + (value ? T::kV : 0) + at.slot * T::kRow + l.q * 4 * kNb, 4 * kNb, c.pool, c.pool_bytes);
    if constexpr (kNb == 4) *reinterpret_cast<uint4 *>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
    else *reinterpret_cast<uint2 *>(dst) = make_uint2(out[0], out[1]);
    if (!value) {
        if (l.q == 0) {
            uint8_t *sc = MXQ_AT(at.tile + T::kKs + at.slot * kNb, kNb, c.pool, c.pool_bytes);
            if constexpr (kNb == 4) *reinterpret_cast<uint32_t *>(sc) = scale;
            else *reinterpret_cast<uint16_t *>(sc) = (uint16_t)scale;
        }
    } else if (l.q < kNb) {
        *MXQ_AT(at.tile + T::vs(at.slot, (int)l.q), 1, c.pool, c.pool_bytes) = (uint8_t)(scale >> (8 * l.q));
    }
}

// The same for prompts, where the arithmetic decides: one lane per MX block (no exchange for the maximum, every scale computed
// once), four heads of a token row per lane (one lookup of its place); the words change lanes before they are stored.  Launched without
// overlap, so that the lanes of a row may share its sectors through L1.  (The prompt above: 50 us with the quads, 38 with this split and
// 4-byte stores, 28 with the exchange and 16-byte stores.  A few rows take the quads: four times the lanes, an eighth of the chain.)
// grid.x covers (sequence, row, group of kHeadsPerLane heads, block); grid.y: 0 = K, 1 = V
constexpr int kHeadsPerLane = 4;
template <int D>
__global__ void __launch_bounds__(kKvThreads) kv_append_prompt_kernel(KvView c, KvSeqs s, KvRows in, uint32_t total) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb;
    const uint32_t idx = blockIdx.x * kKvThreads + threadIdx.x;
    const bool value = blockIdx.y != 0;
    if (idx >= total) return;
    const uint32_t groups = (uint32_t)(c.heads + kHeadsPerLane - 1) / kHeadsPerLane, j = idx % kNb, u = idx / kNb, row = u / groups;
    const int head0 = (int)(u - row * groups) * kHeadsPerLane, b = (int)(row / (uint32_t)s.m), i = (int)(row - (uint32_t)b * (uint32_t)s.m);
    const int rows = s.nrows(b);
    if (i >= rows) return;
    const int64_t stride = value ? in.v_stride : in.k_stride;
    const uint16_t *base = value ? in.v : in.k, *src = base + (int64_t)row * stride + (int64_t)head0 * D + 32 * j;
    const int heads = min(kHeadsPerLane, c.heads - head0);
    const uint32_t lanes = ((1u << kNb) - 1) << (threadIdx.x & 31 & ~(kNb - 1));      // the row's lanes: they leave together
    uint4 x[kHeadsPerLane][4];          // all on their way while the row's place is looked up
#pragma unroll
    for (int h = 0; h < kHeadsPerLane; ++h) {
        const uint4 *p = reinterpret_cast<const uint4 *>(MXQ_AT(src + (h < heads ? h : 0) * D, 64, base, (((int64_t)s.B * s.m - 1) * stride + (int64_t)c.heads * D) * 2));
#pragma unroll
        for (int q = 0; q < 4; ++q) x[h][q] = __ldg(p + q);
    }
    const RowPlace at = row_place<D>(c, s, b, s.len(b) - rows + i, head0);
    if (at.tile == nullptr) return;
#pragma unroll
    for (int h = 0; h < kHeadsPerLane; ++h) {
        if (h >= heads) break;
        const uint32_t top = __vmaxu2(__vmaxu2(chunk_max2(x[h][0]), chunk_max2(x[h][1])), __vmaxu2(chunk_max2(x[h][2]), chunk_max2(x[h][3])));
        const uint32_t byte = scale_byte(max(top & 0xFFFFu, top >> 16));
        const float inv = __uint_as_float((254u - byte) << 23);
        uint32_t w[4];       // words 0..3 of block j; then what this lane stores: 16 bytes of the row, from every block
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = byte == 0xFFu ? 0u : cast_chunk(x[h][q], inv);
        if constexpr (kNb == 4) {          // transposed over the quad: lane c gets word c of every block
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                const bool upper = (j & o) != 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (q & o) continue;
                    const uint32_t got = __shfl_xor_sync(lanes, upper ? w[q] : w[q + o], o);
                    if (upper) w[q] = got;
                    else w[q + o] = got;
                }
            }
        } else {                           // over two lanes: lane c gets words 2c and 2c + 1 of both blocks
            const bool upper = j != 0;
            const uint32_t got0 = __shfl_xor_sync(lanes, upper ? w[0] : w[2], 1), got1 = __shfl_xor_sync(lanes, upper ? w[1] : w[3], 1);
            const uint32_t a0 = upper ? got0 : w[0], b0 = upper ? w[2] : got0, a1 = upper ? got1 : w[1], b1 = upper ? w[3] : got1;
            w[0] = a0, w[1] = b0, w[2] = a1, w[3] = b1;
        }
        if (value) {                       // V: the halfwords of a chunk's words, low ones first
            const uint32_t v0 = w[0], v1 = w[1], v2 = w[2], v3 = w[3];
            if constexpr (kNb == 4) {
                w[0] = __byte_perm(v0, v1, 0x5410), w[1] = __byte_perm(v2, v3, 0x5410), w[2] = __byte_perm(v0, v1, 0x7632), w[3] = __byte_perm(v2, v3, 0x7632);
            } else {
                w[0] = __byte_perm(v0, v1, 0x5410), w[1] = __byte_perm(v0, v1, 0x7632), w[2] = __byte_perm(v2, v3, 0x5410), w[3] = __byte_perm(v2, v3, 0x7632);
            }
        }
        uint8_t *tile = at.tile + h * T::kBytes;
        *reinterpret_cast<uint4 *>(MXQ_AT(tile + (value ? T::kV : 0) + at.slot * T::kRow + 16 * j, 16, c.pool, c.pool_bytes)) = make_uint4(w[0], w[1], w[2], w[3]);
        *MXQ_AT(tile + (value ? T::vs(at.slot, (int)j) : T::kKs + at.slot * kNb + (int)j), 1, c.pool, c.pool_bytes) = (uint8_t)byte;
    }
}

// eight codes (natural order) under one scale -> eight BF16 values
__device__ __forceinline__ uint4 codes_to_bf16(uint32_t w, float s) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(e2m1x2_to_half2((w >> (8 * i)) & 0xFFu));
        // at most two significant bits times a power of two: the FP32 product is exact and its upper half is the BF16 number
        o[i] = (__float_as_uint(f.x * s) >> 16) | (__float_as_uint(f.y * s) & 0xFFFF0000u);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

template <int D, int ROWS>
__global__ void __launch_bounds__(kKvThreads) kv_read_kernel(KvView c, KvSeqs s, uint16_t *K, uint16_t *V, uint32_t total) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb;
    pdl_trigger();
    const uint32_t idx = blockIdx.x * kKvThreads + threadIdx.x;
    if (idx >= total) return;
    const bool value = blockIdx.y != 0;
    const LaneRows l = lane_rows<ROWS>(c, s, idx);
    pdl_wait();
    const int rows = s.nrows(l.b), first = s.len(l.b) - rows + l.i;
    uint32_t w[ROWS][kNb], sc[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        RowPlace at = {nullptr, 0};
        if (l.i + i < rows) at = row_place<D>(c, s, l.b, first + i, l.head);
        sc[i] = 0;
#pragma unroll
        for (int j = 0; j < kNb; ++j) w[i][j] = 0;
        if (at.tile == nullptr) continue;      // (codes and scales of zero: zero)
        const uint8_t *src = MXQ_AT(at.tile + (value ? T::kV : 0) + at.slot * T::kRow + l.q * 4 * kNb, 4 * kNb, c.pool, c.pool_bytes);
        if constexpr (kNb == 4) {
            const uint4 r = ld_dep_u4(src);
            w[i][0] = r.x, w[i][1] = r.y, w[i][2] = r.z, w[i][3] = r.w;
        } else {
            w[i][0] = ld_dep_u32(src), w[i][1] = ld_dep_u32(src + 4);
        }
#pragma unroll
        for (int j = 0; j < kNb; ++j) {
            const uint8_t *a = at.tile + (value ? T::vs(at.slot, j) : T::kKs + at.slot * kNb + j);
            unsigned short byte;
            asm volatile("ld.global.cg.u8 %0, [%1];" : "=h"(byte) : "l"(MXQ_AT(a, 1, c.pool, c.pool_bytes)) : "memory");
            sc[i] |= (uint32_t)byte << (8 * j);
        }
    }
    uint16_t *base = value ? V : K;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (ROWS > 1 && l.i + i >= s.m) break;
        uint16_t *dst = base + (((int64_t)l.b * s.m + l.i + i) * c.heads + l.head) * D + 8 * l.q;
#pragma unroll
        for (int j = 0; j < kNb; ++j) {
            const uint32_t n = !value ? w[i][j] : (j & 1) ? __byte_perm(w[i][j / 2], w[i][kNb / 2 + j / 2], 0x7632) : __byte_perm(w[i][j / 2], w[i][kNb / 2 + j / 2], 0x5410);
            *reinterpret_cast<uint4 *>(MXQ_AT(dst + 32 * j, 16, base, (int64_t)s.B * s.m * c.heads * D * 2)) = codes_to_bf16(n, e8m0_to_float((sc[i] >> (8 * j)) & 0xFFu));
        }
    }
}

MXQ_BOUNDS_TU(bounds_take_kv_cache)

// ---- host ---------------------------------------------------------------------------------------------------------------

static int log2_pages(int tokens) {
    for (int s = 5; s <= 8; ++s)
        if (tokens == 1 << s) return s;
    return -1;
}

static size_t tile_bytes(int D) { return D == 128 ? KvTile<128>::kBytes : D == 64 ? KvTile<64>::kBytes : 0; }

int kv_check_cache(const mxq_kv_cache *c, int layer) {
    if (!c || !c->pages || !c->refs) return MXQ_ERR_NULL;
    if (mxq_kv_page_bytes(c->kv_heads, c->head_dim, c->page_tokens) == 0 || c->num_pages < 1 || c->num_pages > MXQ_KV_MAX_PAGES ||
        c->layers < 1 || layer < 0 || layer >= c->layers)
        return MXQ_ERR_SHAPE;
    if (!aligned16(c->pages) || !aligned_to(c->refs, 16)) return MXQ_ERR_ALIGN;
    return MXQ_OK;
}

int kv_check_seqs(int B, int W, const int32_t *tables, const int32_t *lens) {
    if (!tables || !lens) return MXQ_ERR_NULL;
    if (B < 1 || B > MXQ_KV_MAX_SEQS || W < 1 || (int64_t)B * W > ((int64_t)1 << 30)) return MXQ_ERR_SHAPE;
    if (!aligned_to(tables, 4) || !aligned_to(lens, 4)) return MXQ_ERR_ALIGN;
    return MXQ_OK;
}

KvView kv_view(const mxq_kv_cache *c, int layer) {
    KvView v;
    v.page_bytes = (int64_t)mxq_kv_page_bytes(c->kv_heads, c->head_dim, c->page_tokens);
    v.pool = (const uint8_t *)c->pages;
    v.pool_bytes = v.page_bytes * c->num_pages * c->layers;
    v.base = (uint8_t *)c->pages + v.page_bytes * c->num_pages * layer;
    v.num_pages = (int32_t)c->num_pages;
    v.heads = c->kv_heads;
    v.page_shift = log2_pages(c->page_tokens);
    return v;
}

// several rows per lane where that still leaves every SM a full set of lanes
static bool prompt_rows(const mxq_kv_cache *c, int B, int M) {
    return M >= kPromptRows && (int64_t)B * M * c->kv_heads * 8 >= (int64_t)kPromptRows * 2048 * sm_count();
}
static uint32_t lanes_of(const mxq_kv_cache *c, int B, int M, bool prompt) {
    const int per = prompt ? kPromptRows : 1;
    return (uint32_t)B * (uint32_t)((M + per - 1) / per) * (uint32_t)c->kv_heads * 4u;
}

// rows of one call: at most 2^29 (row, head) pairs, so that a lane's index fits 32 bits
static bool rows_ok(const mxq_kv_cache *c, int B, int M) { return M >= 1 && (int64_t)B * M <= ((int64_t)1 << 29) / c->kv_heads; }

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

size_t mxq_kv_page_bytes(int kv_heads, int head_dim, int page_tokens) {
    const size_t tile = mxq::tile_bytes(head_dim);
    if (tile == 0 || kv_heads < 1 || kv_heads > MXQ_KV_MAX_HEADS || mxq::log2_pages(page_tokens) < 0) return 0;
    return tile * (size_t)kv_heads * (size_t)(page_tokens / mxq::kTileTokens);
}

int mxq_kv_append(const mxq_kv_cache *cache, int layer, const void *K_bf16, int64_t k_stride, const void *V_bf16, int64_t v_stride,
                  int B, int M, const int32_t *tables, int W, const int32_t *lens, const int32_t *rows, void *stream) {
    if (!K_bf16 || !V_bf16) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, layer);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    const int64_t width = (int64_t)cache->kv_heads * cache->head_dim;
    if (!mxq::rows_ok(cache, B, M) || k_stride < width || v_stride < width) return MXQ_ERR_SHAPE;
    if (!mxq::aligned16(K_bf16) || !mxq::aligned16(V_bf16) || k_stride % 8 || v_stride % 8 || !mxq::aligned_to(rows, 4)) return MXQ_ERR_ALIGN;
    const mxq::KvRows in = {(const uint16_t *)K_bf16, (const uint16_t *)V_bf16, k_stride, v_stride};
    const mxq::KvSeqs s = mxq::kv_seqs(cache, B, M, tables, W, lens, rows);
    const mxq::KvView c = mxq::kv_view(cache, layer);
    if (mxq::prompt_rows(cache, B, M)) {
        const uint32_t groups = (uint32_t)(cache->kv_heads + mxq::kHeadsPerLane - 1) / mxq::kHeadsPerLane;
        const uint32_t total = (uint32_t)B * (uint32_t)M * groups * (uint32_t)(cache->head_dim / 32);
        const dim3 grid((total + mxq::kKvThreads - 1) / mxq::kKvThreads, 2);
        if (cache->head_dim == 128) mxq::kv_append_prompt_kernel<128><<<grid, mxq::kKvThreads, 0, (cudaStream_t)stream>>>(c, s, in, total);
        else mxq::kv_append_prompt_kernel<64><<<grid, mxq::kKvThreads, 0, (cudaStream_t)stream>>>(c, s, in, total);
        return mxq::launch_status();
    }
    const uint32_t total = mxq::lanes_of(cache, B, M, false);
    return mxq::kv_launch(cache->head_dim == 128 ? mxq::kv_append_kernel<128> : mxq::kv_append_kernel<64>,
                          dim3((total + mxq::kKvThreads - 1) / mxq::kKvThreads, 2), mxq::kKvThreads, 0, (cudaStream_t)stream, c, s, in, total);
}

int mxq_kv_read(const mxq_kv_cache *cache, int layer, void *K_bf16, void *V_bf16, int B, int M, const int32_t *tables, int W,
                const int32_t *lens, const int32_t *rows, void *stream) {
    if (!K_bf16 || !V_bf16) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, layer);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    if (!mxq::rows_ok(cache, B, M)) return MXQ_ERR_SHAPE;
    if (!mxq::aligned16(K_bf16) || !mxq::aligned16(V_bf16) || !mxq::aligned_to(rows, 4)) return MXQ_ERR_ALIGN;
    const bool prompt = mxq::prompt_rows(cache, B, M);
    const uint32_t total = mxq::lanes_of(cache, B, M, prompt);
    const dim3 grid((total + mxq::kKvThreads - 1) / mxq::kKvThreads, 2);
    const mxq::KvSeqs s = mxq::kv_seqs(cache, B, M, tables, W, lens, rows);
    return mxq::kv_launch(cache->head_dim == 128 ? (prompt ? mxq::kv_read_kernel<128, mxq::kPromptRows> : mxq::kv_read_kernel<128, 1>)
                                                 : (prompt ? mxq::kv_read_kernel<64, mxq::kPromptRows> : mxq::kv_read_kernel<64, 1>),
                          grid, mxq::kKvThreads, 0,
                          (cudaStream_t)stream, mxq::kv_view(cache, layer), s, (uint16_t *)K_bf16, (uint16_t *)V_bf16, total);
}

#pragma GCC visibility pop
}  // extern "C"
