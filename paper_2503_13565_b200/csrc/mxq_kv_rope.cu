// mxq_kv_append_rope: rotary positions on the way into the cache.  The queries of the new token rows are rotated and stored, the keys
// rotated and cast into the pages of the 4-bit cache, the values cast, in one launch; mxq_rope_table computes the table it reads.
//
//     (x_a, x_b) -> (x_a cos - x_b sin, x_b cos + x_a sin)      for the pairs (a, b) of a head: (d, d + R/2) or (2d, 2d + 1)
//
// A stream like the append itself: 2 bytes per element read, 2 (queries) or 0.53 (keys, values) written.  The rotation is FP32 with every
// product and sum rounded once (no contraction), so that a row's codes are defined to the bit; keys are cast from there, without a
// stop at BF16.  A warp has one token row: its lookups and angles serve all heads, and four lanes share a head as in the append.
// Measured in a replayed graph: one row of 32 + 8 heads 2.2 us, 61 x 9 rows of a token tree 2.7 us (launch and three dependent loads: length,
// table row, page); 13958 rows of 32 + 8 heads of 128 in a batch padded to 3 x 8191 (395 MB, the zeros of the queries that are not there among them)
// 73 us, 5.4 TB/s = 82 % of the copy rate: what is missing are warps (103 registers, 16 warps per SM) to cover the loads.
#include "mxq_kv.cuh"

namespace mxq {

constexpr int kRopeThreads = 128;
enum { kPairs = 0, kWhole = 1, kHalves = 2 };   // neighbours; halves of a head that is rotated whole; halves of its first part

struct RopeCall {
    const float *table;      // [positions][R]: cos, sin
    const int32_t *where;    // [B][M] or nullptr
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    int64_t q_stride, qo_stride, k_stride, v_stride;
    int64_t positions;
    int32_t q_heads, rotary;
    int32_t parts, rounds;   // warps per token row, groups of eight heads per warp
};

template <int D>
struct Unit {                // one head of a token row: a query, key or value
    const uint16_t *src, *base;
    int64_t extent;          // bytes from base on
    int kind, head;          // kind 0 query, 1 key, 2 value, 3 none
};

template <int D>
__device__ __forceinline__ Unit<D> rope_unit(const RopeCall &r, const KvSeqs &s, int kv_heads, int64_t row, int unit) {
    Unit<D> u;
    u.kind = unit < r.q_heads ? 0 : unit < r.q_heads + kv_heads ? 1 : unit < r.q_heads + 2 * kv_heads ? 2 : 3;
    u.head = u.kind == 0 ? unit : unit - r.q_heads - (u.kind == 2 ? kv_heads : 0);
    const int64_t stride = u.kind == 0 ? r.q_stride : u.kind == 1 ? r.k_stride : r.v_stride;
    u.base = u.kind == 0 ? r.q : u.kind == 1 ? r.k : r.v;
    u.src = u.base + row * stride + (int64_t)u.head * D;
    u.extent = (((int64_t)s.B * s.m - 1) * stride + (int64_t)(u.kind == 0 ? r.q_heads : kv_heads) * D) * 2;
    return u;
}

// eight entries of the table, NaN where the position lies outside it
__device__ __forceinline__ void table8(float (&f)[8], const RopeCall &r, int64_t pos, int at) {
    if ((uint64_t)pos >= (uint64_t)r.positions) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(0x7FC00000u);
        return;
    }
    const float4 *p = reinterpret_cast<const float4 *>(MXQ_AT(r.table + pos * r.rotary + at, 32, r.table, r.positions * r.rotary * 4));
    const float4 a = __ldg(p), b = __ldg(p + 1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ void table4(float (&f)[4], const RopeCall &r, int64_t pos, int at) {
    if ((uint64_t)pos >= (uint64_t)r.positions) {
        f[0] = f[1] = f[2] = f[3] = __uint_as_float(0x7FC00000u);
        return;
    }
    const float4 a = __ldg(reinterpret_cast<const float4 *>(MXQ_AT(r.table + pos * r.rotary + at, 16, r.table, r.positions * r.rotary * 4)));
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
}

// the two results of a pair, every operation rounded once
__device__ __forceinline__ float turn_a(float a, float b, float c, float s) { return __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s)); }
__device__ __forceinline__ float turn_b(float a, float b, float c, float s) { return __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s)); }

// A warp takes a token row, eight heads at a time: lane q of a quad holds elements 8q .. 8q+7 of every MX block of the quad's head
// (16-byte accesses; what the quad stores of a key or a value is as in the append).  The row's angles stay in registers over the heads.
template <int D, int MODE>
__global__ void __launch_bounds__(kRopeThreads) kv_append_rope_kernel(KvView c, KvSeqs s, RopeCall r, uint32_t warps) {
    constexpr int kNb = D / 32;
    pdl_trigger();
    const uint32_t warp = blockIdx.x * (kRopeThreads / 32) + threadIdx.x / 32;
    pdl_wait();
    if (warp >= warps) return;
    const uint32_t row = warp / (uint32_t)r.parts, part = warp - row * (uint32_t)r.parts;
    const int b = (int)(row / (uint32_t)s.m), i = (int)(row - (uint32_t)b * (uint32_t)s.m);
    const int quad = (threadIdx.x & 31) >> 2, q = threadIdx.x & 3;
    const uint32_t lanes = 0xFu << (4 * quad);
    int unit = (int)part * r.rounds * 8 + quad;

    // a decode step's heads are on their way before the row's place is known; a prompt's wait for it, since rows that are not there are not read
    uint4 x[kNb];
    Unit<D> u = rope_unit<D>(r, s, c.heads, row, unit);
    auto load = [&]() {
#pragma unroll
        for (int j = 0; j < kNb; ++j)
            if (u.kind != 3) x[j] = ld_dep_u4(MXQ_AT(u.src + 32 * j + 8 * q, 16, u.base, u.extent));
    };
    if (r.rounds == 1) load();

    const int rows = s.nrows(b), place = s.len(b) - rows + i;
    const bool there = i < rows && place >= 0;
    if (!there) {            // (the whole warp: it has one row)
        for (int h = unit; h < min(r.q_heads, unit + 8 * r.rounds); h += 8) {
            uint16_t *dst = r.q_out + (int64_t)row * r.qo_stride + (int64_t)h * D + 8 * q;
#pragma unroll
            for (int j = 0; j < kNb; ++j)
                *reinterpret_cast<uint4 *>(MXQ_AT(dst + 32 * j, 16, r.q_out, (((int64_t)s.B * s.m - 1) * r.qo_stride + (int64_t)r.q_heads * D) * 2)) = make_uint4(0, 0, 0, 0);
        }
        return;
    }
    if (r.rounds != 1) load();
    const int64_t pos = r.where == nullptr ? place : (int)ld_dep_u32(MXQ_AT(r.where + row, 4, r.where, (size_t)s.B * s.m * 4));
    RowPlace at = {nullptr, 0};
    at = row_place<D>(c, s, b, place, 0);
    const int half = r.rotary / 2;
    // the angles of this lane's elements: of pairs in the first half of its blocks (kWhole), of each of its blocks (kPairs)
    float cs[kNb / 2 * 8], sn[kNb / 2 * 8];
    if constexpr (MODE == kWhole) {
#pragma unroll
        for (int j = 0; j < kNb / 2; ++j) {
            float f[8], g[8];
            table8(f, r, pos, 32 * j + 8 * q), table8(g, r, pos, half + 32 * j + 8 * q);
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[8 * j + e] = f[e], sn[8 * j + e] = g[e];
        }
    } else if constexpr (MODE == kPairs) {
#pragma unroll
        for (int j = 0; j < kNb; ++j) {
            float f[4] = {1.f, 1.f, 1.f, 1.f}, g[4] = {0.f, 0.f, 0.f, 0.f};
            const int first = 32 * j + 8 * q;
            if (first < r.rotary) table4(f, r, pos, first / 2), table4(g, r, pos, half + first / 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[4 * j + e] = f[e], sn[4 * j + e] = g[e];
        }
    }

    for (int round = 0; round < r.rounds; ++round) {
        const Unit<D> now = u;
        float f[kNb][8];
#pragma unroll
        for (int j = 0; j < kNb; ++j) unpack_bf16(f[j], x[j]);
        unit += 8;
        if (round + 1 < r.rounds) {          // the next heads are on their way meanwhile
            u = rope_unit<D>(r, s, c.heads, row, unit);
            load();
        }
        if (now.kind == 3) break;            // (quads leave whole)
        if (now.kind != 2) {
            if constexpr (MODE == kWhole) {
#pragma unroll
                for (int j = 0; j < kNb / 2; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = f[j][e], z = f[j + kNb / 2][e];
                        f[j][e] = turn_a(a, z, cs[8 * j + e], sn[8 * j + e]);
                        f[j + kNb / 2][e] = turn_b(a, z, cs[8 * j + e], sn[8 * j + e]);
                    }
            } else if constexpr (MODE == kPairs) {
#pragma unroll
                for (int j = 0; j < kNb; ++j) {
                    if (32 * j + 8 * q >= r.rotary) continue;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = f[j][2 * e], z = f[j][2 * e + 1];
                        f[j][2 * e] = turn_a(a, z, cs[4 * j + e], sn[4 * j + e]);
                        f[j][2 * e + 1] = turn_b(a, z, cs[4 * j + e], sn[4 * j + e]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < kNb; ++j) {
                    const int first = 32 * j + 8 * q;
                    if (first >= r.rotary) continue;
                    const bool upper = first >= half;            // (half is a multiple of 8: the eight elements lie on one side)
                    float g[8], co[8], si[8];
                    unpack_bf16(g, ld_dep_u4(MXQ_AT(now.src + (upper ? first - half : first + half), 16, now.base, now.extent)));
                    table8(co, r, pos, upper ? first - half : first), table8(si, r, pos, upper ? first : half + first);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[j][e] = upper ? turn_b(g[e], f[j][e], co[e], si[e]) : turn_a(f[j][e], g[e], co[e], si[e]);
                }
                __syncwarp(lanes);           // (the queries may be rotated in place: the quad has read before it stores)
            }
        }
        if (now.kind == 0) {
            uint16_t *dst = r.q_out + (int64_t)row * r.qo_stride + (int64_t)now.head * D + 8 * q;
#pragma unroll
            for (int j = 0; j < kNb; ++j)
                *reinterpret_cast<uint4 *>(MXQ_AT(dst + 32 * j, 16, r.q_out, (((int64_t)s.B * s.m - 1) * r.qo_stride + (int64_t)r.q_heads * D) * 2)) = pack_bf16(f[j]);
            continue;
        }
        uint32_t w[kNb], scale = 0;
#pragma unroll
        for (int j = 0; j < kNb; ++j) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[j][e]) & 0x7FFFFFFFu);
            top = max(top, __shfl_xor_sync(lanes, top, 1));
            top = max(top, __shfl_xor_sync(lanes, top, 2));
            const uint32_t byte = scale_byte(top >> 16);         // (the upper half has the whole exponent)
            const float inv = __uint_as_float((254u - byte) << 23);
            w[j] = 0;
            if (byte != 0xFFu) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[j] |= float2_to_e2m1x2(f[j][2 * e] * inv, f[j][2 * e + 1] * inv) << (8 * e);
            }
            scale |= byte << (8 * j);
        }
        if (at.tile == nullptr) continue;
        const RowPlace mine = {at.tile + (int64_t)now.head * KvTile<D>::kBytes, at.slot};
        store_quarter<D>(c, mine, now.kind == 2, (uint32_t)q, w, scale);
    }
}

// One thread per (position, pair).  Made once per model: 131072 positions of 64 pairs take 40 us (67 MB: 10 us at the copy rate), the sine and cosine
// in 64 bits the most of it, which far positions need.
__global__ void __launch_bounds__(256) rope_table_kernel(const double *inv_freq, int64_t positions, int half, float amplitude, float *table) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= positions * half) return;
    const int64_t p = at / half, i = at - p * half;
    double sn, cs;
    sincos((double)p * *MXQ_AT(inv_freq + i, 8, inv_freq, half * 8), &sn, &cs);
    *MXQ_AT(table + p * 2 * half + i, 4, table, positions * half * 8) = (float)(amplitude * cs);
    *MXQ_AT(table + p * 2 * half + half + i, 4, table, positions * half * 8) = (float)(amplitude * sn);
}

MXQ_BOUNDS_TU(bounds_take_kv_rope)

// ---- host ---------------------------------------------------------------------------------------------------------------

template <int D>
static int rope_launch(int mode, const KvView &c, const KvSeqs &s, RopeCall r, cudaStream_t stream) {
    // few rows: a warp per eight heads, so that a row's latency is one load's; many rows: a warp per row, whose lookups and angles
    // are then shared by all of its heads
    const int64_t rows = (int64_t)s.B * s.m, groups = (r.q_heads + 2 * (int64_t)c.heads + 7) / 8, slots = (int64_t)sm_count() * 32;
    r.rounds = (int)max((int64_t)1, min(groups, rows * groups / slots));
    r.parts = (int)((groups + r.rounds - 1) / r.rounds);
    const uint32_t warps = (uint32_t)(rows * r.parts);
    const dim3 grid((warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32));
    return launch_pdl(mode == kPairs ? kv_append_rope_kernel<D, kPairs> : mode == kWhole ? kv_append_rope_kernel<D, kWhole> : kv_append_rope_kernel<D, kHalves>,
                      grid, kRopeThreads, 0, stream, c, s, r, warps);
}

static bool rotary_ok(int rotary) { return rotary >= 16 && rotary % 16 == 0; }

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

int mxq_rope_table(const double *inv_freq, int64_t positions, int rotary_dim, float amplitude, float *table, void *stream) {
    if (!inv_freq || !table) return MXQ_ERR_NULL;
    if (positions < 1 || positions > ((int64_t)1 << 31) || !mxq::rotary_ok(rotary_dim) || rotary_dim > 128) return MXQ_ERR_SHAPE;
    if (!mxq::aligned_to(inv_freq, 8) || !mxq::aligned16(table)) return MXQ_ERR_ALIGN;
    const int64_t ctas = (positions * (rotary_dim / 2) + 255) / 256;
    mxq::rope_table_kernel<<<(unsigned)ctas, 256, 0, (cudaStream_t)stream>>>(inv_freq, positions, rotary_dim / 2, amplitude, table);
    return mxq::launch_status();
}

int mxq_kv_append_rope(const mxq_kv_cache *cache, int layer, const void *Q_bf16, int64_t q_stride, int q_heads, void *Q_out, int64_t q_out_stride,
                       const void *K_bf16, int64_t k_stride, const void *V_bf16, int64_t v_stride, int B, int M, const int32_t *tables, int W,
                       const int32_t *lens, const int32_t *rows, const mxq_rope *rope, const int32_t *positions, void *stream) {
    if (!K_bf16 || !V_bf16 || !rope || !rope->table || !Q_bf16 != !Q_out) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, layer);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    const int D = cache->head_dim;
    const int64_t width = (int64_t)cache->kv_heads * D;
    if (!Q_bf16) q_heads = 0, q_stride = q_out_stride = 0;
    else if (q_heads < 1 || q_heads > 65536 || q_stride < (int64_t)q_heads * D || q_out_stride < (int64_t)q_heads * D) return MXQ_ERR_SHAPE;
    if (!mxq::kv_rows_ok(q_heads + 2 * cache->kv_heads, B, M) || k_stride < width || v_stride < width || !mxq::rotary_ok(rope->rotary_dim) ||
        rope->rotary_dim > D || (rope->style != MXQ_ROPE_HALVES && rope->style != MXQ_ROPE_PAIRS) || rope->positions < 1 ||
        rope->positions > ((int64_t)1 << 31))
        return MXQ_ERR_SHAPE;
    if (!mxq::aligned16(K_bf16) || !mxq::aligned16(V_bf16) || !mxq::aligned16(Q_bf16) || !mxq::aligned16(Q_out) || !mxq::aligned16(rope->table) ||
        k_stride % 8 || v_stride % 8 || q_stride % 8 || q_out_stride % 8 || !mxq::aligned_to(rows, 4) || !mxq::aligned_to(positions, 4))
        return MXQ_ERR_ALIGN;
    mxq::RopeCall r;
    r.table = rope->table, r.where = positions, r.positions = rope->positions, r.rotary = rope->rotary_dim;
    r.q = (const uint16_t *)Q_bf16, r.k = (const uint16_t *)K_bf16, r.v = (const uint16_t *)V_bf16, r.q_out = (uint16_t *)Q_out;
    r.q_stride = q_stride, r.qo_stride = q_out_stride, r.k_stride = k_stride, r.v_stride = v_stride, r.q_heads = q_heads;
    r.parts = r.rounds = 0;
    const mxq::KvSeqs s = mxq::kv_seqs(cache, B, M, tables, W, lens, rows);
    const mxq::KvView c = mxq::kv_view(cache, layer);
    const int mode = rope->style == MXQ_ROPE_PAIRS ? mxq::kPairs : rope->rotary_dim == D ? mxq::kWhole : mxq::kHalves;
    return D == 128 ? mxq::rope_launch<128>(mode, c, s, r, (cudaStream_t)stream) : mxq::rope_launch<64>(mode, c, s, r, (cudaStream_t)stream);
}

#pragma GCC visibility pop
}  // extern "C"
