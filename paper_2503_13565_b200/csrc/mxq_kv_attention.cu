// mxq_kv_attention: softmax(scale * q . K^T) . V over the pages of a 4-bit cache.
//
// The mathematics.  A step reads every K and V row of the cache once (D + D / 16 bytes per token and kv head) for a handful
// of query rows, so the cache's bytes bound it as long as decoding 4-bit codes and the two products keep up with them.
//   - One pass with a running maximum m and sum l per row (base 2: the softmax scale times log2 e multiplies the score).
//     The maximum only moves when a score exceeds it by 2^4 (kMaxSlack), so that the warp-wide reduction and the rescaling of
//     the accumulators happen a few times per sequence, not per tile; weights up to 2^4 are accounted for in the ranges below.
//   - Both products run on m16n8k16 with the TOKENS (K) or the head dimension (V) as the 16 rows and eight query rows as the
//     8 columns: a decode step with few rows wastes no half of a 16-row tile.  Codes become FP16 with the conversion
//     instruction, exactly, without their scales.
//   - K: S^T[16 tokens][8 rows] += K[16][16 d] . Q^T.  A block of 32 d is two instructions; their sum is scaled per token in
//     FP32 (the product of codes and q is exact, q being normalised per row by a power of two to a largest element of 2^14 in
//     FP16, which holds BF16's 8 bits over 2^28 of range below it).  So a score stays finite while K is below 2^103.
//   - V: O^T[16 d][8 rows] += V^T[16 d][16 tokens] . P^T.  V's scale varies along the contracted tokens and per block of
//     32 d, so it goes into P: one multiplication of the packed weights per block, shared by the block's two instructions.
//     FP16 holds P * scale at 11 bits over 2^24 between the largest weight times the largest scale met so far (`ref`, an
//     exponent common to the warp's accumulators) and the smallest.  Weights below that are still right to 11 bits: a tile that has any
//     adds them in a second product over accumulators scaled up by the width of the first (two tiers; four for weights smaller
//     yet).  A tile with weights or scales spread even wider, or a NaN scale, takes the step in BF16, whose range holds any, with
//     the weights as a sum of two BF16 numbers.  (The tiers took the long case below, peaked weights, from 0.61 to 0.39 ms.)
//   - S^T leaves the tensor core with a lane holding one token and two rows; the second product wants one row and two
//     tokens: one 8x8 transposition (movmatrix) per packed register.
//
// The split.  Lengths live on the device, so the grid is fixed: as many CTAs as fit.  The work, all (sequence, kv head, row tile)
// segments, is cut along the tokens into items, which CTAs draw from a counter as they become free: tiles cost between one
// product and four, and equal shares left the GPU waiting for the unluckiest CTA (batched decode 58 us, items 39).  Within an item each
// of the four warps takes every fourth 32-token tile and keeps its own m, l, O and a ring of two tiles, each filled by ONE bulk copy
// that completes on an mbarrier; no warp waits for another until the item ends.  (Waits are bounded: where a tile never arrives a
// status bit is set, the CTA requests nothing more, and what it had still to deliver is NaN.)  The results of a segment's items go to the
// workspace, in slots in the order of the tokens; the CTA that delivered the last of them adds them up in that order.  Nobody waits for it, and it learns that it was the last one item
// later, when the ticket's answer has long arrived.  So which CTA did what does not show in the result.
//
// What bounds it.  Not the bytes: 2 x 131071 tokens of 32 heads (1.14 GB) take 249 us with even weights, 4.6 TB/s = 70 % of the copy rate,
// 268 us (65 %) with peaked ones, whose tiles need the tiers; bringing the tiles in without computing takes 177 us.  No unit is saturated:
// a warp spends some 660 instructions on a tile, the integer pipe (half rate: unpacking nibbles into the order of the products, scale
// bytes) is 51 % busy, and a scheduler issues in every second cycle; the rest is the latency of one warp's chain of products, shuffles and
// exponentials, and of the barriers at an item's end, with only 12 warps per SM to hide it (the accumulators and both operands of
// 32 x 128 tiles: 165 registers).  More warps or more work per warp spill, and spills lose more than they give: the L1 is what the rings
// leave.  32 decode rows over 279 to 8047 tokens (77 MB): 39 us, 20 of them without computing; one row over 2047 tokens: 13 us, 9 without
// computing: launch, the division of the work, one item of two tiles per warp, the join; tree verification, 8 x 16 rows, head dimension
// 64: 36.5 us, 23 without computing.  Requesting the next item's tiles before this one's result is put together gained nothing (the
// SM's other CTAs fill the gap) and cost registers.
// A prompt's rows are taken, 16 flattened rows per pass over K and V, tiles behind the last token that a row sees included: 2048 rows of
// 32 heads over themselves 812 us, 256 rows behind 8192 tokens 322 us (42 and 108 TFLOP/s).
#include <math.h>

#include <atomic>
#include <type_traits>

#include "mxq_kv.cuh"
#include "mxq_kv_division.h"
#include "mxq_tcgen05.cuh"

namespace mxq {

struct KvQuery {
    const uint16_t *q;       // [B][M][heads][D], token rows q_stride elements apart
    int64_t q_stride;
    const uint64_t *tree;    // [B][M] or nullptr
    uint16_t *o;             // [B][M][heads][D]
    float *lse;              // [B][M][heads] or nullptr
    int32_t heads, group;    // query heads, query heads per kv head
    uint32_t group_magic;    // floor(2^32 / group) + 1 (0: group = 1): r / group = umulhi(r, group_magic) for r * group < 2^32
    float scale_log2;        // scale * log2(e)
    unsigned *counter;       // workspace: next item; parts delivered, per cut segment (both zero between calls); slots of partial results
    unsigned *tickets;
    float *partials;
    uint32_t slots;
#ifdef MXQ_DEBUG_BOUNDS
    int32_t lost_tile;       // test hook: this tile of sequence 0, kv head 0 is waited for but never requested
#endif
};

constexpr int kWeightBias = 10;                // weights carry a factor 2^10 from the exponential on: in FP16 they keep 11 bits down to 2^-14
constexpr float kMaxSlack = 4.f;               // how far (log2) a score may exceed the running maximum
constexpr int kScaleHeadroom = 1;              // how far (log2) a V scale may exceed `ref`: P * 2^(scale - ref) <= 2^(10 + 4 + 1) fits FP16,
constexpr int kHalfRange = 14;                 // and is a normal number while it is at least 2^-14
constexpr int kScaleSpread = 14;               // scales this far below ref still take the FP16 step
constexpr int kScaleLag = 3;                   // how far (log2) a tile's largest scale may lie below ref
constexpr int kScaleDrop = 12;                 // how far ref may fall below its highest: accumulators are below 2^18 per token, and
                                               // the deepest of the tiers below scales them by up to 2^72

template <int NT>
constexpr int kAttRows = att_rows(NT);
template <int D, int NT>
constexpr int kAttCtasPerSm = att_ctas_per_sm(D, NT);
template <int D, int NT>
constexpr size_t kAttSlotFloats = (size_t)kAttRows<NT> * (D + 2);
template <int D, int NT>
constexpr uint32_t kAttMaxParts = att_max_parts(D, NT);   // parts of a segment
template <int D, int NT>
constexpr size_t kAttSmem = (size_t)att_smem(D);

// ---- fragments ------------------------------------------------------------------------------------------------------------

// four code bytes -> four pairs of halves
__device__ __forceinline__ void decode4(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
template <bool kBf16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (kBf16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t o;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(o) : "r"(v));
    return o;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t o;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(hi), "f"(lo));
    return o;
}
__device__ __forceinline__ uint32_t pack_bf162(float lo, float hi) {
    uint32_t o;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(hi), "f"(lo));
    return o;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
    uint32_t o;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}
__device__ __forceinline__ uint32_t mul_bf162(uint32_t a, uint32_t b) {
    uint32_t o;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}
__device__ __forceinline__ uint32_t min_half2(uint32_t a, uint32_t b) {
    uint32_t o;
    asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}
__device__ __forceinline__ bool all_le_half2(uint32_t a, uint32_t b) {
    return __hble2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Scale byte j of a word as a factor: the byte in the exponent's place.  The lowest mantissa bit is set so that 0xFF is a NaN (the
// factor is then 1 + 2^-23 of the power of two, the same for every score); byte 0 becomes 2^-149: blocks scaled by 2^-127 count as zero.
template <int J>
__device__ __forceinline__ float scale_factor(uint32_t w) {
    if constexpr (J == 3) return __uint_as_float(__byte_perm(w, 0, 0x4344) * 128u | 1u);      // (shifts to the left only: they are multiplications on the other pipe)
    else return __uint_as_float((w * (1u << (23 - 8 * (J & 3))) & 0x7F800000u) | 1u);
}
__device__ __forceinline__ float scale_factor(uint32_t w, int j) {   // (j a constant after unrolling)
    return j == 0 ? scale_factor<0>(w) : j == 1 ? scale_factor<1>(w) : j == 2 ? scale_factor<2>(w) : scale_factor<3>(w);
}
// pairs of FP32 operations in one instruction
__device__ __forceinline__ uint64_t pair2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split2(uint64_t r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void scale4(float (&o)[4], float f01, float f23) {   // o[0..1] *= f01, o[2..3] *= f23
    uint64_t a, b;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a) : "l"(pair2(o[0], o[1])), "l"(pair2(f01, f01)));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(b) : "l"(pair2(o[2], o[3])), "l"(pair2(f23, f23)));
    split2(a, o[0], o[1]), split2(b, o[2], o[3]);
}

// x * 2^e for e <= 127 (below -252 as -252) in two steps
__device__ __forceinline__ float scale_by_power(float x, int e) {
    const int first = max(e, -126);
    return x * __uint_as_float((uint32_t)(first + 127) << 23) * __uint_as_float((uint32_t)(max(e - first, -126) + 127) << 23);
}
__device__ __forceinline__ uint32_t lds_u32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
template <int N>
__device__ __forceinline__ void lds_words(uint32_t a, uint32_t (&w)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "");
    if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a));
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a));
    else w[0] = lds_u32(a);
}
// ---- one segment, as its CTA sees it ----------------------------------------------------------------------------------------

struct Segment {
    int b, head, r0;         // sequence, kv head, first flattened row of the tile
    int len, base;           // tokens; tokens before the rows
    int rows_total;          // flattened rows of the sequence (token rows * group)
};

// A warp's state of a segment.  Column c of column block nt is flattened row r0 + 8 * nt + c; a lane (g = lane / 4, tig = lane % 4) holds
// columns 2 * tig and 2 * tig + 1.
__device__ unsigned int g_kv_status = 0;   // sticky: bit 0 a requested tile never arrived

struct Owner {                    // the items that a thread's sequences own, and the first of these sequences
    uint32_t big_lo, big_count, small_lo, small_count, slot_lo, tiles;
    AttCut cut;
    int len, rows;
};
struct Part {                     // a segment whose part has been delivered: its rows, how many parts it has, the first one's slot
    int b, head, r0, nrows;
    uint32_t parts, slot0;
};

template <int D, int NT>
struct WarpState {
    float o[D / 16][NT][4];   // rows of block j: d = 32 j + 4 g + {0, 1} in o[2j], + {2, 3} in o[2j + 1]; [d][column]: 00 01 10 11
    float m[NT][2], l[NT][2];     // maximum and sum; m = 0 while over = -inf
    float over[NT][2];            // how far a biased score may exceed m: kWeightBias + kMaxSlack, or -inf before the first token the row sees
    int ref, ref_max;
};

// token row of a flattened row
__device__ __forceinline__ int token_row(const KvQuery &a, int r) { return a.group_magic ? (int)__umulhi((uint32_t)r, a.group_magic) : r; }

// what a flattened row sees: tokens before `until`, and token base + j (of at most 64 rows) if bit j is set
struct Sight {
    int until, base;
    uint64_t bits;
    __device__ __forceinline__ bool sees(int t) const { return t < until || (t >= base && t < base + 64 && ((bits >> (t - base)) & 1) != 0); }
};
__device__ __noinline__ Sight sight_of(const KvSeqs &s, const KvQuery &a, const Segment &g, int r) {
    Sight v = {0, g.len, 0};                    // (no such row: nothing)
    if (r >= g.rows_total) return v;
    const int i = token_row(a, r);
    if (a.tree == nullptr) {
        v.until = min(g.base + i + 1, g.len);
        return v;
    }
    const uint64_t *p = MXQ_AT(a.tree + (int64_t)g.b * s.m + i, 8, a.tree, (size_t)s.B * s.m * 8);
    const uint32_t lo = ld_dep_u32(p), hi = ld_dep_u32(reinterpret_cast<const uint32_t *>(p) + 1);
    const int rows = g.len - g.base;
    v.until = v.base = g.base;
    v.bits = ((uint64_t)hi << 32 | lo) & (rows >= 64 ? ~0ull : (1ull << rows) - 1);
    return v;
}

template <int D, int NT>
__device__ __forceinline__ void rescale(WarpState<D, NT> &w, const float (&f)[NT][2]) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
        {
            const uint64_t ff = pair2(f[n][0], f[n][1]);
            float(&o)[4] = w.o[i][n];
            uint64_t a, b;
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a) : "l"(pair2(o[0], o[1])), "l"(ff));
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(b) : "l"(pair2(o[2], o[3])), "l"(ff));
            split2(a, o[0], o[1]), split2(b, o[2], o[3]);
        }
}

// O += P . V for a whole tile, in FP16.  p[u][n][h]: packed weights of row g of column block n, tokens 16 u + tig + 8 h (low half) and
// + 4 (high half).  kTiers == 2: deep[..] are the weights too small for p, scaled up by `up`; `down` = 1 / up.
template <int D, int NT, int kTiers>
__device__ __forceinline__ void add_values(WarpState<D, NT> &w, uint32_t tile, int g, int tig, const uint32_t (&p)[2][NT][2],
                                           const uint32_t (&deep)[2][NT][2], float up, float down) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb, kW = kNb / 2;   // words of V codes per lane and token
    // exponent field of 2^(scale - ref): never below 1 here, so both halves fit one 32-bit multiply-add
    const uint32_t bias = (uint32_t)(15 - w.ref) * (0x10001u << 10);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint32_t sw[kNb], v[4][kW];             // scales: [h, block pair] words of (A.j, B.j, A.j+1, B.j+1); codes
        lds_words<kNb>(tile + T::kVs + 16 * kNb * u + 4 * kNb * tig, sw);
#pragma unroll
        for (int k = 0; k < 4; ++k) lds_words<kW>(tile + T::kV + (16 * u + tig + 4 * k) * T::kRow + 2 * kNb * g, v[k]);
#pragma unroll
        for (int x = 0; x < kW; ++x) {
            uint32_t e[2][4], o[2][4];          // pairs (token A, token B) of even and odd elements
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t A = v[2 * h][x], B = v[2 * h + 1][x];
                decode4((A & 0x0F0F0F0Fu) | ((B * 16u) & 0xF0F0F0F0u), e[h]);
                decode4(((A >> 4) & 0x0F0F0F0Fu) | (B & 0xF0F0F0F0u), o[h]);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int j = 2 * x + y;
                uint32_t sc[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)     // (the two tokens' scales as 16-bit numbers)
                    sc[h] = __byte_perm(sw[h * kW + x], 0, y ? 0x4342 : 0x4140) * 1024u + bias;
                auto product = [&](int n, const uint32_t(&q)[2][NT][2]) {
                    const uint32_t b0 = mul_half2(q[u][n][0], sc[0]), b1 = mul_half2(q[u][n][1], sc[1]);
                    mma16816<false>(w.o[2 * j][n], e[0][2 * y], o[0][2 * y], e[1][2 * y], o[1][2 * y], b0, b1);
                    mma16816<false>(w.o[2 * j + 1][n], e[0][2 * y + 1], o[0][2 * y + 1], e[1][2 * y + 1], o[1][2 * y + 1], b0, b1);
                };
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if constexpr (kTiers == 2) {
                        scale4(w.o[2 * j][n], up, up), scale4(w.o[2 * j + 1][n], up, up);
                        product(n, deep);
                        scale4(w.o[2 * j][n], down, down), scale4(w.o[2 * j + 1][n], down, down);
                    }
                    product(n, p);
                }
            }
        }
    }
}

// The same for the 16 tokens of group u (from token t0 of the sequence on), in BF16: any spread of weights and scales; NaN scales count only where the row sees the token.
template <int D, int NT, class Sees>
__device__ __forceinline__ void add_values_wide(WarpState<D, NT> &w, uint32_t tile, int u, int t0, int g, int tig, const uint32_t (&p)[NT][2], Sees sees) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb, kW = kNb / 2;
    uint32_t sw[kNb];
    lds_words<kNb>(tile + T::kVs + 16 * kNb * u + 4 * kNb * tig, sw);
    const uint32_t row = tile + T::kV + (16 * u + tig) * T::kRow + 2 * kNb * g;
    const uint32_t bias = ((uint32_t)(127 + kWeightBias - w.ref) & 0xFFFFu) * 0x10001u;
    auto widen = [](uint32_t h) {
        const float2 f = __half22float2(*reinterpret_cast<__half2 *>(&h));
        return pack_bf162(f.x, f.y);
    };
#pragma unroll
    for (int x = 0; x < kW; ++x) {
        uint32_t ev[2][4], od[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t A = lds_u32(row + 8 * h * T::kRow + 4 * x), B = lds_u32(row + (8 * h + 4) * T::kRow + 4 * x);
            decode4((A & 0x0F0F0F0Fu) | ((B << 4) & 0xF0F0F0F0u), ev[h]);
            decode4(((A >> 4) & 0x0F0F0F0Fu) | (B & 0xF0F0F0F0u), od[h]);
#pragma unroll
            for (int i = 0; i < 4; ++i) ev[h][i] = widen(ev[h][i]), od[h][i] = widen(od[h][i]);
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int j = 2 * x + y;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t b[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t word = sw[h * kW + x];
                    uint32_t f = __viaddmax_s16x2(__byte_perm(word, 0, y ? 0x4342 : 0x4140), bias, 0u) << 7;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (((word >> (16 * y + 8 * e)) & 0xFFu) == 0xFFu)
                            f = (f & ~(0xFFFFu << (16 * e))) | ((sees(n, t0 + tig + 8 * h + 4 * e) ? 0x7FC0u : 0u) << (16 * e));
                    b[h] = mul_bf162(p[n][h], f);
                }
                mma16816<true>(w.o[2 * j][n], ev[0][2 * y], od[0][2 * y], ev[1][2 * y], od[1][2 * y], b[0], b[1]);
                mma16816<true>(w.o[2 * j + 1][n], ev[0][2 * y + 1], od[0][2 * y + 1], ev[1][2 * y + 1], od[1][2 * y + 1], b[0], b[1]);
            }
        }
    }
}

// A wait for tile number `at` of a warp, up to about a second.  It returns the same to all lanes of the warp: those that come to
// the long wait agree through a word behind the warp's barriers (tile number and outcome; the first one's stands), and where a lane has
// left the short one, the tile has arrived for good and no other can run out of time.  (A vote after every wait instead: tree
// verification 36.4 -> 37.8 us.)
__device__ __noinline__ bool tile_wait_long(uint32_t bar, uint32_t at) {
    const uint64_t t0 = global_ns();
    const uint32_t parity = (at / kAttStages) & 1u, verdict = bar + 8 * (kAttStages - at % kAttStages);
    bool here = false;
    while (!here && global_ns() - t0 <= 1000000000ull)
        for (int i = 0; i < 256 && !here; ++i) here = mbar_try_wait(bar, parity);
    const uint32_t mine = 2u * at + (here ? 3u : 2u);
    uint32_t seen = lds_u32(verdict);
    while (seen >> 1 != at + 1u) {
        uint32_t was;
        asm volatile("atom.shared.cas.b32 %0, [%1], %2, %3;" : "=r"(was) : "r"(verdict), "r"(seen), "r"(mine) : "memory");
        seen = was == seen ? mine : was;
    }
    return (seen & 1u) != 0 && (here || mbar_wait(bar, parity));
}
__device__ __forceinline__ bool tile_wait(uint32_t bar, uint32_t at) {
    const uint32_t parity = (at / kAttStages) & 1u;
    for (int i = 0; i < 64; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    return tile_wait_long(bar, at);
}
// What follows where tile `at` did not arrive (never in normal operation): the CTA requests nothing more, and what it has still to deliver
// becomes NaN.  What the warp has requested, up to tile `requested`, gets one more wait each first, as the rings' memory is used
// for other things.
__device__ __noinline__ void tile_lost(uint32_t bars, uint32_t at, uint32_t requested, int *lost) {
    *lost = 1;
    if ((threadIdx.x & 31) == 0) atomicOr(&g_kv_status, 1u);
    for (uint32_t i = at; i < requested; ++i) (void)mbar_wait(bars + 8 * (i % kAttStages), (i / kAttStages) & 1u);
    __syncwarp();
}

template <int D, int NT>
__global__ void __launch_bounds__(kAttThreads, (kAttCtasPerSm<D, NT>)) kv_attention_kernel(KvView c, KvSeqs s, KvQuery a) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb;
    extern __shared__ __align__(128) uint8_t att_smem_raw[];
    __shared__ uint64_t sh_scan[kAttWarps][2];
    __shared__ int sh_item[10];
    __shared__ Owner sh_owner[kAttThreads];
    __shared__ uint32_t sh_next;
    __shared__ float sh_ml[kAttWarps][kAttRows<NT>][2];
    __shared__ int sh_last, sh_lost;       // (sh_lost: a tile never arrived)
    __shared__ __align__(8) uint64_t sh_bars[kAttWarps][kAttStages + 1];      // (the last: see tile_wait_long)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, tig = lane & 3;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(att_smem_raw) + warp * kAttStages * T::kBytes;
    float *const merge = reinterpret_cast<float *>(att_smem_raw);   // [warp][row][D + 4], between items
    constexpr int kMergeRow = D + 4;
    static_assert(T::kBytes * kAttWarps * kAttStages == att_smem(D), "the rings are the shared memory the join's table has");
    static_assert(kAttWarps * kAttRows<NT> * kMergeRow * 4 <= kAttWarps * kAttStages * T::kBytes, "the merge buffer lies over the rings");

    const uint32_t bars = (uint32_t)__cvta_generic_to_shared(sh_bars[warp]);
    uint32_t issued = 0;      // tiles the warp has requested before this segment: ring slots and phases run on
    if (lane == 0) {
        sh_bars[warp][kAttStages] = 0;
        for (int i = 0; i < kAttStages; ++i) mbar_init(bars + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 0) sh_lost = 0;
    pdl_trigger();
    pdl_wait();
    asm volatile("fence.proxy.async;" ::: "memory");      // tiles may have been written by the kernel before, with ordinary stores

    // ---- the items: parts of segments (sequence, kv head, row tile) ----
    auto shape_of = [&](int len, int rows, uint32_t &n, uint32_t &tiles) {      // tiles of a segment, segments per kv head
        n = rows == 0 ? 1u : max(1u, ((uint32_t)len + kTileTokens - 1) / kTileTokens);      // (no rows: nothing to read, nothing to join)
        tiles = max(1u, (uint32_t)(rows * a.group + kAttRows<NT> - 1) / kAttRows<NT>);
    };
    // Two column blocks' accumulators at head dimension 128 leave no register for the sizes: there they stay in shared
    // memory (8 x 8 rows over 16384 tokens: 170 us, in registers 184); elsewhere reading them costs more (tree verification: 37.1 us, in registers 36.6).
    constexpr bool kSizesShared = D == 128 && NT == 2;
    __shared__ AttSizes sh_sizes;
    AttSizes sizes_own = {0, 0};
    const AttSizes &sizes = kSizesShared ? sh_sizes : sizes_own;
    auto cut_of = [&](uint32_t n) { return att_cut(sizes, n, kAttMaxParts<D, NT>); };
    const int each = (s.B + kAttThreads - 1) / kAttThreads, b_first = tid * each, b_last = min(s.B, b_first + each);
    uint32_t bigs, items;                          // all big items, all items
    {
        int len0 = 0, rows0 = 0;                   // the first of this thread's sequences
        uint64_t work = 0;
        for (int i = b_first; i < b_last; ++i) {
            const int len = s.len(i), rows = s.nrows(i);
            if (i == b_first) len0 = len, rows0 = rows;
            uint32_t n, tiles;
            shape_of(len, rows, n, tiles);
            work += (uint64_t)n * (tiles * (uint32_t)c.heads);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) work += __shfl_xor_sync(0xffffffffu, work, o);
        if (lane == 0) sh_scan[warp][0] = work;
        __syncthreads();
        work = 0;
        for (int w = 0; w < kAttWarps; ++w) work += sh_scan[w][0];
        const uint32_t share = (uint32_t)min(work / gridDim.x, (uint64_t)1 << 30);      // of a CTA
        if constexpr (!kSizesShared) sizes_own = att_sizes(share, NT);
        else if (tid == 0) sh_sizes = att_sizes(share, NT);
        __syncthreads();                           // (and sh_scan is free again)
        uint64_t mine[2] = {0, 0};                 // big items and small ones; slots (items of segments that are cut)
        for (int i = b_first; i < b_last; ++i) {
            uint32_t n, tiles;
            shape_of(i == b_first ? len0 : s.len(i), i == b_first ? rows0 : s.nrows(i), n, tiles);
            const AttCut k = cut_of(n);
            const uint32_t segs = tiles * (uint32_t)c.heads;
            mine[0] += (uint64_t)k.bigs * segs | (uint64_t)(k.parts - k.bigs) * segs << 32;
            mine[1] += k.parts > 1 ? (uint64_t)k.parts * segs : 0;
        }
        uint64_t upto[2] = {mine[0], mine[1]}, total = 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint64_t before = __shfl_up_sync(0xffffffffu, upto[e], o);
                if (lane >= o) upto[e] += before;
            }
        if (lane == 31) sh_scan[warp][0] = upto[0], sh_scan[warp][1] = upto[1];
        __syncthreads();
        for (int w = 0; w < kAttWarps; ++w) {
            if (w < warp) upto[0] += sh_scan[w][0], upto[1] += sh_scan[w][1];
            total += sh_scan[w][0];
        }
        bigs = (uint32_t)total, items = bigs + (uint32_t)(total >> 32);
        uint32_t n, tiles;
        shape_of(len0, rows0, n, tiles);
        Owner &o = sh_owner[tid];
        o.cut = cut_of(n), o.tiles = tiles, o.len = len0, o.rows = rows0;
        o.big_lo = (uint32_t)(upto[0] - mine[0]), o.big_count = (uint32_t)mine[0];
        o.small_lo = bigs + (uint32_t)((upto[0] - mine[0]) >> 32), o.small_count = (uint32_t)(mine[0] >> 32);
        o.slot_lo = (uint32_t)(upto[1] - mine[1]);
    }

    // Items are taken in turn as CTAs become free; which CTA computes an item does not matter to its result.  Whether a delivered part
    // was its segment's last is asked one item later, when the answer has arrived.
    Part pending = {};
    pending.parts = 0;
    unsigned before = 0;                           // thread 0: parts of the pending segment delivered before this CTA's
    for (uint32_t item = blockIdx.x;;) {
        const bool have = item < items, drawn = have && items > gridDim.x;
        if (!have && pending.parts == 0) break;
        unsigned taken = 0;
        if (drawn && tid == 0) taken = atomicAdd(MXQ_AT(a.counter, 4, a.counter, 4), 1u);
        const bool is_big = item < bigs;
        const Owner &mine = sh_owner[tid];
        const uint32_t lo = is_big ? mine.big_lo : mine.small_lo;
        if (have && item - lo < (is_big ? mine.big_count : mine.small_count)) {
            uint32_t at = lo, slot = mine.slot_lo, tiles = mine.tiles;
            AttCut k = mine.cut;
            int i = b_first, len = mine.len, rows = mine.rows;
            for (;;) {
                const uint32_t segs = tiles * (uint32_t)c.heads, count = (is_big ? k.bigs : k.parts - k.bigs) * segs;
                if (item - at < count) break;
                at += count, slot += k.parts > 1 ? k.parts * segs : 0, ++i;
                len = s.len(i), rows = s.nrows(i);
                uint32_t n;
                shape_of(len, rows, n, tiles);
                k = cut_of(n);
            }
            // the segment, the item's place among its parts, its tiles
            const uint32_t of = is_big ? k.bigs : k.parts - k.bigs, seg = of == 1 ? item - at : (item - at) / of, p = item - at - seg * of;
            sh_item[0] = i, sh_item[1] = len, sh_item[2] = rows, sh_item[3] = (int)seg, sh_item[4] = (int)tiles, sh_item[5] = (int)k.parts;
            sh_item[6] = (int)(is_big ? p : k.bigs + p), sh_item[7] = (int)(slot + seg * k.parts);
            sh_item[8] = (int)(is_big ? p * k.big : k.bigs * k.big + p * k.small), sh_item[9] = (int)(is_big ? k.big : k.small);
        }
        __syncthreads();
        bool whole = true;
        Part mine_now = {};
        [[maybe_unused]] const size_t ws_bytes = (size_t)a.slots * kAttSlotFloats<D, NT> * 4, o_bytes = (size_t)s.B * s.m * a.heads * D * 2;
        // final results of flattened row r of a sequence
        auto out_row = [&](int b, int head, int r) {
            const int i = token_row(a, r);
            return ((int64_t)b * s.m + i) * a.heads + head * a.group + r - i * a.group;
        };
        auto store_part = [&](int64_t row, int d, const float4 &v) {
            *reinterpret_cast<uint2 *>(MXQ_AT(a.o + row * D + d, 8, a.o, o_bytes)) = make_uint2(pack_bf162(v.x, v.y), pack_bf162(v.z, v.w));
        };
        auto store_lse = [&](int64_t row, float m, float l) {
            // (no weight at all: -inf; scores that are all NaN leave m at -inf too, but their sum is NaN)
            if (a.lse != nullptr) *MXQ_AT(a.lse + row, 4, a.lse, o_bytes / D * 2) = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147181f;
        };
        if (have) {
        const int b = sh_item[0], len = sh_item[1], rows = sh_item[2];
        const uint32_t seg = (uint32_t)sh_item[3], tiles = (uint32_t)sh_item[4], parts = (uint32_t)sh_item[5], part = (uint32_t)sh_item[6];
        const uint32_t slot0 = (uint32_t)sh_item[7], tile0 = (uint32_t)sh_item[8], ntiles = (uint32_t)sh_item[9];      // slot of the segment's first part, if it is cut
        const uint32_t head = tiles == 1 ? seg : seg / tiles, row_tile = tiles == 1 ? 0u : seg - head * tiles;
        Segment sg;
        sg.b = b, sg.head = (int)head, sg.r0 = (int)row_tile * kAttRows<NT>;
        sg.len = len, sg.base = len - rows, sg.rows_total = rows * a.group;
        const int nrows = min(max(sg.rows_total - sg.r0, 0), kAttRows<NT>);

        // ---- the rows' queries: on their way while the first tiles are looked up ----
        uint4 qx[NT][kNb];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = sg.r0 + 8 * nt + g, i = token_row(a, r);
            const uint16_t *src = a.q + ((int64_t)b * s.m + i) * a.q_stride + (int64_t)(sg.head * a.group + r - i * a.group) * D + 8 * tig;
#pragma unroll
            for (int j = 0; j < kNb; ++j) {
                qx[nt][j] = make_uint4(0, 0, 0, 0);
                if (r < sg.rows_total) qx[nt][j] = ld_dep_u4(MXQ_AT(src + 32 * j, 16, a.q, (((int64_t)s.B * s.m - 1) * a.q_stride + (int64_t)a.heads * D) * 2));
            }
        }

        // ---- the warp's tiles: number k is the segment's tile first_tile + k * kAttWarps ----
        const int last_tile = (int)min(((uint32_t)len + kTileTokens - 1) / kTileTokens, tile0 + ntiles), first_tile = (int)tile0 + warp;
        const int count = nrows > 0 && sh_lost == 0 && first_tile < last_tile ? (last_tile - first_tile + kAttWarps - 1) / kAttWarps : 0;
        const uint8_t *source = nullptr;   // lane i: where tile i of the warp's next 32 lies (nullptr: nowhere)
        uint32_t exist = 0, there = 0;     // bit i: that tile exists; the tiles requested so far, the newest lowest
        auto issue = [&](int k) {
            there <<= 1;
            if (k >= count) return;
            const int at = k & 31;
            if (at == 0) {
                const int t = (first_tile + (k + lane) * kAttWarps) * kTileTokens;
                source = nullptr;
                if (k + lane < count) {
                    const int page = s.page(b, t >> c.page_shift);
                    if (kv_page_ok(c, page)) source = kv_tile<D>(c, page, t & ((1 << c.page_shift) - 1), sg.head);
                }
                exist = __ballot_sync(0xffffffffu, source != nullptr);
            }
            there |= (exist >> at) & 1u;
            if (lane == at) {              // the lane that knows a tile requests it; one that is not there completes at once
                const uint32_t slot = (issued + (uint32_t)k) % kAttStages, bar = bars + 8 * slot;
                mbar_expect_tx(bar, source != nullptr ? T::kBytes : 0);
#ifdef MXQ_DEBUG_BOUNDS
                if (first_tile + k * kAttWarps == a.lost_tile && sg.b == 0 && sg.head == 0) return;
#endif
                if (source != nullptr) bulk_load(ring + slot * T::kBytes, MXQ_AT(source, T::kBytes, c.pool, c.pool_bytes), T::kBytes, bar);
            }
        };
#pragma unroll
        for (int k = 0; k < kAttStages; ++k) issue(k);

        // ---- query fragments: elements 32 j + 8 tig .. + 7 of row g, normalised by a power of two ----
        uint4 qf[NT][kNb];
        float factor[NT][2];               // score -> log2 domain, for the lane's two columns
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const uint4(&x)[kNb] = qx[nt];
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < kNb; ++j) top = __vmaxu2(top, chunk_max2(x[j]));
            top = max(top & 0xFFFFu, top >> 16);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // exponent field e of the largest element -> 2^14 (beside an Inf or NaN finite elements are scaled as beside the largest number:
            // they stay finite, and the scores are what the Inf or NaN makes them)
            const int e = min((int)(top >> 7), 254), up = min(268 - e, 254);
            const float mul = __uint_as_float((uint32_t)up << 23);
            const float back = up == 254 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)(254 - up) << 23);
#pragma unroll
            for (int j = 0; j < kNb; ++j) {
                const uint32_t in[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
                uint32_t out[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = pack_half2(__uint_as_float(in[i] << 16) * mul, __uint_as_float(in[i] & 0xFFFF0000u) * mul);
                qf[nt][j] = make_uint4(out[0], out[1], out[2], out[3]);
            }
#pragma unroll
            for (int e2 = 0; e2 < 2; ++e2) {
                factor[nt][e2] = a.scale_log2 * __shfl_sync(0xffffffffu, back, (2 * tig + e2) * 4);
            }
        }

        WarpState<D, NT> w;
        w.ref = w.ref_max = 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) w.m[nt][e] = 0.f, w.over[nt][e] = -INFINITY, w.l[nt][e] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) w.o[i][nt][e] = 0.f;
        }

        int k = 0;
        for (; k < count; ++k) {
            const uint32_t at = issued + (uint32_t)k, slot = at % kAttStages, tile = ring + slot * T::kBytes;
            const int t0 = (first_tile + k * kAttWarps) * kTileTokens;
            if (!tile_wait(bars + 8 * slot, at)) break;
            if ((there >> (kAttStages - 1)) & 1u) {
                const int tok = (g >> 1) + 4 * (g & 1);      // row g of the product is this token of the group, row g + 8 the one 8 further
                // ---- scores ----
                float x[2][NT][4];       // of the tile's two groups of 16 tokens
                {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        uint32_t k0[kNb], k1[kNb], s0, s1;
                        lds_words<kNb>(tile + (16 * u + tok) * T::kRow + 4 * kNb * tig, k0);
                        lds_words<kNb>(tile + (16 * u + tok + 8) * T::kRow + 4 * kNb * tig, k1);
                        const uint32_t sa = tile + T::kKs + (16 * u + tok) * kNb;
                        if constexpr (kNb == 4) {
                            s0 = lds_u32(sa), s1 = lds_u32(sa + 8 * kNb);
                        } else {
                            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(s0) : "r"(sa));
                            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(s1) : "r"(sa + 8 * kNb));
                        }
#pragma unroll
                        for (int j = 0; j < kNb; ++j) {
                            uint32_t h0[4], h1[4];
                            decode4(k0[j], h0);
                            decode4(k1[j], h1);
                            const float c0 = scale_factor(s0, j), c1 = scale_factor(s1, j);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const uint4 &q = qf[nt][j];
                                float d[4] = {0.f, 0.f, 0.f, 0.f};
                                mma16816<false>(d, h0[0], h1[0], h0[1], h1[1], q.x, q.y);
                                mma16816<false>(d, h0[2], h1[2], h0[3], h1[3], q.z, q.w);
                                float(&v)[4] = x[u][nt];
                                if (j == 0) v[0] = d[0] * c0, v[1] = d[1] * c0, v[2] = d[2] * c1, v[3] = d[3] * c1;
                                else v[0] += d[0] * c0, v[1] += d[1] * c0, v[2] += d[2] * c1, v[3] += d[3] * c1;
                            }
                        }
                    }
                }
                // ---- relative to the running maximum; what a row does not see; a new maximum ----
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint64_t f = pair2(factor[nt][0], factor[nt][1]), m = pair2(kWeightBias - w.m[nt][0], kWeightBias - w.m[nt][1]);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float(&v)[4] = x[u][nt];
                            split2(fma2(pair2(v[2 * h], v[2 * h + 1]), f, m), v[2 * h], v[2 * h + 1]);
                        }
                }
                if (t0 + kTileTokens > sg.base) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const Sight sight = sight_of(s, a, sg, sg.r0 + 8 * nt + 2 * tig + e);
#pragma unroll
                            for (int u = 0; u < 2; ++u)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    if (!sight.sees(t0 + 16 * u + tok + 8 * h)) x[u][nt][2 * h + e] = -INFINITY;
                        }
                }
                bool over = false;
                float top[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float v = fmaxf(x[0][nt][e], x[0][nt][2 + e]);
                        v = fmaxf(v, fmaxf(x[1][nt][e], x[1][nt][2 + e]));
                        top[nt][e] = v;
                        over |= v > w.over[nt][e];
                    }
                if (__any_sync(0xffffffffu, over)) {
                    float f[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float v = top[nt][e];
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
                            const bool none = w.over[nt][e] == -INFINITY;      // no token seen before: m is 0 for want of a better
                            float up = none ? v - kWeightBias : fmaxf(v - kWeightBias, 0.f);      // how far the maximum rises
                            f[nt][e] = none ? 1.f : exp2_fast(-up);
                            if (v == -INFINITY) up = 0.f;
                            else w.over[nt][e] = kWeightBias + kMaxSlack;
                            w.m[nt][e] += up;
                            w.l[nt][e] *= f[nt][e];
#pragma unroll
                            for (int u = 0; u < 2; ++u) x[u][nt][e] -= up, x[u][nt][2 + e] -= up;
                        }
                    rescale(w, f);
                }
                // ---- weights ----
                uint32_t pk[2][NT][2], least = 0x7C007C00u;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint64_t sum = pair2(w.l[nt][0], w.l[nt][1]);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float &p0 = x[u][nt][2 * h], &p1 = x[u][nt][2 * h + 1];
                            p0 = exp2_fast(p0), p1 = exp2_fast(p1);
                            sum = add2(sum, pair2(p0, p1));
                            pk[u][nt][h] = pack_half2(p0, p1);
                            least = min_half2(least, pk[u][nt][h]);
                        }
                    split2(sum, w.l[nt][0], w.l[nt][1]);
                }
                // ---- V scales: largest and smallest ----
                const bool tail = t0 + kTileTokens > len;
                const uint32_t sv_at = tile + T::kVs + 4 * lane;
                uint32_t sv = 0, in = 0xFFFFFFFFu;           // a word of them per lane, and the bytes of tokens that are there
                if (8 * kNb == 32 || lane < 8 * kNb) sv = lds_u32(sv_at);
                else in = 0;
                uint32_t up_ = sv, dn_ = 8 * kNb == 32 ? sv : sv | ~in;
                if (tail) {
                    const int t = t0 + 16 * (4 * lane / (16 * kNb)) + (4 * lane / (4 * kNb)) % 4 + 8 * ((4 * lane / (2 * kNb)) % 2);
                    in &= (t < len ? 0x00FF00FFu : 0u) | (t + 4 < len ? 0xFF00FF00u : 0u);
                    up_ = sv & in, dn_ = sv | ~in;
                }
                uint32_t hi2 = __vmaxu2(__byte_perm(up_, 0, 0x4240), __byte_perm(up_, 0, 0x4341));
                uint32_t lo2 = __vminu2(__byte_perm(dn_, 0, 0x4240), __byte_perm(dn_, 0, 0x4341));
                hi2 = __vmaxu2(hi2, __byte_perm(hi2, 0, 0x1032)), lo2 = __vminu2(lo2, __byte_perm(lo2, 0, 0x1032));
                int hi = (int)(__reduce_max_sync(0xffffffffu, hi2) & 0xFFFFu);
                const int lo = (int)(__reduce_min_sync(0xffffffffu, lo2) & 0xFFFFu);
                bool nan = false;
                if (hi > w.ref + kScaleHeadroom || hi + kScaleLag < w.ref || tail) {
                    nan = hi == 255;
                    if (nan) {       // the largest that is a number
                        hi = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int v = (int)(((sv & in) >> (8 * i)) & 0xFFu);
                            if (v != 255) hi = max(hi, v);
                        }
                        hi = (int)__reduce_max_sync(0xffffffffu, (uint32_t)hi);
                    }
                    // ref follows the tiles' largest scale up and (within what FP32 accumulators bear) down
                    if (hi > w.ref + kScaleHeadroom || hi + kScaleLag < w.ref) {
                        w.ref_max = max(w.ref_max, hi);
                        const int ref = max(hi, w.ref_max - kScaleDrop);
                        const float f = scale_by_power(1.f, w.ref - ref);
                        float ff[NT][2];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) ff[nt][0] = ff[nt][1] = f;
                        rescale(w, ff);
                        w.ref = ref;
                    }
                    if (tail) {      // tokens that are not there carry no weight: any scale that fits will do
                        if (lane < 8 * kNb) asm volatile("st.shared.u32 [%0], %1;" ::"r"(sv_at), "r"((sv & in) | ((uint32_t)w.ref * 0x01010101u & ~in)) : "memory");
                        __syncwarp();
                    }
                }
                // ---- O += P V: which form holds these weights? ----
                const int range = kHalfRange - max(w.ref - lo, 0);      // binades of weight the scales leave to FP16
                const float small = __uint_as_float((uint32_t)(127 - max(range, 0)) << 23);
                const bool plain = __all_sync(0xffffffffu, all_le_half2(pack_half2(small, small), least)) && range >= kHalfRange - kScaleSpread && !nan;   // (NaN compares false)
                float low = 1.f;             // the smallest weight that is not zero
                // tiers below `small`: each as wide as what FP16 holds, 2^width
                const int width = range + kWeightBias;
                const float step = __uint_as_float((uint32_t)(127 - max(width, 0)) << 23), tiny = small * step;
                if (!plain) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) low = fminf(low, x[u][nt][e] == 0.f ? 1.f : x[u][nt][e]);
                }
                if (plain) {
                    uint32_t p[2][NT][2];
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int h = 0; h < 2; ++h) p[u][nt][h] = transpose8x8(pk[u][nt][h]);
                    add_values<D, NT, 1>(w, tile, g, tig, p, p, 1.f, 1.f);
                } else if (!nan && range >= kHalfRange - kScaleSpread && !__any_sync(0xffffffffu, low < tiny * step * step)) {
                    // tiers 3 and 2 if there are such weights, then 1 and 0: tier i > 0 holds weights in small * step^i .. small * step^(i - 1)
                    const float up = __uint_as_float((uint32_t)(127 + width) << 23);
                    const bool four = __any_sync(0xffffffffu, low < tiny);
#pragma unroll 1
                    for (int pass = four ? 0 : 1; pass < 2; ++pass) {
                        const float gain = pass == 0 ? up * up : 1.f, bound = pass == 0 ? tiny : INFINITY, part_ = pass == 0 ? tiny * step : small;
                        const float from = pass == 1 && four ? tiny : 0.f;
                        if (four) {
                            float ff[NT][2];
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) ff[nt][0] = ff[nt][1] = pass == 0 ? up * up : step * step;
                            rescale(w, ff);
                        }
                        uint32_t p[2][NT][2], deep[2][NT][2];
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    float lo_[2], hi_[2];
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        const float v = x[u][nt][2 * h + e], in_ = v < from || v >= bound ? 0.f : v * gain;
                                        lo_[e] = v < part_ ? in_ * up : 0.f;
                                        hi_[e] = v < part_ ? 0.f : in_;
                                    }
                                    p[u][nt][h] = transpose8x8(pack_half2(hi_[0], hi_[1]));
                                    deep[u][nt][h] = transpose8x8(pack_half2(lo_[0], lo_[1]));
                                }
                        add_values<D, NT, 2>(w, tile, g, tig, p, deep, up, step);
                    }
                } else {
                    constexpr float kUnbias = 1.f / (1 << kWeightBias);          // (the factor goes to the scales, which may lie 126 and more below ref)
#pragma unroll 1
                    for (int part_ = 0; part_ < 2; ++part_)       // the weights' upper and lower eight bits
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            uint32_t p[NT][2];
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const float x0 = x[u][nt][2 * h] * kUnbias, x1 = x[u][nt][2 * h + 1] * kUnbias;
                                    uint32_t b = pack_bf162(x0, x1);
                                    if (part_ == 1) b = pack_bf162(x0 - __uint_as_float(b << 16), x1 - __uint_as_float(b & 0xFFFF0000u));
                                    p[nt][h] = transpose8x8(b);
                                }
                            add_values_wide<D, NT>(w, tile, u, t0 + 16 * u, g, tig, p, [&](int nt, int t) { return sight_of(s, a, sg, sg.r0 + 8 * nt + g).sees(t); });
                        }
                }
            }
            __syncwarp();
            issue(k + kAttStages);
        }

        // ---- join the warps: each as (maximum, sum, average), eight rows at a time over the drained rings ----
        __syncwarp();
        if (k < count) tile_lost(bars, issued + (uint32_t)k, issued + (uint32_t)min(count, k + kAttStages), &sh_lost);
        issued += (uint32_t)count;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (sh_lost != 0) w.l[nt][e] = NAN;
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) w.l[nt][e] += __shfl_xor_sync(0xffffffffu, w.l[nt][e], o);
                if (g == 0) sh_ml[warp][8 * nt + 2 * tig + e][0] = w.over[nt][e] == -INFINITY ? -INFINITY : w.m[nt][e] - kWeightBias, sh_ml[warp][8 * nt + 2 * tig + e][1] = w.l[nt][e];
            }
        whole = parts == 1;
        mine_now = {b, sg.head, sg.r0, nrows, parts, slot0};
        float *const slot = a.partials + (size_t)(slot0 + part) * kAttSlotFloats<D, NT>;
        {
            __syncthreads();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (8 * nt + 2 * tig + e >= nrows) break;
                    const float inv = w.l[nt][e] == 0.f ? 0.f : 1.f / w.l[nt][e];
                    float *dst = merge + (warp * kAttRows<NT> + 8 * nt + 2 * tig + e) * kMergeRow + 4 * g;
#pragma unroll
                    for (int j = 0; j < kNb; ++j) {
                        float v[4] = {w.o[2 * j][nt][e], w.o[2 * j][nt][2 + e], w.o[2 * j + 1][nt][e], w.o[2 * j + 1][nt][2 + e]};
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = scale_by_power(v[i] * inv, w.ref - 127);
                        *reinterpret_cast<float4 *>(dst + 32 * j) = make_float4(v[0], v[1], v[2], v[3]);
                    }
                }
            __syncthreads();
            for (int r = warp; r < nrows; r += kAttWarps) {      // a warp per row
                float m = -INFINITY, l = 0.f;
#pragma unroll
                for (int i = 0; i < kAttWarps; ++i) m = fmaxf(m, sh_ml[i][r][0]);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int i = 0; i < kAttWarps; ++i) {
                    const float li = sh_ml[i][r][1], f = li == 0.f ? 0.f : li * exp2_fast(sh_ml[i][r][0] - m);
                    l += f;
                    if (4 * lane < D && li != 0.f) {
                        const float4 x = *reinterpret_cast<const float4 *>(merge + (i * kAttRows<NT> + r) * kMergeRow + 4 * lane);
                        v.x += f * x.x, v.y += f * x.y, v.z += f * x.z, v.w += f * x.w;
                    }
                }
                const float inv = l == 0.f ? 0.f : 1.f / l;
                v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
                if (whole) {
                    const int64_t row = out_row(b, sg.head, sg.r0 + r);
                    if (4 * lane < D) store_part(row, 4 * lane, v);
                    if (lane == 0) store_lse(row, m, l);
                } else {
                    if (4 * lane < D) *reinterpret_cast<float4 *>(MXQ_AT(slot + r * D + 4 * lane, 16, a.partials, ws_bytes)) = v;
                    if (lane == 0) *reinterpret_cast<float2 *>(MXQ_AT(slot + kAttRows<NT> * D + 2 * r, 8, a.partials, ws_bytes)) = make_float2(m, l);
                }
            }
        }

        // rows the sequence does not have
        if (part == 0 && sg.r0 == 0)
            for (int r = sg.rows_total + warp; r < s.m * a.group; r += kAttWarps) {
                const int64_t row = out_row(b, sg.head, r);
                if (4 * lane < D) store_part(row, 4 * lane, make_float4(0.f, 0.f, 0.f, 0.f));
                if (lane == 0) store_lse(row, -INFINITY, 0.f);
            }
        }   // (have)

        // ---- join the parts of the segment delivered to before: the CTA that brought the last one adds them, in order ----
        auto ticket_of = [&](const Part &p) { return MXQ_AT(a.tickets + p.slot0, 4, a.tickets, (size_t)a.slots * 4); };
        if (pending.parts != 0 || !whole) {
            if (tid == 0) {
                sh_last = pending.parts != 0 && before == pending.parts - 1;
                if (sh_last) {
                    __threadfence();
                    *ticket_of(pending) = 0;
                }
            }
            __syncthreads();          // (and every thread's part of this item's result is stored before the ticket below)
            if (sh_last) {
                const int nrows = pending.nrows;
                const uint32_t parts = pending.parts, slot0 = pending.slot0;
                const float *const p0 = a.partials + (size_t)slot0 * kAttSlotFloats<D, NT>;
                float2 *const table = reinterpret_cast<float2 *>(att_smem_raw);       // [part][row]: maximum and sum, then the part's share (its bounds are in mxq_kv_division.h)
                float4 *const sums = reinterpret_cast<float4 *>(att_smem_raw + ((size_t)parts * nrows * 8 + 15) / 16 * 16);
                const int pairs = (int)parts * nrows;
                for (int x = tid; x < pairs; x += kAttThreads) {
                    const int i = x / nrows, r = x - i * nrows;
                    *MXQ_AT(table + x, 8, att_smem_raw, (kAttSmem<D, NT>)) = __ldcg(reinterpret_cast<const float2 *>(MXQ_AT(p0 + i * (kAttSlotFloats<D, NT>) + kAttRows<NT> * D + 2 * r, 8, a.partials, ws_bytes)));
                }
                __syncthreads();
                float m = -INFINITY, l = 0.f;       // of row `lane`
                if (lane < nrows) {
                    for (int i = warp; i < (int)parts; i += kAttWarps) m = fmaxf(m, table[i * nrows + lane].x);
                    for (int i = warp; i < (int)parts; i += kAttWarps) {
                        const float2 ml = table[i * nrows + lane];
                        l += ml.y == 0.f ? 0.f : ml.y * exp2_fast(ml.x - m);
                    }
                    sh_ml[warp][lane][0] = m, sh_ml[warp][lane][1] = l;
                }
                __syncthreads();
                m = -INFINITY, l = 0.f;
                if (lane < nrows) {
#pragma unroll
                    for (int i = 0; i < kAttWarps; ++i) m = fmaxf(m, sh_ml[i][lane][0]);
#pragma unroll
                    for (int i = 0; i < kAttWarps; ++i) l += sh_ml[i][lane][1] == 0.f ? 0.f : sh_ml[i][lane][1] * exp2_fast(sh_ml[i][lane][0] - m);
                    if (sh_lost != 0) l = NAN;        // (a copy that comes late may have changed the table)
                    if (warp == 0) store_lse(out_row(pending.b, pending.head, pending.r0 + lane), m, l);
                }
                const float inv = l == 0.f ? 0.f : 1.f / l;
                for (int x0 = 32 * warp; x0 < pairs; x0 += kAttThreads) {
                    const int x = x0 + lane, r = x % nrows;
                    const float rm = __shfl_sync(0xffffffffu, m, r), ri = __shfl_sync(0xffffffffu, inv, r);
                    if (x < pairs) table[x].x = table[x].y == 0.f ? 0.f * ri : table[x].y * exp2_fast(table[x].x - rm) * ri;
                }
                __syncthreads();
                // four elements of a row per thread; with few rows several threads share the parts
                constexpr int kCols = D / 4, kAhead = 8;       // loads in flight per thread (one request of 100000 tokens: 64 us, a loop unrolled by four 72)
                const int tasks = nrows * kCols, shares = tasks < kAttThreads ? kAttThreads / tasks : 1;
                auto add_parts = [&](int task, int from, int stride) {
                    const int r = task / kCols, d = 4 * (task % kCols);
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int i0 = from; i0 < (int)parts; i0 += kAhead * stride) {
                        float4 x[kAhead];
#pragma unroll
                        for (int u = 0; u < kAhead; ++u) {
                            const int i = i0 + u * stride;
                            x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (i < (int)parts) x[u] = __ldcg(reinterpret_cast<const float4 *>(MXQ_AT(p0 + i * (kAttSlotFloats<D, NT>) + r * D + d, 16, a.partials, ws_bytes)));
                        }
#pragma unroll
                        for (int u = 0; u < kAhead; ++u) {
                            const int i = i0 + u * stride;
                            const float f = i < (int)parts ? table[i * nrows + r].x : 0.f;
                            v.x += f * x[u].x, v.y += f * x[u].y, v.z += f * x[u].z, v.w += f * x[u].w;
                        }
                    }
                    return v;
                };
                if (shares == 1) {
                    for (int task = tid; task < tasks; task += kAttThreads)
                        store_part(out_row(pending.b, pending.head, pending.r0 + task / kCols), 4 * (task % kCols), add_parts(task, 0, 1));
                } else {
                    const int task = tid % tasks, share = tid / tasks;
                    if (share < shares) *MXQ_AT(sums + tid, 16, att_smem_raw, (kAttSmem<D, NT>)) = add_parts(task, share, shares);
                    __syncthreads();
                    if (share == 0) {
                        float4 v = sums[task];
                        for (int i = 1; i < shares; ++i) {
                            const float4 x = sums[i * tasks + task];
                            v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
                        }
                        store_part(out_row(pending.b, pending.head, pending.r0 + task / kCols), 4 * (task % kCols), v);
                    }
                }
            }
        }
        pending.parts = 0;
        if (!whole) {
            pending = mine_now;
            if (tid == 0) {
                __threadfence();
                before = atomicAdd(ticket_of(pending), 1u);
            }
        }
        if (tid == 0) {
            sh_next = drawn ? gridDim.x + taken : items;
            if (drawn && taken == items - 1) *a.counter = 0;       // one draw per item: this was the last
        }
        fence_async_proxy();  // (the rings held ordinary stores; bulk copies come next)
        __syncthreads();      // the rings and sh_ml are free again
        item = sh_next;
    }
}

MXQ_BOUNDS_TU(bounds_take_kv_attention)

// returns and clears this kernel's sticky status word (see mxq_linear_device_status)
int kv_take_status(uint32_t *out) {
    unsigned int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_kv_status, sizeof v) != cudaSuccess) return MXQ_ERR_CUDA;
    if (v != 0 && cudaMemcpyToSymbol(g_kv_status, &zero, sizeof zero) != cudaSuccess) return MXQ_ERR_CUDA;
    *out = v;
    return MXQ_OK;
}

// ---- host -------------------------------------------------------------------------------------------------------------------

// Column blocks per row tile: two from nine rows on.  (Four would decode K and V half as often, but their accumulators leave only
// two warps per scheduler: 8 x 8 rows over 4-fold grouped heads, 16384 tokens: 251 us with up to four blocks, 180 with two, 206 with one.)
static int att_column_blocks(int M, int group) { return (int64_t)M * group <= 8 ? 1 : 2; }

template <int D, int NT>
static int att_grid() { return sm_count() * kAttCtasPerSm<D, NT>; }

// Workspace: the counter, a ticket per cut segment (under its first part's slot), slots for the parts.  Counter and tickets lie in the
// same place for every shape, so that calls of different shapes may share a workspace: they find them zero.
constexpr int kAttMostCtasPerSm = 4;
static size_t att_partials_offset() { return 16 + (((size_t)kAttSlotsPerCta * kAttMostCtasPerSm * sm_count() * 4 + 255) / 256 * 256); }
template <int D, int NT>
static size_t att_workspace() {
    static_assert(kAttCtasPerSm<D, NT> <= kAttMostCtasPerSm, "");
    return att_partials_offset() + (size_t)kAttSlotsPerCta * att_grid<D, NT>() * kAttSlotFloats<D, NT> * 4;
}

// test hook (mxq_debug_kv_lost_tile): consumed by the next launch
[[maybe_unused]] static std::atomic<int> g_lost_tile{-1};

template <int D, int NT>
static int att_launch(const KvView &c, const KvSeqs &s, KvQuery a, void *workspace, cudaStream_t stream) {
    constexpr size_t smem = kAttSmem<D, NT>;
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return MXQ_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kv_attention_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
            cudaFuncSetAttribute(kv_attention_kernel<D, NT>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) {
            (void)cudaGetLastError();
            return MXQ_ERR_CUDA;
        }
        configured[dev] = true;
    }
    a.counter = (unsigned *)workspace;
    a.tickets = (unsigned *)((char *)workspace + 16);
    a.partials = (float *)((char *)workspace + att_partials_offset());
    a.slots = kAttSlotsPerCta * (uint32_t)att_grid<D, NT>();
#ifdef MXQ_DEBUG_BOUNDS
    a.lost_tile = g_lost_tile.exchange(-1, std::memory_order_relaxed);
#endif
    return kv_launch(kv_attention_kernel<D, NT>, dim3((unsigned)att_grid<D, NT>()), kAttThreads, smem, stream, c, s, a);
}

// the template instance that covers a call: f(head dimension, column blocks) with both as constants
template <class F>
static auto att_pick(int head_dim, int M, int group, F f) {
    using std::integral_constant;
    const bool one = att_column_blocks(M, group) == 1;
    if (head_dim == 128)
        return one ? f(integral_constant<int, 128>(), integral_constant<int, 1>()) : f(integral_constant<int, 128>(), integral_constant<int, 2>());
    return one ? f(integral_constant<int, 64>(), integral_constant<int, 1>()) : f(integral_constant<int, 64>(), integral_constant<int, 2>());
}

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

size_t mxq_kv_attention_workspace_bytes(int B, int M, int q_heads, int kv_heads, int head_dim) {
    if (B < 1 || B > MXQ_KV_MAX_SEQS || M < 1 || kv_heads < 1 || kv_heads > MXQ_KV_MAX_HEADS || q_heads < kv_heads || q_heads % kv_heads ||
        mxq_kv_page_bytes(kv_heads, head_dim, 32) == 0)
        return 0;
    const int group = q_heads / kv_heads;
    if ((int64_t)M * group > 65536 || (int64_t)B * M * q_heads > (1 << 30)) return 0;
    return mxq::att_pick(head_dim, M, group, [](auto d, auto nt) { return mxq::att_workspace<d(), nt()>(); });
}

int mxq_kv_attention(const mxq_kv_cache *cache, int layer, const void *Q_bf16, int64_t q_stride, int B, int M, int q_heads,
                     const int32_t *tables, int W, const int32_t *lens, const int32_t *rows, const uint64_t *tree, float scale,
                     void *O_bf16, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    if (!Q_bf16 || !O_bf16) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, layer);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    const size_t need = mxq_kv_attention_workspace_bytes(B, M, q_heads, cache->kv_heads, cache->head_dim);
    if (need == 0 || q_stride < (int64_t)q_heads * cache->head_dim || (tree && M > MXQ_MAX_T)) return MXQ_ERR_SHAPE;
    if (!mxq::aligned16(Q_bf16) || !mxq::aligned16(O_bf16) || q_stride % 8 || !mxq::aligned_to(lse, 4) || !mxq::aligned_to(tree, 8) ||
        !mxq::aligned_to(rows, 4) || !mxq::aligned16(workspace))
        return MXQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < need) return MXQ_ERR_WORKSPACE;
    const int group = q_heads / cache->kv_heads;
    mxq::KvQuery a = {};
    a.q = (const uint16_t *)Q_bf16, a.q_stride = q_stride, a.tree = tree, a.o = (uint16_t *)O_bf16, a.lse = lse;
    a.heads = q_heads, a.group = group, a.scale_log2 = scale * 1.44269504f;
    a.group_magic = group == 1 ? 0u : (uint32_t)((1ull << 32) / (unsigned)group + 1);
    const mxq::KvSeqs s = mxq::kv_seqs(cache, B, M, tables, W, lens, rows);
    const mxq::KvView c = mxq::kv_view(cache, layer);
    return mxq::att_pick(cache->head_dim, M, group,
                         [&](auto d, auto nt) { return mxq::att_launch<d(), nt()>(c, s, a, workspace, (cudaStream_t)stream); });
}

int mxq_debug_kv_lost_tile(int tile) {
#ifdef MXQ_DEBUG_BOUNDS
    mxq::g_lost_tile.store(tile, std::memory_order_relaxed);
    return MXQ_OK;
#else
    (void)tile;
    return MXQ_ERR_SHAPE;
#endif
}

#pragma GCC visibility pop
}  // extern "C"
