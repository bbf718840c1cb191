// Layout of the 4-bit key/value cache (see mxq_kv_cache in mxq.h) and what its kernels share.
//
// A tile holds 32 tokens of one head: K codes [32][D/2], V codes [32][D/2], K scales [32][nb], V scales [32 * nb], with
// nb = D / 32 MX blocks per row.  Within a row the bytes are permuted so that the attention kernel's fragments of the
// m16n8k16 product are single wide loads from consecutive addresses:
//   K: the product contracts over d, eight codes of one block per lane and word.  Chunk c (of 4) of a row holds word c of
//      every block: byte c*4*nb + 4*j + i = natural byte 16*j + 4*c + i.
//   V: the product contracts over tokens, its rows are d.  Chunk g (of 8) holds two bytes of every block:
//      byte g*2*nb + 2*j + i = natural byte 16*j + 2*g + i.
//   V scales: lane tig of a quad weighs tokens tig, tig + 4 (one register) and tig + 8, tig + 12 of a group of 16; the two
//      tokens of a register lie side by side, so that a lane's scales are one load:
//      token 16*u + tig + 4*e + 8*h, block j at 16*nb*u + 4*nb*tig + 2*nb*h + 2*j + e.
#pragma once
#include "mxq_device.cuh"
#include "mxq_host.h"

namespace mxq {

constexpr int kTileTokens = 32;

template <int D>
struct KvTile {
    static constexpr int kNb = D / 32;                       // MX blocks per row
    static constexpr int kRow = D / 2;                       // code bytes per row
    static constexpr int kV = kTileTokens * kRow;            // offsets in a tile: K codes at 0, V codes,
    static constexpr int kKs = 2 * kTileTokens * kRow;       // K scales,
    static constexpr int kVs = kKs + kTileTokens * kNb;      // V scales
    static constexpr int kBytes = kVs + kTileTokens * kNb;
    __host__ __device__ static constexpr int vs(int t, int j) {   // offset of the V scale of (token, block)
        return kVs + 16 * kNb * (t >> 4) + 4 * kNb * (t & 3) + 2 * kNb * ((t >> 3) & 1) + 2 * j + ((t >> 2) & 1);
    }
};

// the cache as a kernel sees it: one layer's base, and what is needed to find a token's tile
struct KvView {
    uint8_t *base;           // first page of the layer
    int64_t page_bytes;
    const uint8_t *pool;     // the whole pool and its size (bounds-checked build)
    int64_t pool_bytes;
    int32_t num_pages;
    int32_t heads;
    int32_t page_shift;      // log2 of the tokens per page
};

// Sequences of a call: tables [B][W], lens [B], rows [B] or nullptr (then m rows in every sequence).
struct KvSeqs {
    const int32_t *tables;
    const int32_t *lens;
    const int32_t *rows;
    int32_t B, W, m, page_tokens;
    __device__ __forceinline__ int len(int b) const {   // never more than the table can hold
        const int n = (int)ld_dep_u32(MXQ_AT(lens + b, 4, lens, (size_t)B * 4));
        return (int)min((int64_t)max(n, 0), (int64_t)W * page_tokens);
    }
    __device__ __forceinline__ int nrows(int b) const {
        if (rows == nullptr) return m;
        return min(max((int)ld_dep_u32(MXQ_AT(rows + b, 4, rows, (size_t)B * 4)), 0), m);
    }
    __device__ __forceinline__ int page(int b, int w) const {
        return (int)ld_dep_u32(MXQ_AT(tables + (int64_t)b * W + w, 4, tables, (size_t)B * W * 4));
    }
};

// tile of (page, slot, head); the caller has checked the page against num_pages
template <int D>
__device__ __forceinline__ uint8_t *kv_tile(const KvView &c, int page, int slot, int head) {
    return c.base + (int64_t)page * c.page_bytes + (int64_t)((slot >> 5) * c.heads + head) * KvTile<D>::kBytes;
}
__device__ __forceinline__ bool kv_page_ok(const KvView &c, int page) { return (unsigned)page < (unsigned)c.num_pages; }

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

// stores lane q's quarter of a row, q = 0..3: its words w[j] of every block (natural bytes 16j + 4q ..), and its share of the scale bytes
// (`scale`: block j's in byte j)
template <int D>
__device__ __forceinline__ void store_quarter(const KvView &c, const RowPlace &at, bool value, uint32_t q, const uint32_t (&w)[D / 32], uint32_t scale) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb;
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
    uint8_t *dst = MXQ_AT(at.tile + (value ? T::kV : 0) + at.slot * T::kRow + q * 4 * kNb, 4 * kNb, c.pool, c.pool_bytes);
    if constexpr (kNb == 4) *reinterpret_cast<uint4 *>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
    else *reinterpret_cast<uint2 *>(dst) = make_uint2(out[0], out[1]);
    if (!value) {
        if (q == 0) {
            uint8_t *sc = MXQ_AT(at.tile + T::kKs + at.slot * kNb, kNb, c.pool, c.pool_bytes);
            if constexpr (kNb == 4) *reinterpret_cast<uint32_t *>(sc) = scale;
            else *reinterpret_cast<uint16_t *>(sc) = (uint16_t)scale;
        }
    } else if (q < kNb) {
        *MXQ_AT(at.tile + T::vs(at.slot, (int)q), 1, c.pool, c.pool_bytes) = (uint8_t)(scale >> (8 * q));
    }
}

// ---- host side --------------------------------------------------------------------------------------------------------
int kv_check_cache(const mxq_kv_cache *cache, int layer);   // MXQ_OK or the error
int kv_check_seqs(int B, int W, const int32_t *tables, const int32_t *lens);
KvView kv_view(const mxq_kv_cache *cache, int layer);
bool kv_rows_ok(int heads, int B, int M);   // a call of B x M rows of `heads` heads fits 32-bit lane indices
inline KvSeqs kv_seqs(const mxq_kv_cache *cache, int B, int M, const int32_t *tables, int W, const int32_t *lens, const int32_t *rows) {
    KvSeqs s;
    s.tables = tables, s.lens = lens, s.rows = rows, s.B = B, s.W = W, s.m = M, s.page_tokens = cache->page_tokens;
    return s;
}
inline bool aligned_to(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace mxq
