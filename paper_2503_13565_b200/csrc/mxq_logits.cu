// The rules that a server applies to logits before it takes their argmax or samples from them: mxq_logits_adjust writes the adjusted
// logits, mxq_greedy_accept_rules verifies speculated tokens against their argmax without writing them, mxq_token_counts keeps the
// counts of generated and prompted tokens that the penalties go by.
//
// For one logit x of token v, in FP32, every operation rounded once:
//     x = x > 0 ? x / repetition : x * repetition     if v was prompted or generated
//     x = x - frequency * count - presence            if v was generated (count times)
//     x = x + bias                                    if v has an entry in the list of biases (the last one counts)
//     x = -inf                                        if the grammar's mask does not allow v
// Row i of a verification counts the proposals before it, draft[0..i), as generated.
//
// A stream over the logits (and the mask's bits).  The rules but the mask touch few tokens: a CTA takes some batches of tokens of all rows
// of a sequence, reads their counts into shared memory once, and keeps one bit per token that is special (counted, biased or proposed) and a
// list of those tokens.  The stream only leaves the special tokens out, a vector of 16 bytes at a time; then the list is gone through,
// a (row, token) pair per thread.  (With the rules inside the stream, a lane's special tokens one after the other, accept over 24 x 8 rows of
// 128256 took 107 us unrolled, the code leaving the instruction cache, and 37 in a loop, the batches of the frequent tokens last.)
// Measured in a replayed graph: accept over 24 sequences x 8 rows x 128256 BF16 logits with histories, 200 biases and masks 30 us (65 MB: 10 us at
// the copy rate), 12 us without rules, which is what mxq_greedy_accept takes; masks add 5 us, biases 3, penalties 9.  Neither memory (1.9 TB/s) nor
// the issue slots (45 %) are full: tables, stream, list and the special tokens come one after the other in a CTA, with barriers between.
// One sequence of 9 x 32000: 6.1 us, a chain of five dependent trips to memory; adjust over 48 x 32001 FP32 logits: 9.2 us (18 MB), the same
// order of steps for one row.
#include <limits.h>

#include <type_traits>

#include "mxq_device.cuh"
#include "mxq_host.h"

namespace mxq {

constexpr int kLogitThreads = 256;
constexpr int kLogitWarps = kLogitThreads / 32;
constexpr int kLogitCtas = 3;            // per SM
constexpr int kBatchLoads = 2;           // 16-byte loads of a batch per lane (those of the next batch are on their way meanwhile)
constexpr int kBatch = 32 * kBatchLoads; // vectors of a warp's batch
constexpr int kPairs = 4;                // (row, special token) pairs of a thread at once

struct LogitCall {
    const void *logits;
    void *out;                 // adjusted logits, or nullptr (accept)
    const int32_t *draft;      // [B][T]
    const uint32_t *counts;    // [B][V] or nullptr
    const float *penalties;    // [B][3] or nullptr
    const int32_t *bias_tokens;
    const float *bias_values;  // [B][J]
    const uint32_t *allowed;   // [B][R][words] or nullptr
    unsigned long long *keys;  // accept: [B][R] running maxima as (ordered value, ~token), 0 = nothing yet
    unsigned *tickets;         // accept: [B] CTAs that have delivered
    int32_t *verifier, *accept_len, *next_token;
    int64_t B, V, words;
    int32_t R, T, J;
    int32_t slices, parts, groups, group_rows;   // CTAs of a sequence: slices x groups of rows; batches of a row that a slice has
};

struct LogitShared {
    unsigned long long key[MXQ_MAX_T + 1];   // accept: best token of every row, as in LogitCall::keys
    int32_t draft[MXQ_MAX_T];
    float penalties[3];
    int32_t said[MXQ_MAX_T + 1];
    int32_t listed, last;
};
// The tables of a slice in dynamic shared memory.  Rows are shifted against one another by up to kVec - 1 tokens (their vectors lie on 16-byte
// boundaries), so a batch's part of the tables has kVec tokens more than a batch.
struct SliceTables {
    uint32_t *count;                         // where there are counts
    uint16_t *bias;                          // where there are biases: the last entry of a token, plus 1
    uint32_t *special, *biased, *proposed;   // bits
    uint16_t *list;                          // places of the special tokens
    __host__ __device__ static int words(int places) { return (places + 31) / 32 + 1; }
    __host__ __device__ static size_t bytes(int places, bool counting, bool biases) {
        return (size_t)places * ((counting ? 4 : 0) + (biases ? 2 : 0) + 2) + 3 * words(places) * 4;     // (places is a multiple of 4)
    }
    __device__ SliceTables(uint32_t *at, int places, bool counting, bool biases) {
        count = at, at += counting ? places : 0;
        bias = reinterpret_cast<uint16_t *>(at), at += biases ? places / 2 : 0;
        special = at, biased = special + words(places), proposed = biased + words(places);
        list = reinterpret_cast<uint16_t *>(proposed + words(places));
    }
    __device__ __forceinline__ static uint32_t bits(const uint32_t *w, int place) { return __funnelshift_r(w[place >> 5], w[(place >> 5) + 1], place & 31); }
    // of a token's entries the last one stays (two places to a word)
    __device__ __forceinline__ void enter(int place, uint32_t entry) const {
        uint32_t *word = reinterpret_cast<uint32_t *>(bias) + place / 2, old = *word, seen;
        const int shift = 16 * (place & 1);
        do {
            if ((old >> shift & 0xFFFFu) >= entry) return;
            seen = old;
            old = atomicCAS(word, seen, (seen & ~(0xFFFFu << shift)) | entry << shift);
        } while (old != seen);
    }
    __device__ __forceinline__ static bool bit(const uint32_t *w, int place) { return w[place >> 5] >> (place & 31) & 1; }
};

__device__ __forceinline__ uint32_t ordered(float x) {   // larger float, larger number; +0 and -0 alike
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t ld_dep_u8(const void *p) {
    unsigned short v;
    asm volatile("ld.global.cg.u8 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
    return v;
}

constexpr uint32_t kNone = 0x007FFFFFu;   // ordered(-inf)

// The largest of a vector's tokens whose bits are set in `open`: NaN never counts, -inf where there is none.
template <typename T>
__device__ __forceinline__ float vector_max(const uint4 &x, uint32_t open) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, open >> e & 1 ? __uint_as_float(w[e]) : -INFINITY);
        return top;
    } else {
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
        __nv_bfloat162 top;
        if (open == 0xFFu) {
            const __nv_bfloat162 *v = reinterpret_cast<const __nv_bfloat162 *>(w);
            const float2 f = __bfloat1622float2(__hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3])));
            return fmaxf(fmaxf(f.x, f.y), -INFINITY);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t keep = ((open >> (2 * i) & 3u) * 0x8001u & 0x10001u) * 0xFFFFu;     // two bits -> two halves of ones
            w[i] = (w[i] & keep) | (0xFF80FF80u & ~keep);
            const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162 *>(&w[i]);
            top = i == 0 ? v : __hmax2(top, v);
        }
        const float2 f = __bfloat1622float2(top);
        return fmaxf(fmaxf(f.x, f.y), -INFINITY);      // (a NaN is left only where all were)
    }
}
template <typename T>
__device__ __forceinline__ float vector_at(const uint4 &x, int e) {
    const int i = sizeof(T) == 4 ? e : e >> 1;
    const uint32_t w = i & 2 ? (i & 1 ? x.w : x.z) : (i & 1 ? x.y : x.x);
    if constexpr (sizeof(T) == 4) return __uint_as_float(w);
    else return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
}
// T: float or uint16_t (BF16 bits)
template <typename T, bool WRITE, bool MASKED>
__global__ void __launch_bounds__(kLogitThreads, kLogitCtas) logit_rules_kernel(LogitCall c) {
    constexpr int kVec = 16 / sizeof(T), kTokens = kBatch * kVec, kPlaces = kTokens + kVec;    // tokens of a batch, its places in the tables
    constexpr uint32_t kAll = (1u << kVec) - 1;
    constexpr int kEntries = MXQ_MAX_BIASES / kLogitThreads;
    extern __shared__ __align__(16) uint32_t tables[];
    __shared__ LogitShared sh;
    pdl_trigger();
    const int64_t b = blockIdx.x % c.B;
    const int slice = (int)(blockIdx.x / c.B) / c.groups, group = (int)(blockIdx.x / c.B) % c.groups;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int parts = c.parts, places = parts * kPlaces;

    // Part p of the slice is batch p * slices + slice of every row: what has many special tokens (frequent ones have neighbouring, low
    // numbers) is spread over the slices.  Batch g of a row holds tokens kTokens * g - shift .., shift the tokens by which the row begins behind
    // a 16-byte boundary; its places in the tables are those of tokens kTokens * g - kVec ...  Rows r0 .. r1: a warp takes a run of their batches.
    const int r0 = group * c.group_rows, r1 = min(c.R, r0 + c.group_rows), batches = parts * (r1 - r0);
    const int from = batches * warp / kLogitWarps, to = batches * (warp + 1) / kLogitWarps;
    const T *logits = static_cast<const T *>(c.logits);
    T *out = static_cast<T *>(c.out);
    const uint8_t *allowed = reinterpret_cast<const uint8_t *>(c.allowed);
    const size_t extent = (size_t)c.B * c.R * c.V * sizeof(T), mask_extent = (size_t)c.B * c.R * c.words * 4;
    auto first_of = [&](int64_t row, int part) { return kTokens * (part * c.slices + slice) - (int)(row * c.V & (kVec - 1)); };
    auto lowest_of = [&](int part) { return kTokens * (part * c.slices + slice) - kVec; };      // token of the part's first place

    // A batch: `first` its first token (negative: the head of a row before its first 16-byte boundary); lane's vector k begins at
    // first + kVec * (32 k + lane).  Most batches lie whole inside their row: all tests below fall away.
    struct Vectors {                                     // a lane's share of a batch, as it comes from memory
        uint4 x[kBatchLoads];
        uint32_t mask[MASKED ? kBatchLoads : 1], next[MASKED ? kBatchLoads : 1];   // the mask's bytes of the vector's first token and behind
    };
    auto inside = [&](int first) { return first >= 0 && first + kTokens <= c.V; };
    auto load = [&](auto kind, Vectors &v, int64_t row, int first) {
        constexpr bool whole = decltype(kind)::value;
        const T *at = logits + row * c.V + (first + lane * kVec);
        const uint8_t *mask = allowed + (MASKED ? row * c.words * 4 : 0);
#pragma unroll
        for (int k = 0; k < kBatchLoads; ++k) {
            const int token = first + kVec * (32 * k + lane);
            if (whole || (token >= 0 && token + kVec <= c.V)) {
                v.x[k] = ld_dep_u4(MXQ_AT(at + k * 32 * kVec, 16, logits, extent));
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    if (token + e < 0 || token + e >= c.V) continue;
                    if constexpr (sizeof(T) == 4) w[e] = ld_dep_u32(MXQ_AT(at + k * 32 * kVec + e, 4, logits, extent));
                    else w[e / 2] |= (__float_as_uint(ld_dep_bf16(MXQ_AT(at + k * 32 * kVec + e, 2, logits, extent))) >> 16) << (16 * (e & 1));
                }
                v.x[k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if constexpr (MASKED) {
                v.mask[k] = v.next[k] = 0xFFu;
                const int byte = (whole ? token : max(token, 0)) >> 3;
                if (whole || token < c.V) v.mask[k] = ld_dep_u8(MXQ_AT(mask + byte, 1, c.allowed, mask_extent));
                // (vectors of a shifted row do not begin on a half byte)
                if ((first & (kVec - 1)) != 0 && (whole || token < c.V) && byte + 1 < 4 * c.words)
                    v.next[k] = ld_dep_u8(MXQ_AT(mask + byte + 1, 1, c.allowed, mask_extent));
            }
        }
    };
    auto live_of = [&](auto kind, int token) -> uint32_t {          // which of a vector's tokens there are
        constexpr bool whole = decltype(kind)::value;
        if (whole || (token >= 0 && token + kVec <= c.V)) return kAll;
        if (token >= c.V) return 0;
        uint32_t live = token < 0 ? kAll << -token & kAll : kAll;
        if (token + kVec > c.V) live &= (1u << (c.V - token)) - 1;
        return live;
    };
    auto open_of = [&](auto kind, const Vectors &v, int k, int token) -> uint32_t {     // ... and which of those the mask allows
        constexpr bool whole = decltype(kind)::value;
        if constexpr (!MASKED) return live_of(kind, token);
        const uint32_t bytes = v.mask[MASKED ? k : 0] | v.next[MASKED ? k : 0] << 8;
        if (whole) return bytes >> (token & 7) & kAll;
        return live_of(kind, token) & (bytes >> (max(token, 0) & 7)) << (max(token, 0) - token);
    };
    auto start = [&](Vectors &v, int64_t row, int first) {
        if (inside(first)) load(std::true_type(), v, row, first);
        else load(std::false_type(), v, row, first);
    };

    const bool counting = c.penalties && c.counts, tabled = counting || c.J > 0 || (c.penalties && c.T > 0);
    const SliceTables tab(tables, places, counting, c.J > 0);
    if (tabled) {
        for (int w = tid; w < 3 * SliceTables::words(places); w += kLogitThreads) tab.special[w] = 0;      // (and the two behind it)
        if (c.J > 0)
            for (int i = tid; i < places / 2; i += kLogitThreads) reinterpret_cast<uint32_t *>(tab.bias)[i] = 0;
    }
    if (!WRITE && tid <= MXQ_MAX_T) sh.key[tid] = 0;
    if (tid == 0) sh.listed = 0;
    __syncthreads();
    pdl_wait();

    // everything that the slice needs is on its way at once
    int r = r0 + from / parts, part = from % parts, first = first_of(b * c.R + r, part);
    Vectors cur, ahead;
    if (from < to) start(cur, b * c.R + r, first);
    if (tabled) {
        int32_t entry[kEntries];
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            entry[u] = -1;
            if (tid + u * kLogitThreads >= c.J) break;
            entry[u] = (int32_t)ld_dep_u32(MXQ_AT(c.bias_tokens + b * c.J + tid + u * kLogitThreads, 4, c.bias_tokens, c.B * c.J * 4));
        }
        int32_t proposal = -1;
        if (tid < c.T) proposal = (int32_t)ld_dep_u32(MXQ_AT(c.draft + b * c.T + tid, 4, c.draft, c.B * c.T * 4));
        if (tid < 3) sh.penalties[tid] = c.penalties ? ld_dep_f32(MXQ_AT(c.penalties + b * 3 + tid, 4, c.penalties, c.B * 12)) : 0.f;
        if (counting) {
            constexpr int kAtOnce = 4;                       // loads in flight per lane: four tokens each, eight lanes make a word of the bitmap
            const uint32_t *counts = c.counts + b * c.V;
            const bool wide = ((b * c.V) & 3) == 0 && (reinterpret_cast<uintptr_t>(c.counts) & 15) == 0;
            for (int begin = 0; begin < places; begin += kAtOnce * 4 * kLogitThreads) {
                uint32_t n[kAtOnce][4];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int place = begin + 4 * (u * kLogitThreads + tid), p = place / kPlaces, v = lowest_of(p) + place - p * kPlaces;
                    n[u][0] = n[u][1] = n[u][2] = n[u][3] = 0;
                    if (place >= places) continue;
                    if (wide && v >= 0 && v + 4 <= c.V) {
                        const uint4 q = ld_dep_u4(MXQ_AT(counts + v, 16, c.counts, c.B * c.V * 4));
                        n[u][0] = q.x, n[u][1] = q.y, n[u][2] = q.z, n[u][3] = q.w;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (v + e >= 0 && v + e < c.V) n[u][e] = ld_dep_u32(MXQ_AT(counts + v + e, 4, c.counts, c.B * c.V * 4));
                    }
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int place = begin + 4 * (u * kLogitThreads + tid);
                    if (place - 4 * lane >= places) continue;        // (a warp's 128 places at once)
                    uint32_t set = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) set |= (n[u][e] != 0 ? 1u : 0u) << (4 * (lane & 7) + e);
                    set |= __shfl_xor_sync(0xffffffffu, set, 1);
                    set |= __shfl_xor_sync(0xffffffffu, set, 2);
                    set |= __shfl_xor_sync(0xffffffffu, set, 4);
                    if (place < places) *reinterpret_cast<uint4 *>(&tab.count[place]) = make_uint4(n[u][0], n[u][1], n[u][2], n[u][3]);
                    if ((lane & 7) == 0 && set != 0) atomicOr(&tab.special[place / 32], set);
                }
            }
        }
        // A token's places: in the batch of its number, and in the next one's if it is among the last kVec of its batch.
        auto place_of = [&](int v, int which) {
            if (v < 0 || v >= c.V) return -1;
            const int g = v / kTokens + which;
            if ((which == 1 && v % kTokens < kTokens - kVec) || g % c.slices != slice || g / c.slices >= parts) return -1;
            return g / c.slices * kPlaces + v - (kTokens * g - kVec);
        };
        auto mark = [&](uint32_t *kind, int place) {
            atomicOr(&kind[place >> 5], 1u << (place & 31));
            atomicOr(&tab.special[place >> 5], 1u << (place & 31));
        };
        if (tid < c.T) {
            sh.draft[tid] = proposal;
            if (c.penalties)
                for (int which = 0; which < 2; ++which) {
                    const int place = place_of(proposal, which);
                    if (place >= 0) mark(tab.proposed, place);
                }
        }
#pragma unroll
        for (int u = 0; u < kEntries; ++u) {
            if (tid + u * kLogitThreads >= c.J) break;
            for (int which = 0; which < 2; ++which) {
                const int place = place_of(entry[u], which);
                if (place < 0) continue;
                mark(tab.biased, place);
                tab.enter(place, tid + u * kLogitThreads + 1);
            }
        }
        __syncthreads();
    }

    // the stream; accept keeps the best vector of this lane's in the row
    float best = -INFINITY;
    int best_token = 0;
    uint4 best_x = make_uint4(0, 0, 0, 0);
    uint32_t best_open = 0;
    for (int n = from; n < to; ++n) {
        const int64_t row = b * c.R + r;
        const int rank = r, now = first, place0 = part * kPlaces + now - lowest_of(part);
        if (++part == parts) part = 0, ++r;
        first = first_of(b * c.R + r, part);
        if (n + 1 < to) start(ahead, b * c.R + r, first);
        // most batches hold few special tokens or none
        bool any = false;
        if (!WRITE && tabled) {
            const int w = (place0 >> 5) + lane;
            any = __any_sync(0xffffffffu, lane < kTokens / 32 + 1 && w < SliceTables::words(places) && tab.special[w] != 0);
        }
        auto process = [&](auto kind) {
            constexpr bool whole = decltype(kind)::value;
#pragma unroll
            for (int k = 0; k < kBatchLoads; ++k) {
                const int token = now + kVec * (32 * k + lane);
                uint32_t open = open_of(kind, cur, k, token);
                const uint4 x = cur.x[k];
                if constexpr (!WRITE) {
                    if (any) open &= ~SliceTables::bits(tab.special, place0 + kVec * (32 * k + lane));
                    const float top = vector_max<T>(x, open);
                    if (top > best) best = top, best_token = token, best_x = x, best_open = open;   // (a lane's tokens ascend)
                } else {
                    const uint32_t live = live_of(kind, token), gone = live & ~open;
                    uint32_t w[4] = {x.x, x.y, x.z, x.w};
                    if (MASKED && gone) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (sizeof(T) == 4) {
                                if (gone >> i & 1) w[i] = 0xFF800000u;
                            } else {
                                const uint32_t drop = ((gone >> (2 * i) & 3u) * 0x8001u & 0x10001u) * 0xFFFFu;
                                w[i] = (w[i] & ~drop) | (0xFF80FF80u & drop);
                            }
                        }
                    }
                    T *dst = out + row * c.V + token;
                    if (whole || live == kAll) {
                        *reinterpret_cast<uint4 *>(MXQ_AT(dst, 16, out, extent)) = make_uint4(w[0], w[1], w[2], w[3]);
                    } else {
#pragma unroll
                        for (int e = 0; e < kVec; ++e) {
                            if (!(live >> e & 1)) continue;
                            if constexpr (sizeof(T) == 4) *MXQ_AT(dst + e, 4, out, extent) = __uint_as_float(w[e]);
                            else *MXQ_AT(dst + e, 2, out, extent) = (T)(w[e / 2] >> (16 * (e & 1)));
                        }
                    }
                }
            }
        };
        if (inside(now)) process(std::true_type());
        else process(std::false_type());
        if constexpr (!WRITE) {
            if (part == 0 || n + 1 == to) {              // the last of this warp's batches of the row
                const uint32_t most = __reduce_max_sync(0xffffffffu, ordered(best));
                if (most != kNone) {
                    // of the vectors that hold the maximum the one with the lowest tokens, and of its tokens, one per lane, the lowest
                    const uint32_t mine = ordered(best) == most ? (uint32_t)(best_token + kVec) : 0xFFFFFFFFu, lowest = __reduce_min_sync(0xffffffffu, mine);
                    const int owner = __ffs(__ballot_sync(0xffffffffu, mine == lowest)) - 1;
                    const uint4 v = make_uint4(__shfl_sync(0xffffffffu, best_x.x, owner), __shfl_sync(0xffffffffu, best_x.y, owner),
                                               __shfl_sync(0xffffffffu, best_x.z, owner), __shfl_sync(0xffffffffu, best_x.w, owner));
                    const uint32_t open = __shfl_sync(0xffffffffu, best_open, owner);
                    const uint32_t hit = __ballot_sync(0xffffffffu, lane < kVec && (open >> (lane & (kVec - 1)) & 1) && ordered(vector_at<T>(v, lane & (kVec - 1))) == most);
                    if (lane == 0) atomicMax(&sh.key[rank - r0], (unsigned long long)most << 32 | (uint32_t)~((int)lowest - kVec + __ffs(hit) - 1));
                }
                best = -INFINITY;
            }
        }
        cur = ahead;
    }
    if (tabled) {
        // the list of the special tokens, in any order
        for (int w0 = 32 * warp; w0 < SliceTables::words(places); w0 += kLogitThreads) {
            uint32_t left = w0 + lane < SliceTables::words(places) ? tab.special[w0 + lane] : 0;
            int before = __popc(left);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int n = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += n;
            }
            int at = 0;
            if (lane == 31 && before != 0) at = atomicAdd(&sh.listed, before);
            at = __shfl_sync(0xffffffffu, at, 31) + before - __popc(left);
            for (; left; left &= left - 1) tab.list[at++] = (uint16_t)(32 * (w0 + lane) + __ffs(left) - 1);
        }
        __syncthreads();     // (the list is there; the stream's stores come before those of the special tokens)

        const int listed = sh.listed, pairs = listed * (r1 - r0);
        const float repetition = sh.penalties[0], presence = sh.penalties[1], frequency = sh.penalties[2];
        for (int u0 = tid; u0 < pairs; u0 += kPairs * kLogitThreads) {
            float x[kPairs];
            uint32_t mask[kPairs];
            int place[kPairs], token[kPairs], rank[kPairs];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                const int u = u0 + i * kLogitThreads, q = u / listed;
                rank[i] = r0 + q;
                place[i] = u < pairs ? tab.list[u - q * listed] : 0;
                const int p = place[i] / kPlaces;
                token[i] = lowest_of(p) + place[i] - p * kPlaces;
                const int64_t row = b * c.R + rank[i];
                const int inside_batch = token[i] - first_of(row, p);      // (the tables overlap: the token may be another batch's in this row)
                mask[i] = 0;
                x[i] = 0.f;
                if (u >= pairs || inside_batch < 0 || inside_batch >= kTokens) continue;
                const int64_t at = row * c.V + token[i];
                if constexpr (sizeof(T) == 4) x[i] = ld_dep_f32(MXQ_AT(logits + at, 4, logits, extent));
                else x[i] = ld_dep_bf16(MXQ_AT(logits + at, 2, logits, extent));
                mask[i] = MASKED ? ld_dep_u8(MXQ_AT(allowed + row * c.words * 4 + (token[i] >> 3), 1, c.allowed, mask_extent)) >> (token[i] & 7) & 1 : 1;
            }
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                if (mask[i] == 0) continue;
                if (c.penalties) {
                    const uint32_t count = counting ? tab.count[place[i]] : 0;
                    uint32_t made = count & 0x7FFFFFFFu;
                    if (SliceTables::bit(tab.proposed, place[i]))
                        for (int j = 0; j < min(rank[i], c.T); ++j) made += sh.draft[j] == token[i];
                    if ((count | made) != 0) x[i] = x[i] > 0.f ? __fdiv_rn(x[i], repetition) : __fmul_rn(x[i], repetition);
                    if (made != 0) x[i] = __fsub_rn(__fsub_rn(x[i], __fmul_rn(frequency, (float)made)), presence);
                }
                if (SliceTables::bit(tab.biased, place[i])) x[i] = __fadd_rn(x[i], ld_dep_f32(MXQ_AT(c.bias_values + b * c.J + tab.bias[place[i]] - 1, 4, c.bias_values, c.B * c.J * 4)));
                if constexpr (WRITE) {
                    const int64_t at = (b * c.R + rank[i]) * c.V + token[i];
                    if constexpr (sizeof(T) == 4) *MXQ_AT(out + at, 4, out, extent) = x[i];
                    else *MXQ_AT(out + at, 2, out, extent) = __bfloat16_as_ushort(__float2bfloat16_rn(x[i]));
                } else if (x[i] > -INFINITY) {           // (neither NaN nor -inf is ever chosen)
                    const unsigned long long key = (unsigned long long)ordered(x[i]) << 32 | (uint32_t)~token[i];
                    if (key > *(volatile unsigned long long *)&sh.key[rank[i] - r0]) atomicMax(&sh.key[rank[i] - r0], key);
                }
            }
        }
    }
    if constexpr (!WRITE) {
        __syncthreads();
        if (tid < r1 - r0 && sh.key[tid] != 0) atomicMax(MXQ_AT(c.keys + b * c.R + r0 + tid, 8, c.keys, c.B * c.R * 8), sh.key[tid]);
        // the last CTA of a sequence finishes it, and leaves keys and ticket zero for the next call
        __syncthreads();
        if (tid == 0) {
            __threadfence();       // (cumulative: the barrier has put the other threads' maxima before it)
            sh.last = atomicAdd(MXQ_AT(c.tickets + b, 4, c.tickets, c.B * 4), 1u) == (unsigned)(c.slices * c.groups) - 1u;
            __threadfence();
        }
        __syncthreads();
        if (!sh.last) return;
        if (tid < c.R) {
            unsigned long long *key = MXQ_AT(c.keys + b * c.R + tid, 8, c.keys, c.B * c.R * 8);
            const unsigned long long k = __ldcg(key);
            const int32_t token = k == 0 ? 0 : (int32_t)~(uint32_t)k;
            sh.said[tid] = token;
            *MXQ_AT(c.verifier + b * c.R + tid, 4, c.verifier, c.B * c.R * 4) = token;
            *key = 0;
        }
        if (tid < c.T && !tabled) sh.draft[tid] = (int32_t)ld_dep_u32(MXQ_AT(c.draft + b * c.T + tid, 4, c.draft, c.B * c.T * 4));
        __syncthreads();
        if (tid == 0) {
            int n = 0;
            while (n < c.T && sh.draft[n] == sh.said[n]) ++n;     // (T <= R)
            *MXQ_AT(c.accept_len + b, 4, c.accept_len, c.B * 4) = n;
            *MXQ_AT(c.next_token + b, 4, c.next_token, c.B * 4) = n < c.R ? sh.said[n] : -1;
            c.tickets[b] = 0;
        }
    }
}

// A thread takes one token.  Tokens repeat: lanes of a warp with the same token add once for all of them, and a prompt's mark that
// is there already is not set again (20000 tokens of a skewed prompt would otherwise queue at a few words).
__global__ void __launch_bounds__(256) token_counts_kernel(uint32_t *counts, int64_t B, int64_t V, const int32_t *tokens, int64_t L, const int32_t *n,
                                                           const int32_t *extra, int prompt, unsigned ctas_per_row) {
    pdl_trigger();
    const int64_t b = blockIdx.x / ctas_per_row, i = (int64_t)(blockIdx.x - b * ctas_per_row) * 256 + threadIdx.x;
    pdl_wait();
    const int64_t have = n ? max((int64_t)0, min(L, (int64_t)(int)ld_dep_u32(MXQ_AT(n + b, 4, n, B * 4)))) : L;
    int token = -1;
    if (i < have) token = (int)ld_dep_u32(MXQ_AT(tokens + b * L + i, 4, tokens, B * L * 4));
    else if (i == L && extra) token = (int)ld_dep_u32(MXQ_AT(extra + b, 4, extra, B * 4));
    const bool mine = token >= 0 && token < V;
    const unsigned same = __match_any_sync(0xffffffffu, mine ? token : -1);
    if (!mine || (int)(threadIdx.x & 31) != __ffs(same) - 1) return;
    uint32_t *at = MXQ_AT(counts + b * V + token, 4, counts, B * V * 4);
    if (!prompt) atomicAdd(at, (uint32_t)__popc(same));
    else if (!(ld_dep_u32(at) >> 31)) atomicOr(at, 0x80000000u);
}

MXQ_BOUNDS_TU(bounds_take_logits)

// ---- host ---------------------------------------------------------------------------------------------------------------

static int check_logits(const void *logits, int dtype, int64_t B, int R, int64_t V, const int32_t *draft, int T, const mxq_logit_rules *rules) {
    if (!logits || !rules || (T > 0 && !draft)) return MXQ_ERR_NULL;
    if (rules->bias_count != 0 && (!rules->bias_tokens || !rules->bias_values)) return MXQ_ERR_NULL;
    if (B < 1 || V < 1 || V > INT_MAX - 65536 || T < 0 || T > MXQ_MAX_T || R < 1 || (R != T && R != T + 1) || B > ((int64_t)INT_MAX / 1024) / R ||
        rules->bias_count < 0 || rules->bias_count > MXQ_MAX_BIASES)
        return MXQ_ERR_SHAPE;
    if (dtype != MXQ_F32 && dtype != MXQ_BF16) return MXQ_ERR_DTYPE;
    const void *words[] = {draft, rules->counts, rules->penalties, rules->bias_tokens, rules->bias_values, rules->allowed};
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MXQ_ERR_ALIGN;
    return aligned16(logits) ? MXQ_OK : MXQ_ERR_ALIGN;
}

constexpr size_t kLogitSmem = 73 * 1024;     // most of a CTA's tables
template <typename T, bool WRITE, bool MASKED>
static int rules_launch(const LogitCall &c, int64_t ctas, size_t smem, cudaStream_t stream) {
    static std::atomic<bool> ready[64];
    const int rc = allow_smem(logit_rules_kernel<T, WRITE, MASKED>, kLogitSmem, ready);
    return rc != MXQ_OK ? rc : launch_pdl(logit_rules_kernel<T, WRITE, MASKED>, dim3((unsigned)ctas), kLogitThreads, smem, stream, c);
}

static int logits_launch(LogitCall &c, const void *logits, int dtype, int64_t B, int R, int64_t V, const int32_t *draft, int T,
                         const mxq_logit_rules *rules, cudaStream_t stream) {
    c.logits = logits, c.draft = draft, c.B = B, c.R = R, c.V = V, c.T = T, c.words = (V + 31) / 32;
    c.counts = rules->counts, c.penalties = rules->penalties, c.allowed = rules->allowed;
    c.bias_tokens = rules->bias_tokens, c.bias_values = rules->bias_values, c.J = rules->bias_count;
    // A CTA takes all rows of its slice, so that the slice's tables are made once; many rows of few sequences are spread over CTAs.  How many
    // batches of a row: the number for which the waves of CTAs take least, a CTA costing about as much as five batches of a warp beside its own.
    const int64_t sms = sm_count(), vec = dtype == MXQ_F32 ? 4 : 8, tokens = kBatch * vec, row_batches = (V + vec - 1 + tokens - 1) / tokens;
    const bool counting = c.counts && c.penalties;
    double least = 0;
    c.parts = 0;
    for (int parts = 1; parts <= 32 && parts <= row_batches; ++parts) {
        const size_t smem = SliceTables::bytes((int)(parts * (tokens + vec)), counting, c.J > 0);
        if (smem > kLogitSmem) break;
        const int64_t slices = (row_batches + parts - 1) / parts;
        const int64_t groups = max((int64_t)1, min(2 * sms / (B * slices), (int64_t)R * parts / kLogitWarps)), rows = (R + groups - 1) / groups;
        const int64_t waves = (B * slices * ((R + rows - 1) / rows) + kLogitCtas * sms - 1) / (kLogitCtas * sms);
        const double cost = (double)waves * (5 + (rows * parts + kLogitWarps - 1) / kLogitWarps);
        if (c.parts != 0 && cost >= least) continue;
        least = cost;
        c.parts = parts, c.slices = (int)slices, c.group_rows = (int)rows, c.groups = (int)((R + rows - 1) / rows);
    }
    const size_t smem = SliceTables::bytes((int)(c.parts * (tokens + vec)), counting, c.J > 0);
    const int64_t ctas = B * c.groups * c.slices;
    if (ctas > INT_MAX) return MXQ_ERR_SHAPE;
    const bool f32 = dtype == MXQ_F32, masked = c.allowed != nullptr;
    return c.out ? (f32 ? (masked ? rules_launch<float, true, true>(c, ctas, smem, stream) : rules_launch<float, true, false>(c, ctas, smem, stream))
                        : (masked ? rules_launch<uint16_t, true, true>(c, ctas, smem, stream) : rules_launch<uint16_t, true, false>(c, ctas, smem, stream)))
                 : (f32 ? (masked ? rules_launch<float, false, true>(c, ctas, smem, stream) : rules_launch<float, false, false>(c, ctas, smem, stream))
                        : (masked ? rules_launch<uint16_t, false, true>(c, ctas, smem, stream) : rules_launch<uint16_t, false, false>(c, ctas, smem, stream)));
}

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

int mxq_logits_adjust(const void *logits, int dtype, int64_t B, int R, int64_t V, const int32_t *draft, int T, const mxq_logit_rules *rules,
                      void *out, void *stream) {
    if (!out) return MXQ_ERR_NULL;
    const int rc = mxq::check_logits(logits, dtype, B, R, V, draft, T, rules);
    if (rc != MXQ_OK) return rc;
    if (!mxq::aligned16(out)) return MXQ_ERR_ALIGN;
    mxq::LogitCall c = {};
    c.out = out;
    return mxq::logits_launch(c, logits, dtype, B, R, V, draft, T, rules, (cudaStream_t)stream);
}

size_t mxq_greedy_accept_rules_workspace_bytes(int64_t B, int R, int64_t V) {
    if (B < 1 || R < 1 || R > MXQ_MAX_T + 1 || V < 1 || B > ((int64_t)INT_MAX / 1024) / R) return 0;
    return ((size_t)B * R * 8 + (size_t)B * 4 + 15) / 16 * 16;
}

int mxq_greedy_accept_rules(const void *logits, int dtype, int64_t B, int R, int64_t V, const int32_t *draft, int T, const mxq_logit_rules *rules,
                            int32_t *verifier, int32_t *accept_len, int32_t *next_token, void *workspace, size_t workspace_bytes, void *stream) {
    if (!verifier || !accept_len || !next_token) return MXQ_ERR_NULL;
    const int rc = mxq::check_logits(logits, dtype, B, R, V, draft, T, rules);
    if (rc != MXQ_OK) return rc;
    if (!workspace || workspace_bytes < mxq_greedy_accept_rules_workspace_bytes(B, R, V)) return MXQ_ERR_WORKSPACE;
    const void *words[] = {verifier, accept_len, next_token};
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MXQ_ERR_ALIGN;
    if (!mxq::aligned16(workspace)) return MXQ_ERR_ALIGN;
    mxq::LogitCall c = {};
    c.keys = static_cast<unsigned long long *>(workspace);
    c.tickets = reinterpret_cast<unsigned *>(c.keys + B * R);
    c.verifier = verifier, c.accept_len = accept_len, c.next_token = next_token;
    return mxq::logits_launch(c, logits, dtype, B, R, V, draft, T, rules, (cudaStream_t)stream);
}

int mxq_token_counts(uint32_t *counts, int64_t B, int64_t V, const int32_t *tokens, int64_t L, const int32_t *n, const int32_t *next_token, int prompt,
                     void *stream) {
    if (!counts || !tokens) return MXQ_ERR_NULL;
    if (B < 1 || V < 1 || V > INT_MAX - 65536 || L < 1 || L > ((int64_t)1 << 31)) return MXQ_ERR_SHAPE;
    const void *words[] = {counts, tokens, n, next_token};
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MXQ_ERR_ALIGN;
    const int64_t per_row = (L + (next_token ? 1 : 0) + 255) / 256;
    if (B > INT_MAX / per_row) return MXQ_ERR_SHAPE;
    return mxq::launch_pdl(mxq::token_counts_kernel, dim3((unsigned)(B * per_row)), 256, 0, (cudaStream_t)stream, counts, B, V, tokens, L, n, next_token, prompt,
                           (unsigned)per_row);
}

#pragma GCC visibility pop
}  // extern "C"
