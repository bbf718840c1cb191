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
// A stream over the logits (and the mask's bits).  The rules but the mask touch few tokens: a CTA reads its slice of the counts
// once for all of its rows and keeps one bit per token that is special (counted, biased or proposed); the stream tests the bits
// of a 16-byte vector at once and leaves the fast path only where one is set.
#include <limits.h>

#include "mxq_device.cuh"
#include "mxq_host.h"

namespace mxq {

constexpr int kLogitThreads = 256;
constexpr int kLogitWarps = kLogitThreads / 32;
constexpr int kMaxSlice = 16384;        // tokens of a CTA's slice (its bitmaps are in shared memory)
constexpr int kSliceStep = 1024;
constexpr int kBatchLoads = 4;          // 16-byte loads in flight per lane

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
    int32_t slices, slice_len, groups, group_rows;   // CTAs of a sequence: slices x groups of rows
};

struct LogitShared {
    uint32_t special[kMaxSlice / 32 + 2], biased[kMaxSlice / 32 + 2];   // bits of tokens slice begin .. slice end + 32
    int32_t list_token[MXQ_MAX_BIASES], list_entry[MXQ_MAX_BIASES];     // the biases of this slice, in any order
    int32_t draft[MXQ_MAX_T];
    int32_t listed;
    float penalties[3];
    int32_t said[MXQ_MAX_T + 1];
    int32_t last;
};

// the rules but the mask, for one token of row r
__device__ __noinline__ float apply_rules(const LogitCall &c, const LogitShared &sh, float x, int64_t b, int r, int v) {
    if (c.penalties) {
        uint32_t count = 0;
        if (c.counts) count = ld_dep_u32(MXQ_AT(c.counts + b * c.V + v, 4, c.counts, c.B * c.V * 4));
        uint32_t made = count & 0x7FFFFFFFu;
        for (int i = 0; i < min(r, c.T); ++i) made += sh.draft[i] == v;
        if (made != 0 || count != 0) x = x > 0.f ? __fdiv_rn(x, sh.penalties[0]) : __fmul_rn(x, sh.penalties[0]);
        if (made != 0) x = __fsub_rn(__fsub_rn(x, __fmul_rn(sh.penalties[2], (float)made)), sh.penalties[1]);
    }
    int entry = -1;
    for (int i = 0; i < sh.listed; ++i)
        if (sh.list_token[i] == v) entry = max(entry, sh.list_entry[i]);
    if (entry >= 0) x = __fadd_rn(x, ld_dep_f32(MXQ_AT(c.bias_values + b * c.J + entry, 4, c.bias_values, c.B * c.J * 4)));
    return x;
}

__device__ __forceinline__ uint32_t ordered(float x) {   // larger float, larger number; +0 and -0 alike
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// T: float or uint16_t (BF16 bits)
template <typename T, bool WRITE>
__global__ void __launch_bounds__(kLogitThreads) logit_rules_kernel(LogitCall c) {
    constexpr int kVec = 16 / sizeof(T);
    __shared__ LogitShared sh;
    pdl_trigger();
    const int slice = blockIdx.x % c.slices, group = blockIdx.x / c.slices % c.groups;
    const int64_t b = blockIdx.x / (c.slices * c.groups);
    const int lo = slice * c.slice_len, hi = (int)min(c.V, (int64_t)lo + c.slice_len), reach = (int)min(c.V, (int64_t)hi + 32);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();

    // the special tokens of the slice (a 16-byte vector may begin in it and end up to 7 tokens behind it)
    const bool counting = c.penalties && c.counts;
    const int bits = (reach - lo + 31) / 32;
    for (int w = warp; w < c.slice_len / 32 + 2; w += kLogitWarps) {
        const int v = lo + 32 * w + lane;
        uint32_t set = 0;
        if (counting && w < bits) set = __ballot_sync(0xffffffffu, v < reach && ld_dep_u32(MXQ_AT(c.counts + b * c.V + min(v, reach - 1), 4, c.counts, c.B * c.V * 4)) != 0);
        if (lane == 0) sh.special[w] = set, sh.biased[w] = 0;
    }
    if (threadIdx.x < c.T) sh.draft[threadIdx.x] = (int32_t)ld_dep_u32(MXQ_AT(c.draft + b * c.T + threadIdx.x, 4, c.draft, c.B * c.T * 4));
    if (threadIdx.x < 3) sh.penalties[threadIdx.x] = c.penalties ? ld_dep_f32(MXQ_AT(c.penalties + b * 3 + threadIdx.x, 4, c.penalties, c.B * 12)) : 0.f;
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    if (c.penalties && threadIdx.x < c.T) {
        const int v = sh.draft[threadIdx.x];
        if (v >= lo && v < reach) atomicOr(&sh.special[(v - lo) >> 5], 1u << ((v - lo) & 31));
    }
    for (int j = threadIdx.x; j < c.J; j += kLogitThreads) {
        const int v = (int)ld_dep_u32(MXQ_AT(c.bias_tokens + b * c.J + j, 4, c.bias_tokens, c.B * c.J * 4));
        if (v < lo || v >= reach) continue;
        atomicOr(&sh.special[(v - lo) >> 5], 1u << ((v - lo) & 31));
        const int at = atomicAdd(&sh.listed, 1);
        sh.list_token[at] = v, sh.list_entry[at] = j;
    }
    __syncthreads();

    // Rows r0 .. r1 of the slice, in batches of 32 x kBatchLoads vectors; a warp takes a run of batches.  A row's vectors lie on
    // 16-byte boundaries: vector n of a row begins at token first + kVec * (n - 1), its first and last may be partial.
    const int r0 = group * c.group_rows, r1 = min(c.R, r0 + c.group_rows);
    constexpr int kBatch = 32 * kBatchLoads;
    const int per_row = (c.slice_len / kVec + 1 + kBatch - 1) / kBatch, batches = per_row * (r1 - r0);
    const int from = (int)((int64_t)batches * warp / kLogitWarps), to = (int)((int64_t)batches * (warp + 1) / kLogitWarps);
    const T *logits = static_cast<const T *>(c.logits);
    T *out = static_cast<T *>(c.out);
    const size_t extent = (size_t)c.B * c.R * c.V * sizeof(T);
    uint32_t best = 0, best_token = 0xFFFFFFFFu;
    for (int n = from; n < to; ++n) {
        const int r = r0 + n / per_row, part = n % per_row;
        const int64_t row = b * c.R + r, base = row * c.V;
        const int first = (int)((kVec - base % kVec) % kVec);          // first token of the row on a 16-byte boundary
        // vectors of this slice: those that begin in it (the head of a row, before `first`, in the first slice)
        const int n0 = lo == 0 ? (first == 0 ? 1 : 0) : (lo - first + kVec - 1) / kVec + 1;
        uint4 x[kBatchLoads];
        int token[kBatchLoads];
        uint32_t live[kBatchLoads];                                     // tokens of the vector that there are
#pragma unroll
        for (int k = 0; k < kBatchLoads; ++k) {
            token[k] = first + kVec * (n0 + part * kBatch + k * 32 + lane - 1);
            live[k] = 0;
            x[k] = make_uint4(0, 0, 0, 0);
            if (max(token[k], 0) >= hi) continue;
            if (token[k] >= 0 && token[k] + kVec <= c.V) {
                live[k] = (1u << kVec) - 1;
                x[k] = ld_dep_u4(MXQ_AT(logits + base + token[k], 16, logits, extent));
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const int v = token[k] + e;
                    if (v < 0 || v >= c.V) continue;
                    live[k] |= 1u << e;
                    if constexpr (sizeof(T) == 4) w[e] = ld_dep_u32(MXQ_AT(logits + base + v, 4, logits, extent));
                    else w[e / 2] |= (__float_as_uint(ld_dep_bf16(MXQ_AT(logits + base + v, 2, logits, extent))) >> 16) << (16 * (e & 1));
                }
                x[k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
#pragma unroll
        for (int k = 0; k < kBatchLoads; ++k) {
            if (live[k] == 0) continue;
            float f[kVec];
            if constexpr (sizeof(T) == 4) {
                f[0] = __uint_as_float(x[k].x), f[1] = __uint_as_float(x[k].y), f[2] = __uint_as_float(x[k].z), f[3] = __uint_as_float(x[k].w);
            } else {
                unpack_bf16(f, x[k]);
            }
            // the bits of tokens token .. token + kVec - 1 (before token 0 there are none: shifted in from below)
            const int t0 = max(token[k], 0), skip = t0 - token[k], off = t0 - lo;
            uint32_t special = __funnelshift_r(sh.special[off >> 5], sh.special[(off >> 5) + 1], off & 31) << skip & live[k];
            uint32_t open = live[k];
            if (c.allowed) {
                const uint32_t *m = c.allowed + row * c.words;
                const size_t all = (size_t)c.B * c.R * c.words * 4;
                const uint32_t m0 = ld_dep_u32(MXQ_AT(m + (t0 >> 5), 4, c.allowed, all));
                const uint32_t m1 = (t0 >> 5) + 1 < c.words ? ld_dep_u32(MXQ_AT(m + (t0 >> 5) + 1, 4, c.allowed, all)) : 0;
                open &= __funnelshift_r(m0, m1, t0 & 31) << skip;
            }
            special &= open;
            if (special) {
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (special >> e & 1) f[e] = apply_rules(c, sh, f[e], b, r, token[k] + e);
            }
            if constexpr (WRITE) {
                if (open != live[k] || special) {
#pragma unroll
                    for (int e = 0; e < kVec; ++e)
                        if (!(open >> e & 1)) f[e] = -INFINITY;
                    if constexpr (sizeof(T) == 4) x[k] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                    else x[k] = pack_bf16(f);
                }
                if (live[k] == (1u << kVec) - 1) {
                    *reinterpret_cast<uint4 *>(MXQ_AT(out + base + token[k], 16, out, extent)) = x[k];
                } else {
                    const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        if (!(live[k] >> e & 1)) continue;
                        T *dst = MXQ_AT(out + base + token[k] + e, sizeof(T), out, extent);
                        if constexpr (sizeof(T) == 4) *dst = __uint_as_float(w[e]);
                        else *dst = (T)(w[e / 2] >> (16 * (e & 1)));
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    if (!(open >> e & 1) || !(f[e] > -INFINITY)) continue;   // (neither NaN nor -inf is ever chosen)
                    const uint32_t o = ordered(f[e]);
                    if (o > best) best = o, best_token = (uint32_t)(token[k] + e);   // (a lane's tokens ascend: a tie stays with the lower one)
                }
            }
        }
        if constexpr (!WRITE) {
            if (n + 1 == to || (n + 1) % per_row == 0) {      // the last of this warp's batches of the row
                const uint32_t top = __reduce_max_sync(0xffffffffu, best);
                const uint32_t token = __reduce_min_sync(0xffffffffu, best == top ? best_token : 0xFFFFFFFFu);
                if (lane == 0 && top != 0)
                    atomicMax(MXQ_AT(c.keys + row, 8, c.keys, c.B * c.R * 8), (unsigned long long)top << 32 | (uint32_t)~token);
                best = 0, best_token = 0xFFFFFFFFu;
            }
        }
    }
    if constexpr (!WRITE) {
        // the last CTA of a sequence finishes it, and leaves keys and ticket zero for the next call
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) sh.last = atomicAdd(MXQ_AT(c.tickets + b, 4, c.tickets, c.B * 4), 1u) == (unsigned)(c.slices * c.groups) - 1u;
        __syncthreads();
        if (!sh.last) return;
        __threadfence();
        if (threadIdx.x < c.R) {
            unsigned long long *key = MXQ_AT(c.keys + b * c.R + threadIdx.x, 8, c.keys, c.B * c.R * 8);
            const unsigned long long k = __ldcg(key);
            const int32_t token = k == 0 ? 0 : (int32_t)~(uint32_t)k;
            sh.said[threadIdx.x] = token;
            *MXQ_AT(c.verifier + b * c.R + threadIdx.x, 4, c.verifier, c.B * c.R * 4) = token;
            *key = 0;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
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

static int logits_launch(LogitCall &c, const void *logits, int dtype, int64_t B, int R, int64_t V, const int32_t *draft, int T,
                         const mxq_logit_rules *rules, cudaStream_t stream) {
    c.logits = logits, c.draft = draft, c.B = B, c.R = R, c.V = V, c.T = T, c.words = (V + 31) / 32;
    c.counts = rules->counts, c.penalties = rules->penalties, c.allowed = rules->allowed;
    c.bias_tokens = rules->bias_tokens, c.bias_values = rules->bias_values, c.J = rules->bias_count;
    // Few sequences: the rows of a slice are spread over CTAs, until there are two CTAs per SM; else a CTA takes all rows of its
    // slice and reads the counts once.  Then slices small enough for eight CTAs per SM.
    const int64_t sms = sm_count(), coarse = (V + 4095) / 4096;
    c.groups = (int)max((int64_t)1, min((int64_t)R, (2 * sms + B * coarse - 1) / (B * coarse)));
    c.group_rows = (R + c.groups - 1) / c.groups;
    c.groups = (R + c.group_rows - 1) / c.group_rows;
    int64_t want = max((int64_t)1, (8 * sms + B * c.groups - 1) / (B * c.groups));
    want = min(want, (V + 2047) / 2048);
    int64_t len = ((V + want - 1) / want + kSliceStep - 1) / kSliceStep * kSliceStep;
    if (len > kMaxSlice) len = kMaxSlice;
    c.slice_len = (int)len;
    c.slices = (int)((V + len - 1) / len);
    const int64_t ctas = B * c.groups * c.slices;
    if (ctas > INT_MAX) return MXQ_ERR_SHAPE;
    if (c.out)
        return launch_pdl(dtype == MXQ_F32 ? logit_rules_kernel<float, true> : logit_rules_kernel<uint16_t, true>, dim3((unsigned)ctas), kLogitThreads, 0, stream, c);
    return launch_pdl(dtype == MXQ_F32 ? logit_rules_kernel<float, false> : logit_rules_kernel<uint16_t, false>, dim3((unsigned)ctas), kLogitThreads, 0, stream, c);
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
