// mxq_lora: low-rank adapters of many requests at once, added to what a shared projection computed; mxq_linear_lora: the 4-bit
// layer and its adapters in one call.
//
//     Y[m] = base[m] + s[a] * B[a] (A[a] x[m]),   a = ids[m]   (A [r][K], B [N][r] BF16; no adapter: Y[m] = base[m])
//
// Two kernels: T = A x into the workspace (shrink), then base + B T (expand).  Both are bound by the adapters' bytes for a few token
// rows and by X, base and Y for many; the products are m16n8k16 mma.sync with the token rows as m, fed from global memory by 16- and 8-byte
// loads whose order along the contracted axis is the same for both operands (the sum does not mind the order).  (tcgen05 has nothing
// to give here: at 16 to 128 ranks the products are 1 to 10 % of the tensor pipe's time, and its operands would have to pass
// through shared memory first.)  T is FP32 and meets B as a sum of BF16 parts: three for an FP32 Y (all 24 bits), two for a BF16 Y (16 bits: what
// is lost is 2^-17 of each product, against the 2^-8 of Y's own rounding).
//
// A CTA takes a window of 16 or 64 token rows and goes through the adapters that its rows have, one after the other: rows that have
// another one are left out (zero in the product, not stored).  For up to 16 rows a CTA takes one adapter only (`slots`).
#include "mxq_device.cuh"
#include "mxq_host.h"

namespace mxq {

constexpr int kShrinkThreads = 256, kShrinkWarps = 8;
constexpr int kWindowMost = 64;

struct LoraCall {
    const uint16_t *x;       // [M][K]
    const uint16_t *a, *b;   // [L][r][K], [L][N][r]
    const float *scale;      // [L] or nullptr
    const int32_t *ids;      // [M]
    const uint8_t *base;     // [M][N] or nullptr (zero)
    uint8_t *y;              // [M][N]
    float *t;                // [splits][M][r]
    int64_t N, K;
    int32_t M, r, L;
    int32_t slots;           // CTAs of a window; slot s takes its adapters s, s + slots, ...
    int32_t splits, split_k; // shrink: CTAs along K, and how much of K each takes (a multiple of 32)
    int32_t base_f32, y_f32;
    int32_t parts;           // BF16 parts of T
};

struct Window {
    int32_t owner[kWindowMost];   // adapter of every row, -1: none
    int32_t list[kWindowMost];    // its distinct adapters in order of their first row
    int32_t count;
};

// filled by warp 0; the caller synchronises.  ids are read ahead of the wait for the previous kernel (they are the caller's, like the
// weights).
__device__ __forceinline__ void load_window(Window &w, const LoraCall &c, int row0, int rows) {
    if (threadIdx.x >= 32) return;
    const int lane = threadIdx.x;
    int o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = 32 * h + lane;
        o[h] = -1;
        if (i < rows && row0 + i < c.M) o[h] = __ldg(MXQ_AT(c.ids + row0 + i, 4, c.ids, (size_t)c.M * 4));
        if (o[h] < 0 || o[h] >= c.L) o[h] = -1;
        w.owner[i] = o[h];
    }
    unsigned first = __ballot_sync(0xffffffffu, (__ffs(__match_any_sync(0xffffffffu, o[0])) - 1 == lane) && o[0] >= 0);
    int n = 0;
    bool known = false;
    for (unsigned left = first; left; left &= left - 1) {
        const int a = __shfl_sync(0xffffffffu, o[0], __ffs(left) - 1);
        known |= o[1] == a;
        if (lane == 0) w.list[n] = a;
        ++n;
    }
    const unsigned same = __match_any_sync(0xffffffffu, o[1]);
    first = __ballot_sync(0xffffffffu, __ffs(same) - 1 == lane && o[1] >= 0 && !known);
    for (unsigned left = first; left; left &= left - 1) {
        const int a = __shfl_sync(0xffffffffu, o[1], __ffs(left) - 1);
        if (lane == 0) w.list[n] = a;
        ++n;
    }
    if (lane == 0) w.count = n;
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---- T = A x --------------------------------------------------------------------------------------------------------------------
// grid (windows, slots, splits).  MT tiles of 16 rows per window; a warp takes tile warp % MT and every (8 / MT)th step of 32 k.  RT: most tiles of 8
// ranks.  A step's element order: lane t of a quad holds k = 8t .. 8t+7 of the 32, of rows and of ranks alike.
template <int MT, int RT>
__global__ void __launch_bounds__(kShrinkThreads) lora_shrink_kernel(LoraCall c) {
    constexpr int kSub = kShrinkWarps / MT;
    extern __shared__ float part[];     // [kSub - 1][MT * 16][r]
    __shared__ Window win;
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tile = warp % MT, sub = warp / MT, row0 = blockIdx.x * MT * 16;
    const int64_t k0 = (int64_t)blockIdx.z * c.split_k, k1 = min(c.K, k0 + c.split_k);
    const int ranks = c.r / 8;
    load_window(win, c, row0, MT * 16);
    __syncthreads();
    bool waited = false;
    for (int at = blockIdx.y; at < win.count; at += c.slots) {
        const int adapter = win.list[at];
        const uint16_t *wa = c.a + (int64_t)adapter * c.r * c.K;
        const int m0 = tile * 16 + g, m1 = m0 + 8;
        const bool own0 = win.owner[m0] == adapter, own1 = win.owner[m1] == adapter;
        const bool any = __any_sync(0xffffffffu, own0 || own1);
        const size_t a_bytes = (size_t)c.L * c.r * c.K * 2, x_bytes = (size_t)c.M * c.K * 2;
        float acc[RT][4];
#pragma unroll
        for (int n = 0; n < RT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
        if (any) {
            for (int64_t k = k0 + 32 * sub; k < k1; k += 32 * kSub) {
                uint4 w[RT];
#pragma unroll
                for (int n = 0; n < RT; ++n)
                    if (n < ranks) w[n] = __ldg(reinterpret_cast<const uint4 *>(MXQ_AT(wa + (int64_t)(8 * n + g) * c.K + k + 8 * t, 16, c.a, a_bytes)));
                if (!waited) {           // (the adapters' first step is on its way before the previous kernel has ended)
                    pdl_wait();
                    waited = true;
                }
                uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
                if (own0) x0 = ld_dep_u4(MXQ_AT(c.x + (int64_t)(row0 + m0) * c.K + k + 8 * t, 16, c.x, x_bytes));
                if (own1) x1 = ld_dep_u4(MXQ_AT(c.x + (int64_t)(row0 + m1) * c.K + k + 8 * t, 16, c.x, x_bytes));
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    if (n >= ranks) break;
                    mma_bf16(acc[n], x0.x, x1.x, x0.y, x1.y, w[n].x, w[n].y);
                    mma_bf16(acc[n], x0.z, x1.z, x0.w, x1.w, w[n].z, w[n].w);
                }
            }
        }
        if (!waited) pdl_wait(), waited = true;
        // the warps' parts of K, added in order
        if (sub > 0 && any) {
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                if (n >= ranks) break;
                float *p = part + ((int64_t)(sub - 1) * MT * 16 + m0) * c.r + 8 * n + 2 * t;
                p[0] = acc[n][0], p[1] = acc[n][1];
                p[8 * c.r] = acc[n][2], p[8 * c.r + 1] = acc[n][3];
            }
        }
        __syncthreads();
        if (sub == 0 && any) {
            const size_t t_bytes = (size_t)c.splits * c.M * c.r * 4;
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                if (n >= ranks) break;
                for (int u = 0; u < kSub - 1; ++u) {
                    const float *p = part + ((int64_t)u * MT * 16 + m0) * c.r + 8 * n + 2 * t;
                    acc[n][0] += p[0], acc[n][1] += p[1], acc[n][2] += p[8 * c.r], acc[n][3] += p[8 * c.r + 1];
                }
                float *out = c.t + ((int64_t)blockIdx.z * c.M + row0 + m0) * c.r + 8 * n + 2 * t;
                if (own0) *reinterpret_cast<float2 *>(MXQ_AT(out, 8, c.t, t_bytes)) = make_float2(acc[n][0], acc[n][1]);
                if (own1) *reinterpret_cast<float2 *>(MXQ_AT(out + 8 * (int64_t)c.r, 8, c.t, t_bytes)) = make_float2(acc[n][2], acc[n][3]);
            }
        }
        __syncthreads();
    }
    if (!waited) pdl_wait();
}

// ---- base + B T -------------------------------------------------------------------------------------------------------------------
// grid (columns / (32 * warps), slots, windows); a warp takes 32 columns.  Tile i of 8 columns holds, in the product's order, columns
// 8t + 2i and 8t + 2i + 1 for t = 0..3, so that a lane ends up with eight consecutive columns of its rows.  KT: most steps of 16 ranks.
__device__ __forceinline__ void load_columns(float (&f)[8], const uint8_t *base, bool f32, int64_t at, int there, bool vec, int64_t n) {
    if (vec) {
        const uint8_t *p = MXQ_AT(base + at * (f32 ? 4 : 2), f32 ? 32 : 16, base, n * (f32 ? 4 : 2));
        if (f32) {
            const uint4 u = ld_dep_u4(p), v = ld_dep_u4(p + 16);
            const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
        } else {
            unpack_bf16(f, ld_dep_u4(p));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = 0.f;
        if (e < there) f[e] = f32 ? ld_dep_f32(MXQ_AT(base + (at + e) * 4, 4, base, n * 4)) : ld_dep_bf16(MXQ_AT(base + (at + e) * 2, 2, base, n * 2));
    }
}
__device__ __forceinline__ void store_columns(const float (&f)[8], uint8_t *y, bool f32, int64_t at, int there, bool vec, int64_t n) {
    if (vec) {
        uint8_t *p = MXQ_AT(y + at * (f32 ? 4 : 2), f32 ? 32 : 16, y, n * (f32 ? 4 : 2));
        if (f32) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4 *>(p) = pack_bf16(f);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e >= there) continue;
        if (f32) *reinterpret_cast<float *>(MXQ_AT(y + (at + e) * 4, 4, y, n * 4)) = f[e];
        else *reinterpret_cast<__nv_bfloat16 *>(MXQ_AT(y + (at + e) * 2, 2, y, n * 2)) = __float2bfloat16_rn(f[e]);
    }
}

// eight bytes of B: ranks 4t .. 4t+3 of step s of a column; zero where there is no such column or rank
__device__ __forceinline__ uint2 load_b(const LoraCall &c, int adapter, int64_t col, int s, int t) {
    if (col >= c.N || 16 * s + 4 * t >= c.r) return make_uint2(0, 0);
    return __ldg(reinterpret_cast<const uint2 *>(MXQ_AT(c.b + ((int64_t)adapter * c.N + col) * c.r + 16 * s + 4 * t, 8, c.b, (size_t)c.L * c.N * c.r * 2)));
}

template <int MT, int KT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) lora_expand_kernel(LoraCall c) {
    extern __shared__ uint4 frag[];      // [MT][steps][parts][32 lanes]: T as the product's first operand
    __shared__ Window win;
    constexpr bool kAhead = MT == 1 && KT <= 4;   // B waits in registers for T
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int row0 = blockIdx.z * MT * 16;
    const int64_t col0 = ((int64_t)blockIdx.x * WARPS + warp) * 32;
    const int steps = (c.r + 15) / 16;
    load_window(win, c, row0, MT * 16);
    __syncthreads();
    uint2 w[kAhead ? KT : 1][4];
    if constexpr (kAhead) {
        if ((int)blockIdx.y < win.count) {
            const int adapter = win.list[blockIdx.y];
#pragma unroll
            for (int s = 0; s < KT; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s < steps) w[s][i] = load_b(c, adapter, col0 + 8 * (g >> 1) + 2 * i + (g & 1), s, t);
        }
    }
    pdl_wait();
    if ((int)blockIdx.y >= win.count && blockIdx.y != 0) return;

    // T of the window's rows: sum over the splits, times the adapter's scale, in two BF16 parts, in the order of the fragments
    const size_t t_bytes = (size_t)c.splits * c.M * c.r * 4;
    for (int n = threadIdx.x; n < MT * 16 * steps * 8; n += 32 * WARPS) {
        const int pair = n % (steps * 8), m = n / (steps * 8);           // ranks 2 * pair, 2 * pair + 1 of row m
        float v[2] = {0.f, 0.f};
        const int adapter = win.owner[m];
        if (adapter >= 0 && 2 * pair < c.r) {
            const float *p = c.t + (int64_t)(row0 + m) * c.r + 2 * pair;
            for (int u = 0; u < c.splits; ++u) {
                const float *q = MXQ_AT(p + (int64_t)u * c.M * c.r, 8, c.t, t_bytes);
                v[0] += ld_dep_f32(q), v[1] += ld_dep_f32(q + 1);
            }
            const float s = c.scale ? __ldg(MXQ_AT(c.scale + adapter, 4, c.scale, (size_t)c.L * 4)) : 1.f;
            v[0] *= s, v[1] *= s;
        }
        // rank 16 s + 4 t + 2 e + {0, 1} of row 16 mt + g + 8 h: register 2 e + h of lane 4 g + t
        const int s = pair / 8, tt = pair % 8 / 2, e = pair & 1, mt = m / 16, row = m % 16;
        uint32_t *dst = reinterpret_cast<uint32_t *>(frag + (mt * steps + s) * c.parts * 32 + 4 * (row & 7) + tt) + 2 * e + (row >> 3);
        for (int u = 0; u < c.parts; ++u) {
            const __nv_bfloat162 part = __floats2bfloat162_rn(v[0], v[1]);
            dst[u * 128] = *reinterpret_cast<const uint32_t *>(&part);
            const float2 f = __bfloat1622float2(part);
            v[0] = isfinite(f.x) ? v[0] - f.x : 0.f, v[1] = isfinite(f.y) ? v[1] - f.y : 0.f;    // (an infinite part leaves nothing)
        }
    }
    __syncthreads();
    if (col0 >= c.N) return;

    const int64_t col = col0 + 8 * t, n = (int64_t)c.M * c.N;
    const int there = (int)max((int64_t)0, min((int64_t)8, c.N - col));
    const bool vec = c.N % 8 == 0;
    // rows without an adapter are copied (by the first slot, unless they are there already)
    if (blockIdx.y == 0 && c.base != c.y) {
        for (int m = g; m < MT * 16; m += 8) {
            if (win.owner[m] >= 0 || row0 + m >= c.M || there == 0) continue;
            const int64_t at = (int64_t)(row0 + m) * c.N + col;
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (c.base) load_columns(f, c.base, c.base_f32, at, there, vec, n);
            store_columns(f, c.y, c.y_f32, at, there, vec, n);
        }
    }
    for (int at = blockIdx.y; at < win.count; at += c.slots) {
        const int adapter = win.list[at];
        float acc[MT][4][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[mt][i][0] = acc[mt][i][1] = acc[mt][i][2] = acc[mt][i][3] = 0.f;
#pragma unroll(kAhead ? KT : 1)
        for (int s = 0; s < (kAhead ? KT : steps); ++s) {
            if (s >= steps) break;
            uint2 b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (kAhead && at == (int)blockIdx.y) b[i] = w[kAhead ? s : 0][i];
                else b[i] = load_b(c, adapter, col0 + 8 * (g >> 1) + 2 * i + (g & 1), s, t);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const bool own0 = win.owner[16 * mt + g] == adapter, own1 = win.owner[16 * mt + g + 8] == adapter;
                if (!__any_sync(0xffffffffu, own0 || own1)) continue;
                for (int p = 0; p < c.parts; ++p) {
                    const uint4 f = frag[((mt * steps + s) * c.parts + p) * 32 + lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i) mma_bf16(acc[mt][i], f.x, f.y, f.z, f.w, b[i].x, b[i].y);
                }
            }
        }
        // (rows of other adapters went through the product too; what they got is dropped here)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int m = 16 * mt + 8 * h + g;
                if (win.owner[m] != adapter || there == 0) continue;
                const int64_t to = (int64_t)(row0 + m) * c.N + col;
                float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (c.base) load_columns(f, c.base, c.base_f32, to, there, vec, n);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[2 * i] += acc[mt][i][2 * h], f[2 * i + 1] += acc[mt][i][2 * h + 1];
                store_columns(f, c.y, c.y_f32, to, there, vec, n);
            }
    }
}

MXQ_BOUNDS_TU(bounds_take_lora)

// ---- host ---------------------------------------------------------------------------------------------------------------

// windows of 64 rows for many rows (a window reads its adapters once), of 16 otherwise
static int window_tiles(int64_t M) { return M >= 512 ? 4 : 1; }

static void lora_plan(LoraCall &c) {
    const int mt = window_tiles(c.M);
    const int64_t windows = (c.M + 16 * mt - 1) / (16 * mt);
    c.slots = mt == 1 ? min(16, min(c.M, c.L)) : 1;
    // splits of K until every SM has two CTAs (of 8 warps), but at least one step of 32 per warp
    const int64_t step = 32 * (kShrinkWarps / mt), most = (c.K + step - 1) / step;
    int64_t want = (2 * (int64_t)sm_count() + windows * c.slots - 1) / (windows * c.slots);
    if (want > most) want = most;
    if (want > 32) want = 32;
    int64_t len = ((c.K + want - 1) / want + step - 1) / step * step;
    c.split_k = (int32_t)len;
    c.splits = (int32_t)((c.K + len - 1) / len);
}

static bool lora_shape_ok(int64_t M, int64_t N, int64_t K, int r, int L) {
    return M >= 1 && M <= MXQ_LORA_MAX_M && shape_ok(N, K) && N <= ((int64_t)1 << 31) && K <= ((int64_t)1 << 30) && r >= 8 && r <= 128 && r % 8 == 0 &&
           L >= 1 && L <= MXQ_LORA_MAX_ADAPTERS;
}

static int lora_check(const void *X, int64_t M, const mxq_lora_adapters *ad, const int32_t *ids, int64_t N, int64_t K, const void *Y, int y_dtype) {
    if (!X || !ad || !ad->A_bf16 || !ad->B_bf16 || !ids || !Y) return MXQ_ERR_NULL;
    if (!lora_shape_ok(M, N, K, ad->rank, ad->count)) return MXQ_ERR_SHAPE;
    if (y_dtype != MXQ_F32 && y_dtype != MXQ_BF16) return MXQ_ERR_DTYPE;
    const void *wide[] = {X, ad->A_bf16, ad->B_bf16, Y};
    for (const void *p : wide)
        if (!aligned16(p)) return MXQ_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(ids) & 3u) || (reinterpret_cast<uintptr_t>(ad->scale) & 3u)) return MXQ_ERR_ALIGN;
    return MXQ_OK;
}

static LoraCall lora_call(const void *X, int64_t M, const mxq_lora_adapters *ad, const int32_t *ids, int64_t N, int64_t K, void *workspace) {
    LoraCall c = {};
    c.x = (const uint16_t *)X, c.a = (const uint16_t *)ad->A_bf16, c.b = (const uint16_t *)ad->B_bf16, c.scale = ad->scale, c.ids = ids;
    c.t = (float *)workspace, c.N = N, c.K = K, c.M = (int32_t)M, c.r = ad->rank, c.L = ad->count;
    lora_plan(c);
    return c;
}

// (48 KB, less the kernels' static shared memory, need no leave)
static bool allow_smem(void (*kernel)(LoraCall), size_t smem) {
    if (smem <= 40 * 1024 || cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) == cudaSuccess) return true;
    (void)cudaGetLastError();
    return false;
}

template <int MT>
static int shrink_launch(const LoraCall &c, cudaStream_t stream) {
    const dim3 grid((unsigned)((c.M + 16 * MT - 1) / (16 * MT)), (unsigned)c.slots, (unsigned)c.splits);
    const size_t smem = (size_t)(kShrinkWarps / MT - 1) * MT * 16 * c.r * 4;
    void (*const kernel)(LoraCall) = c.r <= 16 ? lora_shrink_kernel<MT, 2> : c.r <= 32 ? lora_shrink_kernel<MT, 4> : c.r <= 64 ? lora_shrink_kernel<MT, 8> : lora_shrink_kernel<MT, 16>;
    if (!allow_smem(kernel, smem)) return MXQ_ERR_CUDA;
    return launch_pdl(kernel, grid, kShrinkThreads, smem, stream, c);
}

template <int MT, int WARPS>
static int expand_launch(const LoraCall &c, cudaStream_t stream) {
    const dim3 grid((unsigned)((c.N + 32 * WARPS - 1) / (32 * WARPS)), (unsigned)c.slots, (unsigned)((c.M + 16 * MT - 1) / (16 * MT)));
    const size_t smem = (size_t)MT * ((c.r + 15) / 16) * c.parts * 32 * 16;
    void (*const kernel)(LoraCall) = c.r <= 16 ? lora_expand_kernel<MT, 1, WARPS> : c.r <= 32 ? lora_expand_kernel<MT, 2, WARPS> : c.r <= 64 ? lora_expand_kernel<MT, 4, WARPS> : lora_expand_kernel<MT, 8, WARPS>;
    if (!allow_smem(kernel, smem)) return MXQ_ERR_CUDA;
    return launch_pdl(kernel, grid, 32 * WARPS, smem, stream, c);
}

static int lora_shrink(const LoraCall &c, cudaStream_t stream) { return window_tiles(c.M) == 4 ? shrink_launch<4>(c, stream) : shrink_launch<1>(c, stream); }
static int lora_expand(LoraCall &c, const void *base, int base_dtype, void *Y, int y_dtype, cudaStream_t stream) {
    c.base = (const uint8_t *)base, c.y = (uint8_t *)Y, c.base_f32 = base_dtype == MXQ_F32, c.y_f32 = y_dtype == MXQ_F32, c.parts = c.y_f32 ? 3 : 2;
    return window_tiles(c.M) == 4 ? expand_launch<4, 8>(c, stream) : expand_launch<1, 4>(c, stream);
}

static size_t align256(size_t v) { return (v + 255u) & ~(size_t)255u; }

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

size_t mxq_lora_workspace_bytes(int64_t M, int64_t N, int64_t K, int rank, int adapters) {
    if (!mxq::lora_shape_ok(M, N, K, rank, adapters)) return 0;
    mxq::LoraCall c = {};
    c.M = (int32_t)M, c.N = N, c.K = K, c.r = rank, c.L = adapters;
    mxq::lora_plan(c);
    return (size_t)c.splits * (size_t)M * (size_t)rank * 4;
}

int mxq_lora(const void *X_bf16, int64_t M, const mxq_lora_adapters *adapters, const int32_t *ids, int64_t N, int64_t K, const void *base,
             void *Y, int y_dtype, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = mxq::lora_check(X_bf16, M, adapters, ids, N, K, Y, y_dtype);
    if (rc != MXQ_OK) return rc;
    if (!mxq::aligned16(base) || !mxq::aligned16(workspace)) return MXQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < mxq_lora_workspace_bytes(M, N, K, adapters->rank, adapters->count)) return MXQ_ERR_WORKSPACE;
    mxq::LoraCall c = mxq::lora_call(X_bf16, M, adapters, ids, N, K, workspace);
    rc = mxq::lora_shrink(c, (cudaStream_t)stream);
    return rc != MXQ_OK ? rc : mxq::lora_expand(c, base, y_dtype, Y, y_dtype, (cudaStream_t)stream);
}

// workspace: [T][FP32 sums of the shared layer, for a BF16 Y][mxq_linear's own]
size_t mxq_linear_lora_workspace_bytes(int M, int64_t N, int64_t K, int rank, int adapters) {
    if (M > MXQ_MAX_M) return 0;
    const size_t t = mxq_lora_workspace_bytes(M, N, K, rank, adapters);
    return t == 0 ? 0 : mxq::align256(t) + mxq::align256((size_t)M * (size_t)N * 4u) + mxq::align256(mxq_linear_workspace_bytes(M, N, K));
}

int mxq_linear_lora(const void *X_bf16, int M, const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t K, const mxq_lora_adapters *adapters,
                    const int32_t *ids, void *Y, int y_dtype, void *workspace, size_t workspace_bytes, void *stream) {
    if (!codes || !scales) return MXQ_ERR_NULL;
    if (M > MXQ_MAX_M) return MXQ_ERR_SHAPE;
    int rc = mxq::lora_check(X_bf16, M, adapters, ids, N, K, Y, y_dtype);
    if (rc != MXQ_OK) return rc;
    if (!mxq::aligned16(codes) || !mxq::aligned16(scales) || !mxq::aligned16(workspace)) return MXQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < mxq_linear_lora_workspace_bytes(M, N, K, adapters->rank, adapters->count)) return MXQ_ERR_WORKSPACE;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const size_t t_bytes = mxq::align256(mxq_lora_workspace_bytes(M, N, K, adapters->rank, adapters->count)), sums = mxq::align256((size_t)M * (size_t)N * 4u);
    float *base = y_dtype == MXQ_F32 ? static_cast<float *>(Y) : reinterpret_cast<float *>(ws + t_bytes);
    // T first: the layer's weight stream starts while it is computed, and B is on its way while the layer ends
    mxq::LoraCall c = mxq::lora_call(X_bf16, M, adapters, ids, N, K, workspace);
    rc = mxq::lora_shrink(c, (cudaStream_t)stream);
    if (rc != MXQ_OK) return rc;
    rc = mxq_linear(X_bf16, M, codes, scales, N, K, base, MXQ_F32, ws + t_bytes + sums, mxq::align256(mxq_linear_workspace_bytes(M, N, K)), stream);
    if (rc != MXQ_OK) return rc;
    return mxq::lora_expand(c, base, MXQ_F32, Y, y_dtype, (cudaStream_t)stream);
}

#pragma GCC visibility pop
}  // extern "C"
