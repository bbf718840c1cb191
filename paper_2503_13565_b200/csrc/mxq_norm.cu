// mxq_rmsnorm: root-mean-square norm of the residual stream with the residual's addition, in BF16 for the next projection and / or
// in 8 bits (MXFP8: E4M3 elements, one E8M0 scale per 32), and mxq_dequantize_mxfp8, the inverse of the cast.
//
//     h = x + residual,   y = h / sqrt(mean(h^2) + eps) * w
//
// A stream: every input is read once and every output written once; a row stays in the registers of one CTA between the sum of its
// squares and its scaling.  Measured in a replayed graph (BF16 stream with the residual read and written, BF16 result): 8000 rows of 4096 41.7 us,
// 6.3 TB/s = 96 % of the copy rate; 8191 rows of 8192 88.5 us (93 %), with the pair beside it 108 us (86 %: the cast's instructions, 61 % of the
// issue slots, and two CTAs per SM that meet at a barrier each; 104 without the look for rows in other units); one row of 4096 1.5 us, the
// launch's own time.  All of it is FP32; what is rounded is what is stored (h and y to BF16 where that is their type, y to E4M3).  The norm is that of
// the unrounded h.
#include "mxq_device.cuh"
#include "mxq_host.h"

namespace mxq {

constexpr int kNormMaxThreads = 1024;

struct NormCall {
    const uint8_t *x, *residual, *weight;
    uint8_t *sum;            // residual_out or nullptr
    uint16_t *y;             // BF16 or nullptr
    uint8_t *codes, *scales; // the pair or nullptr
    int64_t x_stride;        // elements
    int64_t rows;
    int32_t K;
    int32_t w_f32;
    float eps;
};

// eight elements of a row that the previous kernel may have written; n elements from `base` on belong to the array
template <bool F32>
__device__ __forceinline__ void load8(float (&f)[8], const uint8_t *base, int64_t at, int64_t n) {
    const uint8_t *p = MXQ_AT(base + at * (F32 ? 4 : 2), F32 ? 32 : 16, base, n * (F32 ? 4 : 2));
    if constexpr (F32) {
        const uint4 a = ld_dep_u4(p), b = ld_dep_u4(p + 16);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
    } else {
        unpack_bf16(f, ld_dep_u4(p));
    }
}
template <bool F32>
__device__ __forceinline__ void store8(const float (&f)[8], uint8_t *base, int64_t at, int64_t n) {
    uint8_t *p = MXQ_AT(base + at * (F32 ? 4 : 2), F32 ? 32 : 16, base, n * (F32 ? 4 : 2));
    if constexpr (F32) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        *reinterpret_cast<uint4 *>(p) = pack_bf16(f);
    }
}

// two FP32 -> two E4M3 codes, `lo` in the low byte: round to nearest even, magnitudes above 448 clamp to 448
__device__ __forceinline__ uint32_t float2_to_e4m3x2(float lo, float hi) {
    unsigned short out;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(out) : "f"(hi), "f"(lo));
    return out;
}

__device__ __forceinline__ void load_weight(float (&w)[8], const NormCall &c, int ch) {
    if (c.w_f32) {
        const float4 *p = reinterpret_cast<const float4 *>(MXQ_AT(c.weight + (int64_t)ch * 32, 32, c.weight, (int64_t)c.K * 4));
        const float4 a = __ldg(p), b = __ldg(p + 1);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    } else {
        unpack_bf16(w, __ldg(reinterpret_cast<const uint4 *>(MXQ_AT(c.weight + (int64_t)ch * 16, 16, c.weight, (int64_t)c.K * 2))));
    }
}

// One CTA per row.  Lane t takes chunks (8 elements) t, t + threads, ...: four neighbouring lanes hold an MX block.
// R: 0 no residual, 1 BF16, 2 FP32.
template <bool XF32, int R, int CHUNKS>
__global__ void __launch_bounds__(kNormMaxThreads) rmsnorm_kernel(NormCall c) {
    pdl_trigger();
    const int chunks = c.K / 8, threads = (int)blockDim.x;
    const int64_t row = blockIdx.x;
    constexpr bool kAhead = CHUNKS == 1;   // (four chunks of both would not fit the registers of 1024 threads)
    float w[CHUNKS][8], h[CHUNKS][8];
    if constexpr (kAhead) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j)   // weights: not written while the library runs, so ahead of the wait
            if ((int)threadIdx.x + j * threads < chunks) load_weight(w[j], c, (int)threadIdx.x + j * threads);
    }
    pdl_wait();
    const int64_t x_n = (c.rows - 1) * c.x_stride + c.K, n = c.rows * c.K;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        const int ch = threadIdx.x + j * threads;
        if (ch < chunks) load8<XF32>(h[j], c.x, row * c.x_stride + ch * 8, x_n);
    }
    if constexpr (R != 0) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int ch = threadIdx.x + j * threads;
            if (ch >= chunks) continue;
            float r[8];
            load8<R == 2>(r, c.residual, row * c.K + ch * 8, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] += r[i];
        }
    }
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        const int ch = threadIdx.x + j * threads;
        if (ch >= chunks) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) sq = fmaf(h[j][i], h[j][i], sq);
        if constexpr (R != 0)
            if (c.sum) store8<R == 2>(h[j], c.sum, row * c.K + ch * 8, n);
    }
    __shared__ float part[kNormMaxThreads / 32];
    sq = warp_sum(sq);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sq;
    __syncthreads();
    const int warps = threads >> 5;
    sq = warp_sum((threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0.f);
    float mean = sq / (float)c.K + c.eps;
    // The rare row (the same for the whole CTA) whose squares overflow, or vanish beside an eps that does not cover them: once more, with h and
    // eps in units of the power of two at the larger of max |h| and sqrt(eps).  (From 2^-100 on what a sum loses below FP32's least is 2^-35 of it.)
    if (sq > 3.402823466e38f || (sq < 0x1p-100f && c.eps < 0x1p-100f)) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int ch = threadIdx.x + j * threads;
            if (ch >= chunks) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(h[j][i]) & 0x7FFFFFFFu);
        }
        top = __reduce_max_sync(0xffffffffu, top);
        __syncthreads();                     // (the sums have been read)
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = __uint_as_float(top);
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < warps ? __float_as_uint(part[threadIdx.x & 31]) : 0u);
        const uint32_t unit = max(top, __float_as_uint(sqrtf(c.eps))) >> 23;
        if (unit != 0xFFu) {                 // (a row with an Inf stays as it is)
            // 2^(127 - unit), from the subnormal 2^-127 to 2^126
            const float to = unit >= 254u ? 0x1p-127f : __uint_as_float((254u - max(unit, 1u)) << 23);
            sq = 0.f;
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j) {
                const int ch = threadIdx.x + j * threads;
                if (ch >= chunks) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) h[j][i] *= to, sq = fmaf(h[j][i], h[j][i], sq);
            }
            sq = warp_sum(sq);
            __syncthreads();
            if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sq;
            __syncthreads();
            mean = warp_sum((threadIdx.x & 31) < warps ? part[threadIdx.x & 31] : 0.f) / (float)c.K + c.eps * to * to;
        }
    }
    const float scale = 1.0f / sqrtf(mean);
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        const int ch = threadIdx.x + j * threads;
        if (ch >= chunks) continue;          // (K is a multiple of 32: the four lanes of a block leave together)
        if constexpr (!kAhead) load_weight(w[j], c, ch);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[j][i] = h[j][i] * scale * w[j][i];
        if (c.y) store8<false>(h[j], reinterpret_cast<uint8_t *>(c.y), row * c.K + ch * 8, n);
        if (c.codes) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(h[j][i]) & 0x7FFFFFFFu);
            const uint32_t quad = 0xFu << (threadIdx.x & 28);
            top = max(top, __shfl_xor_sync(quad, top, 1));
            top = max(top, __shfl_xor_sync(quad, top, 2));
            // scale 2^(floor(log2 max) - 8), at least 2^-127 (256 = 2^8 is the largest power of two of E4M3)
            const uint32_t e = top >> 23, byte = e == 0xFFu ? 0xFFu : e > 8u ? e - 8u : 0u;
            const float inv = __uint_as_float((254u - byte) << 23);
            uint32_t lo = 0, hi = 0;
            if (byte != 0xFFu) {
                lo = float2_to_e4m3x2(h[j][0] * inv, h[j][1] * inv) | float2_to_e4m3x2(h[j][2] * inv, h[j][3] * inv) << 16;
                hi = float2_to_e4m3x2(h[j][4] * inv, h[j][5] * inv) | float2_to_e4m3x2(h[j][6] * inv, h[j][7] * inv) << 16;
            }
            *reinterpret_cast<uint2 *>(MXQ_AT(c.codes + row * c.K + ch * 8, 8, c.codes, n)) = make_uint2(lo, hi);
            if ((ch & 3) == 0) *MXQ_AT(c.scales + row * (c.K / 32) + ch / 4, 1, c.scales, n / 32) = (uint8_t)byte;
        }
    }
}

// one lane per 16 codes
template <bool F32>
__global__ void __launch_bounds__(256) dequantize_mxfp8_kernel(const uint8_t *codes, const uint8_t *scales, int64_t n, uint8_t *out) {
    pdl_trigger();
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16;
    pdl_wait();
    if (at >= n) return;
    const uint4 q = ld_dep_u4(MXQ_AT(codes + at, 16, codes, n));
    unsigned short byte;
    asm volatile("ld.global.cg.u8 %0, [%1];" : "=h"(byte) : "l"(MXQ_AT(scales + at / 32, 1, scales, n / 32)) : "memory");
    const float s = e8m0_to_float(byte);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = (w[2 * half + i / 2] >> (16 * (i & 1))) & 0xFFFFu;
            uint32_t h2;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((unsigned short)pair));
            const float2 v = __half22float2(*reinterpret_cast<__half2 *>(&h2));
            f[2 * i] = v.x * s, f[2 * i + 1] = v.y * s;
        }
        store8<F32>(f, out, at + 8 * half, n);
    }
}

MXQ_BOUNDS_TU(bounds_take_norm)

// ---- host ---------------------------------------------------------------------------------------------------------------

template <bool XF32, int R>
static int norm_launch(const NormCall &c, int per, unsigned threads, cudaStream_t stream) {
    if (per == 1) return launch_pdl(rmsnorm_kernel<XF32, R, 1>, dim3((unsigned)c.rows), threads, 0, stream, c);
    return launch_pdl(rmsnorm_kernel<XF32, R, 4>, dim3((unsigned)c.rows), threads, 0, stream, c);
}

static bool dtype_ok(int d) { return d == MXQ_F32 || d == MXQ_BF16; }

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

int mxq_rmsnorm(const void *X, int x_dtype, int64_t x_stride, const void *residual, int r_dtype, void *residual_out, const void *weight,
                int w_dtype, float eps, int64_t M, int64_t K, void *Y_bf16, uint8_t *codes, uint8_t *scales, void *stream) {
    if (!X || !weight || (!Y_bf16 && !codes) || !codes != !scales || (residual_out && !residual)) return MXQ_ERR_NULL;
    if (M < 1 || M > 0x7FFFFFFF || K < 32 || K % 32 || K > MXQ_MAX_NORM_K || x_stride < K || x_stride > ((int64_t)1 << 40) || !(eps >= 0.f) ||
        !(eps < INFINITY))
        return MXQ_ERR_SHAPE;
    if (!mxq::dtype_ok(x_dtype) || !mxq::dtype_ok(w_dtype) || (residual && !mxq::dtype_ok(r_dtype))) return MXQ_ERR_DTYPE;
    const void *all[] = {X, residual, residual_out, weight, Y_bf16, codes, scales};
    for (const void *p : all)
        if (!mxq::aligned16(p)) return MXQ_ERR_ALIGN;
    if (x_stride % (x_dtype == MXQ_F32 ? 4 : 8)) return MXQ_ERR_ALIGN;
    mxq::NormCall c;
    c.x = (const uint8_t *)X, c.residual = (const uint8_t *)residual, c.weight = (const uint8_t *)weight, c.sum = (uint8_t *)residual_out;
    c.y = (uint16_t *)Y_bf16, c.codes = codes, c.scales = scales;
    c.x_stride = x_stride, c.rows = M, c.K = (int32_t)K, c.w_f32 = w_dtype == MXQ_F32, c.eps = eps;
    const int chunks = (int)(K / 8);
    // One chunk per lane as long as a CTA has lanes enough (8191 rows of 8192: 87 us; two chunks in half the lanes 114, four 101), else four
    // (4000 rows of 16384: 103 us; two 120).
    const int per = chunks <= mxq::kNormMaxThreads ? 1 : 4;
    const unsigned threads = (unsigned)(((chunks + per - 1) / per + 31) / 32 * 32);
    cudaStream_t st = (cudaStream_t)stream;
    const int r = !residual ? 0 : r_dtype == MXQ_F32 ? 2 : 1;
    if (x_dtype == MXQ_F32)
        return r == 0 ? mxq::norm_launch<true, 0>(c, per, threads, st) : r == 1 ? mxq::norm_launch<true, 1>(c, per, threads, st)
                                                                                 : mxq::norm_launch<true, 2>(c, per, threads, st);
    return r == 0 ? mxq::norm_launch<false, 0>(c, per, threads, st) : r == 1 ? mxq::norm_launch<false, 1>(c, per, threads, st)
                                                                              : mxq::norm_launch<false, 2>(c, per, threads, st);
}

int mxq_dequantize_mxfp8(const uint8_t *codes, const uint8_t *scales, int64_t N, int64_t K, void *out, int out_dtype, void *stream) {
    if (!codes || !scales || !out) return MXQ_ERR_NULL;
    if (!mxq::shape_ok(N, K) || K > ((int64_t)1 << 40) || N > ((int64_t)1 << 42) / K) return MXQ_ERR_SHAPE;
    if (!mxq::dtype_ok(out_dtype)) return MXQ_ERR_DTYPE;
    if (!mxq::aligned16(codes) || !mxq::aligned16(scales) || !mxq::aligned16(out)) return MXQ_ERR_ALIGN;
    const int64_t n = N * K, ctas = (n / 16 + 255) / 256;
    if (ctas > 0x7FFFFFFF) return MXQ_ERR_SHAPE;
    return mxq::launch_pdl(out_dtype == MXQ_F32 ? mxq::dequantize_mxfp8_kernel<true> : mxq::dequantize_mxfp8_kernel<false>, dim3((unsigned)ctas), 256, 0,
                           (cudaStream_t)stream, codes, scales, n, (uint8_t *)out);
}

#pragma GCC visibility pop
}  // extern "C"
