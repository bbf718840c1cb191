// mxq_kv_attention: softmax(scale * q . K^T) . V over the pages of a 4-bit cache.
//
// Plain form: one warp per (sequence, token row, query head) walks the tokens with a running maximum and sum in FP32; a lane
// decodes D / 32 consecutive elements of every K and V row.
#include <math.h>

#include "mxq_kv.cuh"

namespace mxq {

struct KvQuery {
    const uint16_t *q;       // [B][M][heads][D], token rows q_stride elements apart
    int64_t q_stride;
    const uint64_t *tree;    // [B][M] or nullptr
    uint16_t *o;             // [B][M][heads][D]
    float *lse;              // [B][M][heads] or nullptr
    int32_t heads, group;    // query heads, query heads per kv head
    float scale_log2;        // scale * log2(e)
};

template <int D>
__global__ void __launch_bounds__(128) kv_attention_plain_kernel(KvView c, KvSeqs s, KvQuery a) {
    using T = KvTile<D>;
    constexpr int kE = D / 32, kBytes = kE / 2;   // elements and code bytes of a row per lane
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int64_t row = unit / a.heads;
    const int hq = (int)(unit - row * a.heads), hk = hq / a.group;
    const int b = (int)(row / s.m), i = (int)(row - (int64_t)b * s.m);
    if (b >= s.B) return;
    pdl_wait();
    const int len = s.len(b), rows = s.nrows(b), base = len - rows;
    const int e0 = lane * kE, j = e0 / 32, nat = lane * kBytes - 16 * j;   // natural byte within the block
    float q[kE], o[kE], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = 0.f, q[e] = ld_dep_bf16(a.q + row * a.q_stride + (int64_t)hq * D + e0 + e);
    const uint64_t tree = a.tree != nullptr && i < rows ? a.tree[row] : 0;
    for (int t = 0; t < (i < rows ? len : 0); ++t) {
        const int d = t - base;
        if (a.tree != nullptr ? (d >= 0 && !((tree >> d) & 1)) : d > i) continue;
        const int page = s.page(b, t >> c.page_shift);
        if (!kv_page_ok(c, page)) continue;
        const uint8_t *tile = kv_tile<D>(c, page, t & ((1 << c.page_shift) - 1), hk);
        const int ts = t & 31;
        float kv[2][kE];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float sc = e8m0_to_float(__ldcg(tile + (w ? T::vs(ts, j) : T::kKs + ts * T::kNb + j)));
#pragma unroll
            for (int y = 0; y < kBytes; ++y) {
                const int n = nat + y, p = w ? (n / 2) * 2 * T::kNb + 2 * j + n % 2 : (n / 4) * 4 * T::kNb + 4 * j + n % 4;
                const float2 f = __half22float2(e2m1x2_to_half2(__ldcg(tile + (w ? T::kV : 0) + ts * T::kRow + p)));
                kv[w][2 * y] = f.x * sc, kv[w][2 * y + 1] = f.y * sc;
            }
        }
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < kE; ++e) dot += q[e] * kv[0][e];
        const float x = warp_sum(dot) * a.scale_log2;
        const float top = fmaxf(m, x), use = top == -INFINITY ? 0.f : top;
        const float alpha = exp2f(m - use), p = exp2f(x - use);
        l = l * alpha + p;
#pragma unroll
        for (int e = 0; e < kE; ++e) o[e] = o[e] * alpha + p * kv[1][e];
        m = top;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        const __nv_bfloat16 r = __float2bfloat16(o[e] * inv);
        a.o[(row * a.heads + hq) * D + e0 + e] = *reinterpret_cast<const uint16_t *>(&r);
    }
    if (lane == 0 && a.lse != nullptr) a.lse[row * a.heads + hq] = (m == -INFINITY ? 0.f : m * 0.69314718f) + logf(l);
}

MXQ_BOUNDS_TU(bounds_take_kv_attention)

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

size_t mxq_kv_attention_workspace_bytes(int B, int M, int q_heads, int kv_heads, int head_dim) {
    if (B < 1 || B > MXQ_KV_MAX_SEQS || M < 1 || kv_heads < 1 || kv_heads > MXQ_KV_MAX_HEADS || q_heads < kv_heads || q_heads % kv_heads ||
        mxq_kv_page_bytes(kv_heads, head_dim, 32) == 0)
        return 0;
    return 4096;
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
    const mxq::KvQuery a = {(const uint16_t *)Q_bf16, q_stride, tree, (uint16_t *)O_bf16, lse, q_heads, q_heads / cache->kv_heads,
                            scale * 1.44269504f};
    const mxq::KvSeqs s = mxq::kv_seqs(cache, B, M, tables, W, lens, rows);
    const int64_t units = (int64_t)B * M * q_heads;
    return mxq::kv_launch(cache->head_dim == 128 ? mxq::kv_attention_plain_kernel<128> : mxq::kv_attention_plain_kernel<64>,
                          dim3((unsigned)((units + 3) / 4)), 128, 0, (cudaStream_t)stream, mxq::kv_view(cache, layer), s, a);
}

#pragma GCC visibility pop
}  // extern "C"
