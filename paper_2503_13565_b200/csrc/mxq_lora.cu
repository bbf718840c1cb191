// mxq_lora: low-rank adapters of many requests at once, added to what a shared projection computed; mxq_linear_lora: the 4-bit
// layer and its adapters in one call.
//
//     Y[m] = base[m] + s[a] * B[a] (A[a] x[m]),   a = ids[m]   (A [r][K], B [N][r] BF16; no adapter: Y[m] = base[m])
//
// Two kernels: T = A x into the workspace (shrink), then base + B T (expand).  Both are bound by the adapters' bytes for a few token
// rows and by X, base and Y for many; the products are m16n8k16 mma.sync with the token rows as m, fed from global memory by 16- and 8-byte
// loads whose order along the contracted axis is the same for both operands (the sum does not mind the order): for few rows they are a hundredth
// of the time.  A prompt's T, a matrix product with one short side, takes the tensor memory path instead (lora_shrink_umma_kernel: 50 -> 41 us
// for the prompt below).
// T is FP32 and meets B as a sum of BF16 parts: three for an FP32 Y (all 24 bits), two for a BF16 Y (16 bits: what
// is lost is 2^-17 of each product, against the 2^-8 of Y's own rounding).
//
// A CTA takes a window of token rows and one adapter, or several one after the other: rows that have another one are left out (zero in the
// product, not stored).
// Measured in a replayed graph: one row, rank 16, beside 4096x4096: 10.1 us (the 4-bit layer alone 5.8); 16 rows of 13 adapters, rank 32,
// beside 11008x4096: 26 us (the layer alone 14; the shrink before it and the expansion behind it are a chain of dependent loads each);
// 64 rows of 32 adapters, rank 64, 11008x4096: 35 us; a prompt of 4095 rows of six adapters, rank 64, 4096x4096: 41 us (107 MB: 16 us at the
// copy rate), the expansion the most of it: it waits for base at 15 warps per SM, the legacy tensor pipe is 29 % busy.
#include <algorithm>

#include "mxq_device.cuh"
#include "mxq_host.h"
#include "mxq_tcgen05.cuh"
#include "mxq_tensor_map.h"

namespace mxq {

constexpr int kWindowMost = 32;

struct LoraCall {
    const uint16_t *x;       // [M][K]
    const uint16_t *a, *b;   // [L][r][K], [L][N][r]
    const float *scale;      // [L] or nullptr
    const int32_t *ids;      // [M]
    const uint8_t *base;     // [M][N] or nullptr (zero)
    uint8_t *y;              // [M][N]
    float *t;                // [splits][M][r]
    uint4 *frag;             // many rows: T as BF16 parts in the order of the product's first operand
    int64_t N, K;
    int32_t M, r, L;
    int32_t slots;           // CTAs of a window; slot s takes its adapters s, s + slots, ...
    int32_t splits, split_k; // shrink: CTAs along K, and how much of K each takes (a multiple of 32)
    int32_t base_f32, y_f32;
    int32_t parts;           // BF16 parts of T
    int32_t stages;          // shrink: steps of a warp's ring
    int32_t tiles;           // many rows: tiles of 16 rows per CTA of the expansion
    int32_t direct;          // many rows, K not split: the shrink writes the fragments itself
    int32_t *plan;           // segments of sorted rows (see lora_order_kernel), else nullptr
    int32_t lost_stage;      // test hook: this stage of X is waited for by the first window's first CTA but never requested
};

struct Window {
    int32_t owner[kWindowMost];   // adapter of every row, -1: none
    int32_t row[kWindowMost];     // the rows; -1: none
    int32_t list[kWindowMost];    // its distinct adapters in order of their first row
    int32_t count;
};

// 17 to 511 rows of many adapters, the batches of a server: rows sorted by adapter and cut into segments of up to 16 rows of one adapter, so that every
// adapter is read about once whatever the rows' order.  plan: [0 ..] first place of segment s and, behind the last, M; [kPlanAdapter ..] its
// adapter, -1: none; [kPlanOrder ..] row at every place; [kPlanCount] segments.
constexpr int kMostSorted = 512, kPlanAdapter = 1024, kPlanOrder = 2048, kPlanCount = 2560, kPlanBytes = 2561 * 4;
__global__ void __launch_bounds__(kMostSorted) lora_order_kernel(LoraCall c) {
    __shared__ uint32_t key[kMostSorted];
    __shared__ int32_t last[kMostSorted / 32], heads[kMostSorted / 32];
    const int i = threadIdx.x, warp = i >> 5, lane = i & 31;
    pdl_wait();              // (no early trigger: the shrink has nothing to do ahead of the plan)
    uint32_t mine = 0xFFFFFFFFu;
    if (i < c.M) {
        const int a = (int)ld_dep_u32(MXQ_AT(c.ids + i, 4, c.ids, (size_t)c.M * 4));
        mine = (a >= 0 && a < c.L ? (uint32_t)a : (uint32_t)MXQ_LORA_MAX_ADAPTERS) << 9 | i;
    }
    for (int size = 2; size <= kMostSorted; size <<= 1) {            // bitonic, over lanes where the partner is in the warp
        for (int step = size >> 1; step > 0; step >>= 1) {
            uint32_t other;
            if (step < 32) {
                other = __shfl_xor_sync(0xffffffffu, mine, step);
            } else {
                __syncthreads();
                key[i] = mine;
                __syncthreads();
                other = key[i ^ step];
            }
            mine = ((i & step) == 0) == ((i & size) == 0) ? min(mine, other) : max(mine, other);
        }
    }
    __syncthreads();
    key[i] = mine;
    __syncthreads();
    const bool head = i == 0 || (key[i - 1] >> 9) != (mine >> 9);
    int start = head ? i : 0;                                        // first place of the adapter's rows: the largest head so far
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, start, o);
        if (lane >= o) start = max(start, n);
    }
    if (lane == 31) last[warp] = start;
    __syncthreads();
    for (int u = 0; u < warp; ++u) start = max(start, last[u]);
    const bool cut = i < c.M && (i - start) % 16 == 0;
    const uint32_t cuts = __ballot_sync(0xffffffffu, cut);
    if (lane == 0) heads[warp] = __popc(cuts);
    __syncthreads();
    int before = __popc(cuts & ((1u << lane) - 1)), all = 0;
    for (int u = 0; u < kMostSorted / 32; ++u) {
        if (u < warp) before += heads[u];
        all += heads[u];
    }
    auto at = [&](int place) { return MXQ_AT(c.plan + place, 4, c.plan, kPlanBytes); };
    if (cut) *at(before) = i, *at(kPlanAdapter + before) = (mine >> 9) == MXQ_LORA_MAX_ADAPTERS ? -1 : (int32_t)(mine >> 9);
    if (i < c.M) *at(kPlanOrder + i) = (int32_t)(mine & (kMostSorted - 1));
    if (i == 0) *at(all) = c.M, *at(kPlanCount) = all;
}
// Segment s as a window of one adapter.  The plan is an earlier kernel's output, so this comes behind the wait; what is used as an index is
// held to the call's rows and adapters, as ids are.  (s < most_segments <= 543: all places lie inside the plan.)
__device__ __forceinline__ void load_segment(int32_t (&owner)[kWindowMost], int32_t (&row)[kWindowMost], int32_t &adapter, const LoraCall &c, int s) {
    auto at = [&](int place) { return (int)ld_dep_u32(MXQ_AT(c.plan + place, 4, c.plan, kPlanBytes)); };
    const int lane = threadIdx.x, count = at(kPlanCount), begin = at(s), end = at(s + 1), a = at(kPlanAdapter + s);      // (four loads at once)
    const bool there = s < count;
    const int first = there ? min(max(begin, 0), c.M) : 0, rows = there ? min(min(end, c.M) - first, 16) : 0;
    adapter = there && a < c.L ? max(a, -1) : -1;
    owner[lane] = lane < rows ? adapter : -1;
    row[lane] = lane < rows ? min(max(at(kPlanOrder + first + lane), 0), c.M - 1) : -1;
}

// the adapter of row m, -1: none, as there is none behind the last row (no branch: nothing waits for the load here)
__device__ __forceinline__ int load_id(const LoraCall &c, int m) {
    const int a = (int)ld_dep_u32(MXQ_AT(c.ids + min(m, c.M - 1), 4, c.ids, (size_t)c.M * 4));
    return m < c.M && a < c.L ? max(a, -1) : -1;
}
// Filled by warp 0; the caller synchronises.  ids are a step's data, which whatever ran before in the stream may have written: a window that is
// loaded ahead of the wait for the previous kernel is a guess, good for fetching weights early, and is compared with the ids behind the wait
// (wrong_window) before anything is made of it.  One row beside 4096 x 4096: 9.8 us, 11.6 with nothing done ahead of the wait.  A plan is only read
// behind it.
__device__ __forceinline__ void load_window(Window &w, const LoraCall &c, int row0, int rows) {
    if (threadIdx.x >= 32) return;
    const int lane = threadIdx.x;
    if (c.plan) {            // (windows are segments then)
        int adapter;
        load_segment(w.owner, w.row, adapter, c, row0 / rows);
        if (lane == 0) w.list[0] = adapter, w.count = adapter >= 0 ? 1 : 0;
        return;
    }
    int a = -1;
    if (lane < rows) a = load_id(c, row0 + lane);
    w.owner[lane] = a;
    w.row[lane] = lane < rows && row0 + lane < c.M ? row0 + lane : -1;
    const bool first = __ffs(__match_any_sync(0xffffffffu, a)) - 1 == lane && a >= 0;
    const unsigned firsts = __ballot_sync(0xffffffffu, first);
    if (first) w.list[__popc(firsts & ((1u << lane) - 1))] = a;
    if (lane == 0) w.count = __popc(firsts);
}

// A warp's look at the ids behind the wait: `id` loaded early, compared where the result is needed.  All warps of a CTA come to the same answer.
__device__ __forceinline__ int window_id(const LoraCall &c, int row0, int rows) { return load_id(c, row0 + min((int)(threadIdx.x & 31), rows - 1)); }
__device__ __forceinline__ bool wrong_window(const Window &w, int id, int rows) {
    return __any_sync(0xffffffffu, id != w.owner[min((int)(threadIdx.x & 31), rows - 1)]);
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---- T = A x --------------------------------------------------------------------------------------------------------------------
// grid (windows, slots, splits).  A window has MW tiles of 16 rows; a warp takes all of them and every WARPSth step of 32 k.  RT: most tiles of 8
// ranks.  A step's element order: lane t of a quad holds k = 8t .. 8t+7 of the 32, of rows and of ranks alike.
// Every lane copies its own 16-byte pieces of the next steps into a ring in shared memory (cp.async) and reads back what it copied: the ring
// holds `stages` steps per warp, no registers are spent on loads in flight, and no warp waits for another one.
__device__ __forceinline__ void copy16(uint32_t smem, const void *global, bool there) {      // zeros where there is nothing
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(global), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
constexpr int kMostStages = 4;
__device__ __forceinline__ void wait_oldest(int stages) {        // of `stages` groups
    if (stages == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Four ranks 4 q .. 4 q + 3 of a step of a row's T as BF16 parts in the order of the product's first operand, [steps][parts][32 lanes] of a 16-row tile.
__device__ __forceinline__ void put_parts(uint4 *tile_step, int row, int quarter, float (&v)[4], int parts) {
    // ranks 4 q + 2 e + {0, 1} of the step, row `row` of the tile: register 2 e + (row >> 3) of lane 4 (row & 7) + q
    uint32_t *dst = reinterpret_cast<uint32_t *>(tile_step + 4 * (row & 7) + quarter) + (row >> 3);
    for (int u = 0; u < parts; ++u) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const __nv_bfloat162 part = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
            dst[u * 128 + 2 * e] = *reinterpret_cast<const uint32_t *>(&part);
            const float2 f = __bfloat1622float2(part);       // (an infinite part leaves nothing)
            v[2 * e] = isfinite(f.x) ? v[2 * e] - f.x : 0.f, v[2 * e + 1] = isfinite(f.y) ? v[2 * e + 1] - f.y : 0.f;
        }
    }
}
__device__ __forceinline__ uint4 *fragment(const LoraCall &c, int tile, int step) {
    const int steps = (c.r + 15) / 16;
    return MXQ_AT(c.frag + ((int64_t)tile * steps + step) * c.parts * 32, c.parts * 512, c.frag, (size_t)((c.M + 15) / 16) * steps * c.parts * 512);
}

template <int MW, int WARPS, int RT>
__global__ void __launch_bounds__(32 * WARPS) lora_shrink_kernel(LoraCall c) {
    constexpr int kRows = 16 * MW;
    extern __shared__ uint4 ring[];     // [warps][stages][RT + 2 * MW][32 lanes]; then the warps' parts of T, [warps][kRows][r] floats
    __shared__ Window win;
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t k0 = (int64_t)blockIdx.z * c.split_k + 32 * warp, k1 = min(c.K, (int64_t)(blockIdx.z + 1) * c.split_k);
    constexpr int kPieces = RT + 2 * MW;          // (tiles of ranks that are not there are zeros)
    const int ranks = c.r / 8, steps = k0 < k1 ? (int)((k1 - k0 + 32 * WARPS - 1) / (32 * WARPS)) : 0;
    const int64_t stride = 16 * c.K;              // bytes from a row to the eighth after it
    uint4 *mine = ring + warp * c.stages * kPieces * 32 + lane;
    const uint32_t mine_address = shared_address(mine);
    const size_t a_bytes = (size_t)c.L * c.r * c.K * 2, x_bytes = (size_t)c.M * c.K * 2, t_bytes = (size_t)c.splits * c.M * c.r * 4;
    bool sure = c.plan != nullptr;
    if (sure) pdl_wait();
    load_window(win, c, blockIdx.x * kRows, kRows);      // this lane's rows: places g + 8 * j, j < 2 * MW
    __syncthreads();
    int id = -1;
    auto again = [&]() {
        __syncthreads();
        load_window(win, c, blockIdx.x * kRows, kRows);
        __syncthreads();
    };
    if (!sure && (int)blockIdx.y >= win.count) {
        pdl_wait();
        sure = true;
        if (wrong_window(win, window_id(c, blockIdx.x * kRows, kRows), kRows)) again();
    }
    for (int at = blockIdx.y; at < win.count;) {
        const int adapter = win.list[at];
        bool own[2 * MW];
#pragma unroll
        for (int j = 0; j < 2 * MW; ++j) own[j] = win.owner[g + 8 * j] == adapter;
        // byte addresses of this lane's pieces of the next step to be copied; a row that is not there is not read (its address is the array's own)
        const uint8_t *wa = reinterpret_cast<const uint8_t *>(c.a + ((int64_t)adapter * c.r + g) * c.K + k0 + 8 * t);
        const uint8_t *xa[2 * MW];
#pragma unroll
        for (int j = 0; j < 2 * MW; ++j) xa[j] = reinterpret_cast<const uint8_t *>(c.x + (own[j] ? (int64_t)win.row[g + 8 * j] * c.K + k0 + 8 * t : 0));
        auto copy_a = [&](int slot) {
            const uint32_t to = mine_address + slot * (kPieces * 512);
            const uint8_t *from = wa;
#pragma unroll
            for (int n = 0; n < RT; ++n, from += stride)
                copy16(to + n * 512, n < ranks ? MXQ_AT(from, 16, c.a, a_bytes) : reinterpret_cast<const uint8_t *>(c.a), n < ranks);
            wa += 64 * WARPS;
        };
        auto copy_x = [&](int slot) {
            const uint32_t to = mine_address + slot * (kPieces * 512) + RT * 512;
#pragma unroll
            for (int j = 0; j < 2 * MW; ++j) {
                copy16(to + j * 512, own[j] ? MXQ_AT(xa[j], 16, c.x, x_bytes) : xa[j], own[j]);
                if (own[j]) xa[j] += 64 * WARPS;
            }
        };
        // (the first adapter's first steps are on their way before the previous kernel has ended)
        for (int u = 0; u < c.stages && u < steps; ++u) copy_a(u);
        if (!sure) pdl_wait();
        for (int u = 0; u < c.stages; ++u) {
            if (u < steps) copy_x(u);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        if (!sure) id = window_id(c, blockIdx.x * kRows, kRows);
        float acc[MW][RT][4];
#pragma unroll
        for (int w = 0; w < MW; ++w)
#pragma unroll
            for (int n = 0; n < RT; ++n) acc[w][n][0] = acc[w][n][1] = acc[w][n][2] = acc[w][n][3] = 0.f;
        for (int step = 0, slot = 0; step < steps; ++step) {
            wait_oldest(c.stages);
            const uint4 *from = mine + slot * (kPieces * 32);
            uint4 x[2 * MW];
#pragma unroll
            for (int j = 0; j < 2 * MW; ++j) x[j] = from[(RT + j) * 32];
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                const uint4 v = from[n * 32];
#pragma unroll
                for (int w = 0; w < MW; ++w) {
                    mma_bf16(acc[w][n], x[2 * w].x, x[2 * w + 1].x, x[2 * w].y, x[2 * w + 1].y, v.x, v.y);
                    mma_bf16(acc[w][n], x[2 * w].z, x[2 * w + 1].z, x[2 * w].w, x[2 * w + 1].w, v.z, v.w);
                }
            }
            if (step + c.stages < steps) copy_a(slot), copy_x(slot);     // (this lane has read the slot)
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (++slot == c.stages) slot = 0;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (!sure) {
            sure = true;
            if (wrong_window(win, id, kRows)) {
                again();
                continue;
            }
        }
        // the warps' parts of K, added in order, four ranks of a row per thread; the ring is free for them now
        __syncthreads();
        float *part = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int w = 0; w < MW; ++w)
#pragma unroll
            for (int n = 0; n < RT; ++n) {
                if (n >= ranks) break;
                float *p = part + (warp * kRows + g + 16 * w) * c.r + 8 * n + 2 * t;
                *reinterpret_cast<float2 *>(p) = make_float2(acc[w][n][0], acc[w][n][1]);
                *reinterpret_cast<float2 *>(p + 8 * c.r) = make_float2(acc[w][n][2], acc[w][n][3]);
            }
        __syncthreads();
        const int quarters = (c.r + 15) / 16 * 4;     // (a last step of eight ranks is filled with zeros)
        for (int i = threadIdx.x; i < kRows * quarters; i += 32 * WARPS) {
            const int row = i / quarters, rank = 4 * (i - row * quarters);
            if (win.owner[row] != adapter) continue;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int u = 0; u < WARPS; ++u) {
                if (rank >= c.r) break;
                const float4 p = *reinterpret_cast<const float4 *>(part + (u * kRows + row) * c.r + rank);
                sum.x += p.x, sum.y += p.y, sum.z += p.z, sum.w += p.w;
            }
            if (c.direct) {                      // the whole sum: straight into the fragments
                const float scale = c.scale ? __ldg(MXQ_AT(c.scale + adapter, 4, c.scale, (size_t)c.L * 4)) : 1.f;
                float v[4] = {sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale};
                put_parts(fragment(c, win.row[row] / 16, rank / 16), win.row[row] % 16, rank % 16 / 4, v, c.parts);
            } else if (rank < c.r) {
                *reinterpret_cast<float4 *>(MXQ_AT(c.t + ((int64_t)blockIdx.z * c.M + win.row[row]) * c.r + rank, 16, c.t, t_bytes)) = sum;
            }
        }
        __syncthreads();
        at += c.slots;
    }
}

// T = A x of many rows on the tensor memory path (K a multiple of 64): a window of 128 token rows is the first operand of tcgen05.mma (BF16, FP32
// accumulator in tensor memory), the adapter's ranks the second; the copy engine brings 128 x 64 and ranks x 64 elements per stage, 128-byte swizzled,
// straight into the operands, so that neither registers nor shared-memory reads stand between memory and the product.  grid (windows, splits,
// slots: the CTAs that find no adapter come last); warp 0 multiplies, warp 1 copies, warps 2 to 5 take a row per thread from tensor memory to the partial sums.  ranks16: columns of the
// product (the ranks, up to a multiple of 16: what is behind an adapter's own is computed and dropped).  No early trigger: the kernel behind this
// one has nothing to do ahead of T, and none that holds tensor memory may settle here while a CTA still waits for its own.
constexpr int kUmmaRows = 128, kUmmaK = 64, kUmmaThreads = 192;
__device__ unsigned int g_lora_status = 0;     // sticky: a bounded wait gave up

__global__ void __launch_bounds__(kUmmaThreads)
lora_shrink_umma_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap amap, LoraCall c, int ring, int ranks16, int columns) {
    extern __shared__ uint8_t raw[];
    __shared__ int32_t owner[kUmmaRows], list[kUmmaRows], count, fail;
    __shared__ uint32_t holder;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row0 = blockIdx.x * kUmmaRows;
    const uint32_t stage = kUmmaRows * kUmmaK * 2 + ranks16 * kUmmaK * 2, base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t full0 = base + ring * stage, empty0 = full0 + ring * 8, done = empty0 + ring * 8;
    const int k0 = blockIdx.y * (c.split_k / kUmmaK), stages = (int)min((int64_t)c.split_k / kUmmaK, c.K / kUmmaK - k0);
    pdl_wait();              // (all wait here: the bounded waits below are for this kernel's own steps only)
    if (warp == 0) {         // the window's adapters, in ascending order
        uint32_t a[kUmmaRows / 32];
#pragma unroll
        for (int j = 0; j < kUmmaRows / 32; ++j) {
            const int m = row0 + 32 * j + lane;
            a[j] = (uint32_t)load_id(c, m);      // (-1 is the largest)
            owner[32 * j + lane] = (int32_t)a[j];
        }
        int n = 0;
        for (;; ++n) {
            uint32_t least = 0xFFFFFFFFu;
#pragma unroll
            for (int j = 0; j < kUmmaRows / 32; ++j) least = min(least, a[j]);
            least = __reduce_min_sync(0xffffffffu, least);
            if (least == 0xFFFFFFFFu) break;
            if (lane == 0) list[n] = (int32_t)least;
#pragma unroll
            for (int j = 0; j < kUmmaRows / 32; ++j)
                if (a[j] == least) a[j] = 0xFFFFFFFFu;
        }
        if (lane == 0) count = n;
    } else if (warp == 1) {
        for (int b = lane; b < 2 * ring + 1; b += 32) mbar_init(full0 + b * 8, 1u);
        if (lane == 0) {
            fail = 0;
            asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&amap) : "memory");
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if ((int)blockIdx.z >= count) return;
    const int first_stages = min(ring, stages);
    auto copy_a = [&](int step, int i, int adapter) {
        const uint32_t slot = (step + i) % ring;
        mbar_expect_tx(full0 + slot * 8, stage);
        tma_load_codes(base + slot * stage + kUmmaRows * kUmmaK * 2, &amap, (k0 + i) * kUmmaK, adapter * c.r, full0 + slot * 8);
    };
    auto copy_x = [&](int step, int i) {
        const uint32_t slot = (step + i) % ring;
#ifdef MXQ_DEBUG_BOUNDS
        if (k0 + i == c.lost_stage && blockIdx.x == 0 && blockIdx.z == 0) return;
#endif
        tma_load_codes(base + slot * stage, &xmap, (k0 + i) * kUmmaK, row0, full0 + slot * 8);
    };
    if (warp == 1 && lane == 0)      // the first adapter's first stages
        for (int u = 0; u < first_stages; ++u) copy_a(0, u, list[blockIdx.z]), copy_x(0, u);
    __syncwarp();
    if (warp == 0) {         // (behind the wait: the previous kernel's CTAs may still want columns of their own before it)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&holder)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&holder);
    volatile int32_t *failed = &fail;

    int step = 0;            // stages of all passes so far: the ring's state
    int issued = first_stages;       // warp 1: stages requested
    for (int at = blockIdx.z, pass = 0; at < count; at += c.slots, ++pass, step += stages) {
        const int adapter = list[at];
        const bool lost = *failed != 0;          // (an earlier pass gave up: the others give NaN at once)
        if (warp == 1) {
            for (int i = pass == 0 ? first_stages : 0; i < stages && !lost; ++i) {
                const int n = step + i;
                if (n >= ring && !mbar_wait_relaxed(empty0 + n % ring * 8, (n / ring - 1) & 1)) {
                    if (lane == 0) atomicOr(&g_lora_status, 1u), *failed = 1;
                    break;
                }
                if (lane == 0) copy_a(step, i, adapter), copy_x(step, i);
                issued = n + 1;
            }
        } else if (warp == 0) {
            // D = F32, A = B = BF16, both K-major, M = 128
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (((uint32_t)ranks16 >> 3) << 17) | ((128u >> 4) << 24);
            const uint32_t hi = (uint32_t)(smem_desc(0, 16, 1024, 2) >> 32), lo = (uint32_t)smem_desc(base, 16, 1024, 2);
            for (int i = 0; i < stages && !lost; ++i) {
                const uint32_t n = step + i, slot = n % ring;
                if (!mbar_wait_relaxed(full0 + slot * 8, (n / ring) & 1)) {
                    if (lane == 0) atomicOr(&g_lora_status, 1u), *failed = 1;
                    break;
                }
                tc_fence_after();
                const uint32_t x_lo = lo + slot * (stage >> 4), a_lo = x_lo + (kUmmaRows * kUmmaK * 2 >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int j = 0; j < kUmmaK / 16; ++j)   // 16 k: 32 bytes further along both rows
                        asm volatile(
                            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                            "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%3, %4};\n\t"
                            "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n\t}"
                            ::"r"(tmem), "r"(x_lo + j * 2), "r"(hi), "r"(a_lo + j * 2), "r"(hi), "r"(idesc), "r"((i | j) ? 1u : 0u)
                            : "memory");
                    tc_commit(empty0 + slot * 8);
                }
                __syncwarp();
            }
            if (!lost && elect_one()) tc_commit(done);
            __syncwarp();
        } else {
            const int row = 32 * (warp & 3) + lane;
            if (!lost && !mbar_wait_relaxed(done, pass & 1) && lane == 0) atomicOr(&g_lora_status, 1u), *failed = 1;
            tc_fence_after();
            float *out = c.t + ((int64_t)blockIdx.y * c.M + row0 + row) * c.r;
            const bool mine = owner[row] == adapter, spoilt = *failed != 0;
            for (int n = 0; n < ranks16; n += 16) {
                float d[16];
                tc_load16(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + n, d);
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    if (!mine || n + j >= c.r) continue;
                    const float poison = spoilt ? __uint_as_float(0x7FC00000u) : 0.f;
                    *reinterpret_cast<float4 *>(MXQ_AT(out + n + j, 16, c.t, (size_t)c.splits * c.M * c.r * 4)) =
                        make_float4(d[j] + poison, d[j + 1] + poison, d[j + 2] + poison, d[j + 3] + poison);
                }
            }
            tc_fence_before();
        }
        __syncthreads();     // the accumulator has been read
        tc_fence_after();
    }
    // A pass that gave up may have left requests in flight, and the CTA must not end before they have landed: those that are complete are waited for
    // (one that is not has a second in all), what else there may be is given time.
    if (warp == 1 && lane == 0 && *failed) {
        const uint64_t t0 = global_ns();
        for (int n = max(0, issued - ring); n < issued; ++n)
            while (!mbar_try_wait(full0 + n % ring * 8, (n / ring) & 1) && global_ns() - t0 < 1000000000ull) __nanosleep(200);
        const uint64_t t1 = global_ns();
        while (global_ns() - t1 < 100000ull) __nanosleep(1000);
    }
    __syncwarp();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}

// ---- base + B T -------------------------------------------------------------------------------------------------------------------
// grid (columns / (32 * warps), slots, windows); a warp takes 32 columns.  Tile i of 8 columns holds, in the product's order, columns
// 8t + 2i and 8t + 2i + 1 for t = 0..3, so that a lane ends up with eight consecutive columns of its rows.  Where N is no multiple of 8 and rows
// start anywhere, base and Y go by the element and the order is the plain one, tile i = columns 8i .. 8i + 7: a lane has columns 2t and 2t + 1 of
// every tile and four lanes share a sector (4000 x 1025, rank 64, FP32: 42 us with the other order, 28 with this one).  KT: most steps of 16 ranks.
__device__ __forceinline__ int own_column(bool vec, int t) { return vec ? 8 * t : 2 * t; }         // a lane's first, and from there on:
__device__ __forceinline__ int element(bool vec, int e) { return vec ? e : 8 * (e >> 1) + (e & 1); }
__device__ __forceinline__ int b_column(bool vec, int g, int i) { return vec ? 8 * (g >> 1) + 2 * i + (g & 1) : 8 * i + g; }
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
        const int o = element(false, e);
        if (o < there) f[e] = f32 ? ld_dep_f32(MXQ_AT(base + (at + o) * 4, 4, base, n * 4)) : ld_dep_bf16(MXQ_AT(base + (at + o) * 2, 2, base, n * 2));
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
        const int o = element(false, e);
        if (o >= there) continue;
        if (f32) *reinterpret_cast<float *>(MXQ_AT(y + (at + o) * 4, 4, y, n * 4)) = f[e];
        else *reinterpret_cast<__nv_bfloat16 *>(MXQ_AT(y + (at + o) * 2, 2, y, n * 2)) = __float2bfloat16_rn(f[e]);
    }
}

// eight bytes of B: ranks 4t .. 4t+3 of step s of a column; zero where there is no such column or rank
__device__ __forceinline__ uint2 load_b(const LoraCall &c, int adapter, int64_t col, int s, int t) {
    if (col >= c.N || 16 * s + 4 * t >= c.r) return make_uint2(0, 0);
    return __ldg(reinterpret_cast<const uint2 *>(MXQ_AT(c.b + ((int64_t)adapter * c.N + col) * c.r + 16 * s + 4 * t, 8, c.b, (size_t)c.L * c.N * c.r * 2)));
}

// the four ranks' sum over the splits, times the adapter's scale
__device__ __forceinline__ void sum_splits(float (&v)[4], const LoraCall &c, int m, int rank, int adapter) {
    const size_t t_bytes = (size_t)c.splits * c.M * c.r * 4;
    const float *p = c.t + (int64_t)m * c.r + rank;
    for (int u0 = 0; u0 < c.splits; u0 += 8) {
        uint4 q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (u0 + u < c.splits) q[u] = ld_dep_u4(MXQ_AT(p + (int64_t)(u0 + u) * c.M * c.r, 16, c.t, t_bytes));
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (u0 + u < c.splits)
                v[0] += __uint_as_float(q[u].x), v[1] += __uint_as_float(q[u].y), v[2] += __uint_as_float(q[u].z), v[3] += __uint_as_float(q[u].w);
    }
    const float s = c.scale ? __ldg(MXQ_AT(c.scale + adapter, 4, c.scale, (size_t)c.L * 4)) : 1.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= s;
}
// A lane's eight columns of a row of base as they come from memory (whole vectors only).
struct Columns {
    uint4 lo, hi;
};
__device__ __forceinline__ Columns load_ahead(const uint8_t *base, bool f32, int64_t at, int64_t n) {
    const uint8_t *p = MXQ_AT(base + at * (f32 ? 4 : 2), f32 ? 32 : 16, base, n * (f32 ? 4 : 2));
    Columns c;
    c.lo = ld_dep_u4(p);
    c.hi = f32 ? ld_dep_u4(p + 16) : make_uint4(0, 0, 0, 0);
    return c;
}
__device__ __forceinline__ void unpack_columns(float (&f)[8], const Columns &c, bool f32) {
    if (!f32) {
        unpack_bf16(f, c.lo);
        return;
    }
    const uint32_t w[8] = {c.lo.x, c.lo.y, c.lo.z, c.lo.w, c.hi.x, c.hi.y, c.hi.z, c.hi.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
}

// Few rows: a CTA has one adapter of the window (there are as many slots as a window can have adapters).  At least four CTAs per SM (three of 128
// ranks): left alone the compiler takes 158 registers for rank 32 (16 rows of 13 adapters, 11008 columns, beside the layer: 27.6 us, so 26.3).
template <int KT, int WARPS, bool PLAN>
__global__ void __launch_bounds__(32 * WARPS, KT <= 4 ? 4 : 3) lora_expand_kernel(LoraCall c) {
    extern __shared__ uint4 frag[];      // [steps][parts][32 lanes]: T as the product's first operand
    __shared__ Window win;
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int steps = (c.r + 15) / 16;
    const bool vec = c.N % 8 == 0;
    const int64_t col0 = ((int64_t)blockIdx.x * WARPS + warp) * 32, col = col0 + own_column(vec, t), n = (int64_t)c.M * c.N;
    if (PLAN) pdl_wait();
    load_window(win, c, blockIdx.z * 16, 16);
    __syncthreads();
    int adapter;
    uint2 w[KT][4];                      // this warp's columns of B wait here for T
    // the rows that this CTA stores: its adapter's; the first slot also copies those without one, unless they are there already
    const int there = (int)max((int64_t)0, min((int64_t)32, c.N - col));
    bool own[2], mine[2];
    int64_t place[2];                    // of the columns in base and Y
    Columns ahead[2];                    // base, on its way while T is made ready
    for (bool sure = PLAN;; sure = true) {           // (a second time where the guess was wrong)
        adapter = (int)blockIdx.y < win.count ? win.list[blockIdx.y] : -2;
        if (adapter >= 0) {
#pragma unroll
            for (int s = 0; s < KT; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s < steps) w[s][i] = load_b(c, adapter, col0 + b_column(vec, g, i), s, t);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = win.row[8 * h + g];
            own[h] = win.owner[8 * h + g] == adapter;
            mine[h] = there > 0 && row >= 0 && (own[h] || (blockIdx.y == 0 && c.base != c.y && win.owner[8 * h + g] < 0));
            place[h] = (int64_t)row * c.N + col;
        }
        int id = -1;
        if (!PLAN) pdl_wait(), id = window_id(c, blockIdx.z * 16, 16);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (c.base && vec && mine[h]) ahead[h] = load_ahead(c.base, c.base_f32, place[h], n);
        if (adapter >= 0) {
            for (int i = threadIdx.x; i < 16 * steps * 4; i += 32 * WARPS) {
                const int quarter = i % (steps * 4), m = i / (steps * 4);       // ranks 4 * quarter .. + 3 of row m
                float v[4] = {0.f, 0.f, 0.f, 0.f};
                if (win.owner[m] == adapter && 4 * quarter < c.r) sum_splits(v, c, win.row[m], 4 * quarter, adapter);
                put_parts(frag + quarter / 4 * c.parts * 32, m, quarter % 4, v, c.parts);
            }
        }
        __syncthreads();
        if (PLAN || sure || !wrong_window(win, id, 16)) break;
        __syncthreads();
        load_window(win, c, blockIdx.z * 16, 16);
        __syncthreads();
    }
    float acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    if (adapter >= 0) {
#pragma unroll
        for (int s = 0; s < KT; ++s) {
            if (s >= steps) break;
            for (int p = 0; p < c.parts; ++p) {
                const uint4 q = frag[(s * c.parts + p) * 32 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) mma_bf16(acc[i], q.x, q.y, q.z, q.w, w[s][i].x, w[s][i].y);
            }
        }
    }
    // (rows of other adapters went through the product as zeros; nothing of it is stored)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (!mine[h]) continue;
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (c.base && vec) unpack_columns(f, ahead[h], c.base_f32);
        else if (c.base) load_columns(f, c.base, c.base_f32, place[h], there, vec, n);
        if (own[h]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[2 * i] += acc[i][2 * h], f[2 * i + 1] += acc[i][2 * h + 1];
        }
        store_columns(f, c.y, c.y_f32, place[h], there, vec, n);
    }
}

// ---- many rows ------------------------------------------------------------------------------------------------------------------------
// T's partial sums -> its fragments, [tiles of 16 rows][steps][parts][32 lanes]: once, not for every block of columns.  A thread per row and four ranks.
// (No early trigger: expansion CTAs that settle beside this kernel's and the shrink's spread unevenly over the SMs.  2000 rows, rank 32, 11008
// outputs, FP32: 75 us with it, 53 without; 512 rows, rank 64, 4096 outputs: 16.5, 14.7.)
__global__ void __launch_bounds__(256) lora_fragments_kernel(LoraCall c) {
    const int quarters = (c.r + 15) / 16 * 4, tiles = (c.M + 15) / 16;
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(n / quarters), quarter = (int)(n - (int64_t)m * quarters);
    pdl_wait();
    if (m >= tiles * 16) return;
    const int adapter = load_id(c, m);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (adapter >= 0 && 4 * quarter < c.r) sum_splits(v, c, m, 4 * quarter, adapter);
    put_parts(fragment(c, m / 16, quarter / 4), m % 16, quarter % 4, v, c.parts);
}

// grid (blocks of 256 columns, blocks of c.tiles tiles of rows); a warp takes 32 columns, whose B stays in registers while the adapter does, and
// goes through the tiles; base of the next tile or two is on its way meanwhile.  VEC: N is a multiple of 8.
constexpr int kMostTiles = 24;
template <int KT, bool F32, bool VEC>
__global__ void __launch_bounds__(256, 2) lora_expand_many_kernel(LoraCall c) {
    constexpr int kParts = F32 ? 3 : 2, kSize = F32 ? 4 : 2;
    extern __shared__ uint4 frag[];      // the rows' fragments of T
    __shared__ int32_t owner[kMostTiles * 16];           // ... and their ids
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t col0 = ((int64_t)blockIdx.x * 8 + warp) * 32, col = col0 + own_column(VEC, t), n = (int64_t)c.M * c.N;
    const int steps = (c.r + 15) / 16, all = (c.M + 15) / 16, tile0 = blockIdx.y * c.tiles, tiles = min(c.tiles, all - tile0);
    const int there = (int)max((int64_t)0, min((int64_t)32, c.N - col));
    const bool copies = c.base != c.y;
    uint2 w[KT][4];
    auto load = [&](int adapter) {
#pragma unroll
        for (int s = 0; s < KT; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s < steps) w[s][i] = load_b(c, adapter, col0 + b_column(VEC, g, i), s, t);
    };
    // this lane's rows m, m + 8 of the tile whose base is loaded next; `place` of its columns in base and Y
    int m = tile0 * 16 + g;
    int64_t place = (int64_t)m * c.N + col;
    const int64_t row8 = 8 * c.N;
    constexpr int kAhead = F32 ? 1 : 2;      // tiles whose base is on its way (the registers hold one of FP32)
    Columns base[2], next_base[2];
    auto load_base = [&](Columns (&base)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            base[h].lo = base[h].hi = make_uint4(0, 0, 0, 0);
            if (!c.base || there <= 0 || m + 8 * h >= c.M) continue;
            if (VEC) {
                const uint8_t *p = MXQ_AT(c.base + (place + h * row8) * kSize, 8 * kSize, c.base, n * kSize);
                base[h].lo = ld_dep_u4(p);
                if (F32) base[h].hi = ld_dep_u4(p + 16);
            } else {
                float f[8];
                load_columns(f, c.base, F32, place + h * row8, there, false, n);
                if (F32) {
                    base[h].lo = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                    base[h].hi = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
                } else {
                    base[h].lo = pack_bf16(f);       // (exactly: they are BF16)
                }
            }
        }
    };
    int current = __reduce_max_sync(0xffffffffu, load_id(c, tile0 * 16 + (lane & 15)));       // whose B is in the registers (a guess: see load_window)
    if (current >= 0) load(current);
    pdl_wait();
    for (int i = threadIdx.x; i < tiles * 16; i += 256) owner[i] = load_id(c, tile0 * 16 + i);
    const int pieces = steps * kParts * 32;
    for (int i = threadIdx.x; i < tiles * pieces; i += 256)
        copy16(shared_address(frag + i), MXQ_AT(c.frag + (int64_t)tile0 * pieces + i, 16, c.frag, (size_t)all * pieces * 16), true);
    load_base(base);
    auto advance = [&]() { m += 16, place += 2 * row8; };
    if (kAhead == 2) advance(), load_base(next_base);      // (rows behind the last are not read)
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    if (col0 >= c.N) return;
    const uint4 *q = frag + lane;
    int64_t now = (int64_t)(tile0 * 16 + g) * c.N + col;
    for (int tile = 0; tile < tiles; ++tile, q += pieces) {
        const int rows = c.M - (tile0 + tile) * 16 - g;            // the lane's rows are there if 0, 8 < rows
        float f[2][8];
        int left[2], none[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            left[h] = owner[16 * tile + g + 8 * h], none[h] = left[h] < 0;
            unpack_columns(f[h], base[h], F32);
        }
        advance();
        if (kAhead == 2) {
#pragma unroll
            for (int h = 0; h < 2; ++h) base[h] = next_base[h];
            if (tile + 2 < tiles) load_base(next_base);
        } else if (tile + 1 < tiles) {
            load_base(base);
        }
        int adapter = __reduce_max_sync(0xffffffffu, max(left[0], left[1]));
        while (adapter >= 0) {               // the tile's adapters, one after the other
            if (adapter != current) load(adapter), current = adapter;
            float acc[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
            for (int s = 0; s < KT; ++s) {
                if (s >= steps) break;
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    const uint4 v = q[(s * kParts + p) * 32];
#pragma unroll
                    for (int i = 0; i < 4; ++i) mma_bf16(acc[i], v.x, v.y, v.z, v.w, w[s][i].x, w[s][i].y);
                }
            }
            // (rows of other adapters went through the product too; what they got is dropped here)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool mine = left[h] == adapter;
#pragma unroll
                for (int i = 0; i < 4; ++i) f[h][2 * i] = mine ? f[h][2 * i] + acc[i][2 * h] : f[h][2 * i], f[h][2 * i + 1] = mine ? f[h][2 * i + 1] + acc[i][2 * h + 1] : f[h][2 * i + 1];
                if (mine) left[h] = -1;
            }
            adapter = __reduce_max_sync(0xffffffffu, max(left[0], left[1]));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (there > 0 && 8 * h < rows && (!none[h] || copies)) store_columns(f[h], c.y, F32, now + h * row8, there, VEC, n);
        now += 2 * row8;
    }
}

MXQ_BOUNDS_TU(bounds_take_lora)

int lora_take_status(uint32_t *out) {
    unsigned int v = 0, zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_lora_status, sizeof v) != cudaSuccess) return MXQ_ERR_CUDA;
    if (v != 0 && cudaMemcpyToSymbol(g_lora_status, &zero, sizeof zero) != cudaSuccess) return MXQ_ERR_CUDA;
    *out = v;
    return MXQ_OK;
}

// ---- host ---------------------------------------------------------------------------------------------------------------

// Up to 16 rows: one window, a CTA of both kernels for each of its adapters.  Up to 511: sorted into segments (see lora_order_kernel).  More, and
// from 64 rows on with 48 rows and more per adapter: windows of rows as they come, in a prompt mostly of one adapter, with a second CTA where
// two meet; T's fragments are made once (256 rows of four adapters, rank 128, 11008 outputs: sorted 46 us, so 30; 128 rows of eight, rank 64, 4096
// outputs: 16, 23).  What the host knows is the number of adapters that are loaded, not those of the batch: all of these had every loaded adapter among
// their rows.  Where many more are loaded the way is that of few rows per adapter (400 rows of one adapter, rank 128, 11008 outputs: 22 us of one
// loaded, 27 of eight, 63 to 69 of nine and more).  From 512 rows on nothing sorts: a tile of 16 rows repeats its product for each adapter that it has
// (4095 rows of 32 adapters, rank 64, 4096 outputs: 44 us in order, 409 in random order; 512 rows 24, 178).
constexpr int kMostSplits = 16;
constexpr int kFewWarps = 8, kManyWarps = 16;     // of a CTA of the shrink (above rank 64 sixteen warps' sums do not fit the registers)
static bool many_rows(const LoraCall &c) { return c.M >= kMostSorted || (c.M >= 64 && c.M >= 48 * (int64_t)c.L); }
static bool few_rows(int64_t M) { return M <= 16; }
// The tensor memory path reads a window's 128 rows once for each of its adapters: for adapters of 80 rows and more on average (512 rows of six,
// 4096 inputs, rank 64: 23 -> 18 us; 1500 rows of twenty, rank 16: 20 -> 24).  By the adapters loaded, as above: 4095 rows of six, rank 64, take 42 us
// of six loaded and 55 of 52 and more.
static bool by_umma(const LoraCall &c) { return many_rows(c) && c.M >= 80 * (int64_t)c.L && c.K % kUmmaK == 0 && c.K <= 0x3FFFFFFF && tensor_map_available(); }
static int64_t most_segments(const LoraCall &c) { return c.M / 16 + min(c.L + 1, c.M); }

static void lora_plan(LoraCall &c) {
    const bool few = few_rows(c.M), many = many_rows(c);
    const int64_t sms = sm_count();
    const bool umma = by_umma(c);
    c.slots = few ? min(c.M, c.L) : umma ? min(4, c.L) : many ? min(2, c.L) : 1;
    // splits of K as long as the SMs hold the CTAs at once, but at least one step of 32 per warp or one stage
    const int64_t step = umma ? kUmmaK : 32 * (many && c.r <= 64 ? kManyWarps : kFewWarps), most = (c.K + step - 1) / step;
    int64_t want = max((int64_t)1, few ? 2 * sms / c.slots : umma ? sms / ((c.M + kUmmaRows - 1) / kUmmaRows) : many ? sms / ((c.M + 31) / 32) : 2 * sms / most_segments(c));
    if (want > most) want = most;
    if (want > kMostSplits) want = kMostSplits;
    int64_t len = ((c.K + want - 1) / want + step - 1) / step * step;
    c.split_k = (int32_t)len;
    c.splits = (int32_t)((c.K + len - 1) / len);
}
// Bound of splits x M: at least one split, at most kMostSplits of one stage each, and more than one only while all windows' (of up to 128 rows) find an SM
// at once.
static int64_t most_split_rows(int64_t M, int64_t K) {
    const int64_t splits = min((int64_t)kMostSplits, (K + kUmmaK - 1) / kUmmaK);
    return max(M, min(splits * M, (int64_t)kUmmaRows * sm_count()));
}
static size_t align256(size_t v) { return (v + 255u) & ~(size_t)255u; }
static size_t sums_bytes(const LoraCall &c) { return align256((size_t)c.splits * (size_t)c.M * (size_t)c.r * 4); }

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

static LoraCall lora_call(const void *X, int64_t M, const mxq_lora_adapters *ad, const int32_t *ids, int64_t N, int64_t K, const void *base, int base_dtype,
                          void *Y, int y_dtype, void *workspace) {
    LoraCall c = {};
    c.x = (const uint16_t *)X, c.a = (const uint16_t *)ad->A_bf16, c.b = (const uint16_t *)ad->B_bf16, c.scale = ad->scale, c.ids = ids;
    c.t = (float *)workspace, c.N = N, c.K = K, c.M = (int32_t)M, c.r = ad->rank, c.L = ad->count;
    c.base = (const uint8_t *)base, c.y = (uint8_t *)Y, c.base_f32 = base_dtype == MXQ_F32, c.y_f32 = y_dtype == MXQ_F32, c.parts = c.y_f32 ? 3 : 2;
    lora_plan(c);
    c.direct = many_rows(c) && !by_umma(c) && c.splits == 1;
    uint8_t *behind = reinterpret_cast<uint8_t *>(c.t) + sums_bytes(c);
    c.frag = reinterpret_cast<uint4 *>(behind);
    c.plan = few_rows(M) || many_rows(c) ? nullptr : reinterpret_cast<int32_t *>(behind);
    return c;
}

constexpr size_t kShrinkSmem = 200 * 1024, kExpandSmem = 100 * 1024;      // most of a CTA of the shrink, of the expansion of many rows

template <int MW, int WARPS, int RT>
static int shrink_launch(const LoraCall &c, cudaStream_t stream) {
    constexpr int kRows = 16 * MW;
    const dim3 grid((unsigned)(c.plan ? most_segments(c) : (c.M + kRows - 1) / kRows), (unsigned)c.slots, (unsigned)c.splits);
    const size_t stage = (size_t)WARPS * (RT + 2 * MW) * 512, parts = (size_t)WARPS * kRows * c.r * 4;
    const int steps = (c.split_k + 32 * WARPS - 1) / (32 * WARPS);
    LoraCall call = c;
    call.stages = max(1, min(min(kMostStages, steps), (int)(kShrinkSmem / stage)));
    const size_t smem = max(stage * call.stages, parts);
    static_assert((size_t)WARPS * kRows * 8 * RT * 4 <= kShrinkSmem && (size_t)WARPS * (RT + 2 * MW) * 512 <= kShrinkSmem, "");
    static std::atomic<bool> ready[64];
    const int rc = allow_smem(lora_shrink_kernel<MW, WARPS, RT>, kShrinkSmem, ready);
    if (rc != MXQ_OK) return rc;
    return launch_pdl(lora_shrink_kernel<MW, WARPS, RT>, grid, 32 * WARPS, smem, stream, call);
}
template <int MW, int WARPS>
static int shrink_by_rank(const LoraCall &c, cudaStream_t stream) {
    return c.r <= 16 ? shrink_launch<MW, WARPS, 2>(c, stream) : c.r <= 32 ? shrink_launch<MW, WARPS, 4>(c, stream) : shrink_launch<MW, WARPS, 8>(c, stream);
}

template <int WARPS, bool PLAN>
static void (*few_kernel(int r))(LoraCall) {
    return r <= 16 ? lora_expand_kernel<1, WARPS, PLAN> : r <= 32 ? lora_expand_kernel<2, WARPS, PLAN> : r <= 64 ? lora_expand_kernel<4, WARPS, PLAN> : lora_expand_kernel<8, WARPS, PLAN>;
}
static int expand_launch(const LoraCall &c, cudaStream_t stream) {
    constexpr int kWarps = 4;
    const dim3 grid((unsigned)((c.N + 32 * kWarps - 1) / (32 * kWarps)), (unsigned)c.slots, (unsigned)(c.plan ? most_segments(c) : 1));
    const size_t smem = (size_t)((c.r + 15) / 16) * c.parts * 32 * 16;
    return launch_pdl(c.plan ? few_kernel<kWarps, true>(c.r) : few_kernel<kWarps, false>(c.r), grid, 32 * kWarps, smem, stream, c);
}

template <int KT, bool F32, bool VEC>
static int many_launch(const LoraCall &c, dim3 grid, size_t smem, cudaStream_t stream) {
    static std::atomic<bool> ready[64];
    const int rc = allow_smem(lora_expand_many_kernel<KT, F32, VEC>, kExpandSmem, ready);
    return rc != MXQ_OK ? rc : launch_pdl(lora_expand_many_kernel<KT, F32, VEC>, grid, 256, smem, stream, c);
}
template <bool F32, bool VEC>
static int many_by_rank(const LoraCall &c, dim3 grid, size_t smem, cudaStream_t stream) {
    return c.r <= 16 ? many_launch<1, F32, VEC>(c, grid, smem, stream) : c.r <= 32 ? many_launch<2, F32, VEC>(c, grid, smem, stream)
         : c.r <= 64 ? many_launch<4, F32, VEC>(c, grid, smem, stream) : many_launch<8, F32, VEC>(c, grid, smem, stream);
}

static int expand_many_launch(LoraCall c, cudaStream_t stream) {
    const int steps = (c.r + 15) / 16, tiles = (c.M + 15) / 16;
    if (!c.direct) {
        const int rc = launch_pdl(lora_fragments_kernel, dim3((unsigned)(((int64_t)tiles * 16 * steps * 4 + 255) / 256)), 256, 0, stream, c);
        if (rc != MXQ_OK) return rc;
    }
    // tiles per CTA: what takes the fewest waves of two CTAs per SM, a CTA costing about as much as three tiles beside its own
    const int64_t columns = (c.N + 255) / 256, slots = 2 * (int64_t)sm_count();
    const size_t tile_bytes = (size_t)steps * c.parts * 512;
    int64_t least = 0;
    for (int t = 4; t <= kMostTiles && t * tile_bytes <= kExpandSmem; ++t) {
        const int64_t cost = (columns * ((tiles + t - 1) / t) + slots - 1) / slots * (t + 3);
        if (t == 4 || cost < least) least = cost, c.tiles = t;
    }
    const dim3 grid((unsigned)columns, (unsigned)((tiles + c.tiles - 1) / c.tiles));
    const size_t smem = c.tiles * tile_bytes;
    const bool vec = c.N % 8 == 0;
    return c.y_f32 ? (vec ? many_by_rank<true, true>(c, grid, smem, stream) : many_by_rank<true, false>(c, grid, smem, stream))
                   : (vec ? many_by_rank<false, true>(c, grid, smem, stream) : many_by_rank<false, false>(c, grid, smem, stream));
}

// test hook (mxq_debug_lora_lost_stage): consumed by the next launch
[[maybe_unused]] static std::atomic<int> g_lost_stage{-1};

static int shrink_umma_launch(LoraCall c, cudaStream_t stream) {
#ifdef MXQ_DEBUG_BOUNDS
    c.lost_stage = g_lost_stage.exchange(-1, std::memory_order_relaxed);
#endif
    const int ranks16 = (c.r + 15) / 16 * 16, columns = ranks16 <= 32 ? 32 : ranks16 <= 64 ? 64 : 128;
    CUtensorMap xmap, amap;
    if (!encode_bf16_tensor_map(c.x, c.M, c.K, kUmmaRows, &xmap) || !encode_bf16_tensor_map(c.a, (int64_t)c.L * c.r, c.K, ranks16, &amap)) return MXQ_ERR_CUDA;
    // a ring that lets two CTAs share an SM where that leaves four stages (the prompt of rank 64: 47 -> 42 us; at rank 128 three stages cost 110 -> 125)
    const int stage = kUmmaRows * kUmmaK * 2 + ranks16 * kUmmaK * 2, half = 105 * 1024 / stage, ring = min(min(8, c.split_k / kUmmaK), half >= 4 ? half : (int)kShrinkSmem / stage);
    const size_t smem = 1024 + (size_t)ring * (stage + 16) + 8;
    static std::atomic<bool> ready[64];
    const int rc = allow_smem(lora_shrink_umma_kernel, 1024 + kShrinkSmem + 8 * 16 + 8, ready);
    if (rc != MXQ_OK) return rc;
    const dim3 grid((unsigned)((c.M + kUmmaRows - 1) / kUmmaRows), (unsigned)c.splits, (unsigned)c.slots);
    return launch_pdl(lora_shrink_umma_kernel, grid, kUmmaThreads, smem, stream, xmap, amap, c, ring, ranks16, columns);
}

static int lora_shrink(const LoraCall &c, cudaStream_t stream) {
    if (by_umma(c)) return shrink_umma_launch(c, stream);
    if (many_rows(c)) return c.r <= 64 ? shrink_by_rank<2, kManyWarps>(c, stream) : shrink_launch<2, kFewWarps, 16>(c, stream);
    if (c.plan) {
        const int rc = launch_pdl(lora_order_kernel, dim3(1), kMostSorted, 0, stream, c);
        if (rc != MXQ_OK) return rc;
    }
    return c.r <= 64 ? shrink_by_rank<1, kFewWarps>(c, stream) : shrink_launch<1, kFewWarps, 16>(c, stream);
}
static int lora_expand(const LoraCall &c, cudaStream_t stream) {
    return many_rows(c) ? expand_many_launch(c, stream) : expand_launch(c, stream);
}

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

size_t mxq_lora_workspace_bytes(int64_t M, int64_t N, int64_t K, int rank, int adapters) {
    if (!mxq::lora_shape_ok(M, N, K, rank, adapters)) return 0;
    // [partial sums][fragments: three BF16 parts of 16-row tiles, or the plan of the segments].  What a call takes depends on its path and falls where
    // windows grow; this is a bound for all of them that never falls from M to M + 1, so that the workspace of the largest batch serves all.
    const size_t fragments = (size_t)((M + 15) / 16) * ((rank + 15) / 16) * 3 * 512;
    return mxq::align256((size_t)mxq::most_split_rows(M, K) * rank * 4) + (mxq::few_rows(M) ? 0 : std::max(fragments, (size_t)mxq::kPlanBytes));
}

int mxq_lora(const void *X_bf16, int64_t M, const mxq_lora_adapters *adapters, const int32_t *ids, int64_t N, int64_t K, const void *base,
             void *Y, int y_dtype, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = mxq::lora_check(X_bf16, M, adapters, ids, N, K, Y, y_dtype);
    if (rc != MXQ_OK) return rc;
    if (!mxq::aligned16(base) || !mxq::aligned16(workspace)) return MXQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < mxq_lora_workspace_bytes(M, N, K, adapters->rank, adapters->count)) return MXQ_ERR_WORKSPACE;
    const mxq::LoraCall c = mxq::lora_call(X_bf16, M, adapters, ids, N, K, base, y_dtype, Y, y_dtype, workspace);
    rc = mxq::lora_shrink(c, (cudaStream_t)stream);
    return rc != MXQ_OK ? rc : mxq::lora_expand(c, (cudaStream_t)stream);
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
    const mxq::LoraCall c = mxq::lora_call(X_bf16, M, adapters, ids, N, K, base, MXQ_F32, Y, y_dtype, workspace);
    rc = mxq::lora_shrink(c, (cudaStream_t)stream);
    if (rc != MXQ_OK) return rc;
    rc = mxq_linear(X_bf16, M, codes, scales, N, K, base, MXQ_F32, ws + t_bytes + sums, mxq::align256(mxq_linear_workspace_bytes(M, N, K)), stream);
    if (rc != MXQ_OK) return rc;
    return mxq::lora_expand(c, (cudaStream_t)stream);
}

int mxq_debug_lora_lost_stage(int stage) {
#ifdef MXQ_DEBUG_BOUNDS
    mxq::g_lost_stage.store(stage, std::memory_order_relaxed);
    return MXQ_OK;
#else
    (void)stage;
    return MXQ_ERR_SHAPE;
#endif
}

#pragma GCC visibility pop
}  // extern "C"
