// mxq_kv_resize, mxq_kv_fork, mxq_kv_compact: the pages of a 4-bit cache as sequences grow, shrink, branch and are cut down
// to an accepted path.
//
// Page tables, lengths and reference counts are small integers; a call is latency, not traffic.  One CTA does the whole
// bookkeeping of a call, so that its steps (drop references, prefix sum of what is wanted, hand out free pages) are
// separated by block barriers instead of launches, and so that the result does not depend on scheduling: the r-th page
// wanted, counted over sequences in order, is the r-th free page of the pool, counted by index.
// Measured in replayed graphs: a resize that changes nothing 2.6 us (16 to 256 sequences); growth and the shrinking back
// together 7.8 us (16 sequences, 1024 pages) and 24 us (256 sequences that grow by up to 64 pages each, 65536 pages), where the search of the counts, a
// chain of loads and barriers per 16384 pages, and the entries' scattered loads and stores bound it; every list is dealt out flat, entry by
// entry, to 1024 threads.  One CTA is a choice (no launch and no flag between the steps), not a limit: the large pool's counts could be
// searched by several.
#include <algorithm>

#include "mxq_kv.cuh"

namespace mxq {

constexpr int kBookThreads = 1024;
constexpr int kBookWarps = kBookThreads / 32;

// inclusive prefix sum over the block of one value per thread; every thread gets the block's total too
template <class V>
__device__ __forceinline__ V block_scan(V v, V *total) {
    __shared__ V part[kBookWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
    }
    if (lane == 31) part[warp] = v;
    __syncthreads();
    if (warp == 0) {
        V p = part[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const V up = __shfl_up_sync(0xffffffffu, p, o);
            if (lane >= o) p += up;
        }
        part[lane] = p;
    }
    __syncthreads();
    if (warp > 0) v += part[warp - 1];
    *total = part[kBookWarps - 1];
    __syncthreads();   // `part` may be written again
    return v;
}

// upto[i] = need[0] + .. + need[i], in place
__device__ __forceinline__ int scan_needs(int *need, int n) {
    int carry = 0;
    for (int base = 0; base < n; base += kBookThreads) {
        const int i = base + (int)threadIdx.x;
        int sum;
        const int v = block_scan(i < n ? need[i] : 0, &sum);
        if (i < n) need[i] = carry + v;
        carry += sum;
    }
    __syncthreads();
    return carry;
}

// Calls give(rank, page) for the free pages (refs == 0) of lowest index, rank = 0 .. min(wanted, free) - 1, and returns how
// many there were.  16384 pages per step (four 16-byte loads a thread), until enough are found.  `give` may write the
// count of its own page.
template <class F>
__device__ __forceinline__ int lowest_free(const int32_t *refs, int num_pages, int wanted, F give) {
    constexpr int kQ = 4, kStep = 4 * kBookThreads;
    int found = 0;
    for (int64_t base = 0; base < num_pages && found < wanted; base += kQ * kStep) {
        uint32_t free_bits[kQ];
        unsigned long long counts = 0;   // 16 bits for each of the kQ loads (their block totals are at most kStep = 4096)
#pragma unroll
        for (int u = 0; u < kQ; ++u) {
            const int64_t p = base + u * kStep + (int64_t)threadIdx.x * 4;
            free_bits[u] = 0;
            if (p + 3 < num_pages) {
                const uint4 r = ld_dep_u4(MXQ_AT(refs + p, 16, refs, (size_t)num_pages * 4));
                free_bits[u] = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
            } else {
                for (int e = 0; e < 4 && p + e < num_pages; ++e)
                    free_bits[u] |= (uint32_t)(ld_dep_u32(MXQ_AT(refs + p + e, 4, refs, (size_t)num_pages * 4)) == 0) << e;
            }
            counts |= (unsigned long long)__popc(free_bits[u]) << (16 * u);
        }
        unsigned long long total;
        const unsigned long long before = block_scan(counts, &total) - counts;
        int at = found;
#pragma unroll
        for (int u = 0; u < kQ; ++u) {
            int rank = at + (int)((before >> (16 * u)) & 0xFFFF);
            uint32_t bits = free_bits[u];
            while (bits != 0 && rank < wanted) {
                const int e = __ffs((int)bits) - 1;
                bits &= bits - 1;
                give(rank++, (int)(base + u * kStep + (int64_t)threadIdx.x * 4 + e));
            }
            at += (int)((total >> (16 * u)) & 0xFFFF);
        }
        found = at;
    }
    return min(found, wanted);
}

// first i with upto[i] > rank
__device__ __forceinline__ int owner_of(const int *upto, int n, int rank) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] > rank) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct Book {
    int32_t *refs, *tables, *lens;
    int32_t num_pages, B, W, page_shift;
};

__device__ __forceinline__ int32_t *ref_of(const Book &k, int page) { return MXQ_AT(k.refs + page, 4, k.refs, (size_t)k.num_pages * 4); }
__device__ __forceinline__ int32_t *entry_of(const Book &k, int b, int w) {
    return MXQ_AT(k.tables + (int64_t)b * k.W + w, 4, k.tables, (size_t)k.B * k.W * 4);
}
__device__ __forceinline__ int book_len(const Book &k, int b) {
    const int n = (int)ld_dep_u32(MXQ_AT(k.lens + b, 4, k.lens, (size_t)k.B * 4));
    return (int)min((int64_t)max(n, 0), (int64_t)k.W << k.page_shift);
}
__device__ __forceinline__ int pages_for(int64_t n, int shift) { return (int)((n + (1 << shift) - 1) >> shift); }

// x-th of the places that a list of counts with prefix sums `upto` describes: which entry, and which of its places
struct Owned {
    int i, k;
};
__device__ __forceinline__ Owned owned(const int *upto, int n, int x) {
    const int i = owner_of(upto, n, x);
    return {i, x - (i ? upto[i - 1] : 0)};
}

// 16-byte pieces of a page's filled tiles, in every layer, by the whole block: a warp per layer, four loads in flight per lane
__device__ __forceinline__ void copy_page(const KvView &c, int layers, int64_t layer_bytes, int from_page, int to_page, int64_t bytes) {
    constexpr int kU = 4;
    const int lane = threadIdx.x & 31;
    for (int layer = (int)threadIdx.x >> 5; layer < layers; layer += kBookWarps) {
        const uint8_t *from = c.base + layer * layer_bytes + (int64_t)from_page * c.page_bytes;
        uint8_t *to = c.base + layer * layer_bytes + (int64_t)to_page * c.page_bytes;
        for (int64_t at0 = lane * 16; at0 < bytes; at0 += kU * 32 * 16) {
            uint4 v[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (at0 + u * 512 < bytes) v[u] = ld_dep_u4(MXQ_AT(from + at0 + u * 512, 16, c.pool, c.pool_bytes));
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (at0 + u * 512 < bytes) *reinterpret_cast<uint4 *>(MXQ_AT(to + at0 + u * 512, 16, c.pool, c.pool_bytes)) = v[u];
        }
    }
}

// A sequence that is cut inside a page which others hold too (a rollback behind a fork) would append into their tokens: it gets
// a page of its own with the tokens that stay.  The copy is this CTA's work as well (49 us for a page of 64 tokens in 32 layers of 8 heads
// of 128): it happens once per branch at most, and a launch of its own would cost every resize.  To find such a page a rollback reads
// the entry and the count of the page it ends in, two dependent loads (0.5 to 1 us).
__global__ void __launch_bounds__(kBookThreads) kv_resize_kernel(Book k, const int32_t *new_lens, KvView c, int layers, int64_t layer_bytes) {
    extern __shared__ int book_smem[];
    // per sequence: pages wanted and pages dropped (both summed up), pages held, the shared page that it ends in or -1
    int *upto = book_smem, *held = book_smem + k.B, *drop = book_smem + 2 * k.B, *split = book_smem + 3 * k.B;
    __shared__ int any_split;
    const int64_t cap = (int64_t)k.W << k.page_shift;
    const int mask = (1 << k.page_shift) - 1;
    if (threadIdx.x == 0) any_split = 0;
    __syncthreads();
    pdl_trigger();
    pdl_wait();
    for (int b = (int)threadIdx.x; b < k.B; b += kBookThreads) {
        const int n = (int)ld_dep_u32(MXQ_AT(new_lens + b, 4, new_lens, (size_t)k.B * 4)), len = book_len(k, b), have = pages_for(len, k.page_shift);
        const bool valid = n >= 0 && n <= cap;
        const int want = valid ? pages_for(n, k.page_shift) : have;
        int page = -1;
        if (valid && n < len && (n & mask) != 0) {
            page = (int)ld_dep_u32(entry_of(k, b, n >> k.page_shift));
            if ((unsigned)page >= (unsigned)k.num_pages || (int)ld_dep_u32(ref_of(k, page)) <= 1) page = -1;
            else any_split = 1;
        }
        upto[b] = page >= 0 ? 1 : max(want - have, 0), held[b] = have, drop[b] = max(have - want, 0), split[b] = page;
    }
    __syncthreads();
    const int wanted = scan_needs(upto, k.B), dropped = scan_needs(drop, k.B);
#pragma unroll 4
    for (int x = (int)threadIdx.x; x < dropped; x += kBookThreads) {
        const Owned o = owned(drop, k.B, x);
        int32_t *e = entry_of(k, o.i, held[o.i] - 1 - o.k);
        const int page = (int)ld_dep_u32(e);
        *e = -1;
        if ((unsigned)page < (unsigned)k.num_pages) atomicSub(ref_of(k, page), 1);
    }
    __syncthreads();
    auto last_place = [&](int b) { return held[b] - (drop[b] - (b ? drop[b - 1] : 0)) - 1; };      // of the pages that stay
    const int found = lowest_free(k.refs, k.num_pages, wanted, [&](int rank, int page) {
        const Owned o = owned(upto, k.B, rank);
        *entry_of(k, o.i, split[o.i] >= 0 ? last_place(o.i) : held[o.i] + o.k) = page;
        *ref_of(k, page) = 1;
    });
    __syncthreads();
    if (found < wanted) {   // the one sequence that got a part of what it asked for gives it back
        const int b = owner_of(upto, k.B, found), first = b ? upto[b - 1] : 0;
        for (int r = first + (int)threadIdx.x; r < found; r += kBookThreads) {
            int32_t *e = entry_of(k, b, held[b] + r - first);
            *ref_of(k, (int)ld_dep_u32(e)) = 0;
            *e = -1;
        }
    }
    for (int b = (int)threadIdx.x; b < k.B; b += kBookThreads) {
        const int n = (int)ld_dep_u32(MXQ_AT(new_lens + b, 4, new_lens, (size_t)k.B * 4));
        const bool none = upto[b] == (b ? upto[b - 1] : 0), fits = none || upto[b] <= found;
        int32_t *len = MXQ_AT(k.lens + b, 4, k.lens, (size_t)k.B * 4);
        if (n >= 0 && n <= cap && fits) *len = n;
        else if (split[b] >= 0) *len = (int)min((int64_t)book_len(k, b), (int64_t)(last_place(b) + 1) << k.page_shift);      // as far back as it goes without a page
    }
    if (any_split == 0) return;
    for (int b = 0; b < k.B; ++b) {
        if (split[b] < 0 || upto[b] > found) continue;
        const int n = (int)ld_dep_u32(MXQ_AT(new_lens + b, 4, new_lens, (size_t)k.B * 4));
        const int tiles = ((n & mask) + kTileTokens - 1) / kTileTokens;
        copy_page(c, layers, layer_bytes, split[b], (int)ld_dep_u32(entry_of(k, b, last_place(b))), c.page_bytes * tiles >> (k.page_shift - 5));
        if (threadIdx.x == 0) atomicSub(ref_of(k, split[b]), 1);
    }
}

// what the copy kernel has to do for child i: pages and filled 32-token tiles of the last page (0: nothing)
struct ForkJob {
    int32_t src, dst, tiles, pad;
};

__global__ void __launch_bounds__(kBookThreads)
kv_fork_kernel(Book k, int n, const int32_t *src, const int32_t *dst, ForkJob *jobs) {
    extern __shared__ int book_smem[];
    // per child: pages wanted (summed up), its fresh page or -1 if the pair is refused, whole pages to share (summed up), source, slot, length
    int *upto = book_smem, *fresh = book_smem + n, *shared = book_smem + 2 * n, *from = book_smem + 3 * n, *to = book_smem + 4 * n, *lens = book_smem + 5 * n;
    const int mask = (1 << k.page_shift) - 1;
    pdl_trigger();
    pdl_wait();
    for (int i = (int)threadIdx.x; i < n; i += kBookThreads) {
        const int s = (int)ld_dep_u32(MXQ_AT(src + i, 4, src, (size_t)n * 4)), d = (int)ld_dep_u32(MXQ_AT(dst + i, 4, dst, (size_t)n * 4));
        const bool in = (unsigned)s < (unsigned)k.B && (unsigned)d < (unsigned)k.B && s != d;
        const bool ok = in && book_len(k, d) == 0;      // an occupied slot is refused
        const int len = ok ? book_len(k, s) : 0;
        from[i] = s, to[i] = d, lens[i] = len;
        fresh[i] = ok ? 0 : -1;
        upto[i] = ok && (len & mask) != 0;
    }
    __syncthreads();
    const int wanted = scan_needs(upto, n);
    const int found = lowest_free(k.refs, k.num_pages, wanted, [&](int rank, int page) { fresh[owner_of(upto, n, rank)] = page; });
    __syncthreads();
    for (int i = (int)threadIdx.x; i < n; i += kBookThreads) {
        const bool part = upto[i] != (i ? upto[i - 1] : 0), fits = fresh[i] >= 0 && (!part || upto[i] <= found);
        const int whole = lens[i] >> k.page_shift;
        ForkJob job = {0, 0, 0, 0};
        if (fits && part) {
            job.src = (int)ld_dep_u32(entry_of(k, from[i], whole));
            job.dst = -1;      // (where the parent's tokens are on no page, so are the child's, and the page stays free)
            if ((unsigned)job.src < (unsigned)k.num_pages) {
                job.dst = fresh[i], job.tiles = ((lens[i] & mask) + kTileTokens - 1) / kTileTokens;
                *ref_of(k, job.dst) = 1;
            }
            *entry_of(k, to[i], whole) = job.dst;
        }
        shared[i] = fits ? whole : 0;
        if (fits) *MXQ_AT(k.lens + to[i], 4, k.lens, (size_t)k.B * 4) = lens[i];
        *MXQ_AT(jobs + i, sizeof(ForkJob), jobs, (size_t)n * sizeof(ForkJob)) = job;
    }
    __syncthreads();
    const int total = scan_needs(shared, n);
#pragma unroll 4
    for (int x = (int)threadIdx.x; x < total; x += kBookThreads) {
        const Owned o = owned(shared, n, x);
        const int page = (int)ld_dep_u32(entry_of(k, from[o.i], o.k));
        *entry_of(k, to[o.i], o.k) = page;
        if ((unsigned)page < (unsigned)k.num_pages) atomicAdd(ref_of(k, page), 1);
    }
}

// Copies the filled part of the last pages: grid = (child, layer, piece), a piece being 16 KB of one 32-token tile row (the
// tiles of all heads, which lie together), four 16-byte loads in flight per thread.  Bound by the copy rate from some tens of
// children on: 64 children of 16 parents, 32 layers of 8 heads (205 MB read and written), fork and the freeing of the children
// together 34 us, the copy alone at the roof 31.3; 4 children of one: 12.5 us for two launches of bookkeeping and 17.8 MB.
constexpr int kCopyThreads = 256, kCopyUnroll = 4, kCopyPiece = kCopyThreads * kCopyUnroll * 16, kMaxGridY = 65535;

__global__ void __launch_bounds__(kCopyThreads)
kv_fork_copy_kernel(const ForkJob *jobs, int n, KvView c, int layers, int64_t layer_bytes, int64_t row_bytes, int pieces) {
    pdl_trigger();
    pdl_wait();
    const uint4 j = ld_dep_u4(MXQ_AT(jobs + blockIdx.x, 16, jobs, (size_t)n * 16));
    const int tile = (int)blockIdx.z / pieces, piece = (int)blockIdx.z - tile * pieces;
    if (tile >= (int)j.z || !kv_page_ok(c, (int)j.x) || !kv_page_ok(c, (int)j.y)) return;
    const int64_t off = tile * row_bytes, first = (int64_t)piece * kCopyPiece;
    for (int layer = (int)blockIdx.y; layer < layers; layer += (int)gridDim.y) {      // (a grid has at most kMaxGridY of them)
        const uint8_t *from = c.base + layer * layer_bytes + (int64_t)(int)j.x * c.page_bytes + off;
        uint8_t *to = c.base + layer * layer_bytes + (int64_t)(int)j.y * c.page_bytes + off;
        uint4 v[kCopyUnroll];
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const int64_t at = first + (u * kCopyThreads + (int)threadIdx.x) * 16;
            if (at < row_bytes) v[u] = ld_dep_u4(MXQ_AT(from + at, 16, c.pool, c.pool_bytes));
        }
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const int64_t at = first + (u * kCopyThreads + (int)threadIdx.x) * 16;
            if (at < row_bytes) *reinterpret_cast<uint4 *>(MXQ_AT(to + at, 16, c.pool, c.pool_bytes)) = v[u];
        }
    }
}

// Moves kept tokens down within the last `rows` positions of a sequence: one warp per (sequence, layer, head).  keep is
// ascending, so token j's source lies at or behind its destination and a batch of pieces may be stored once all of the
// batch is loaded: later sources lie behind every destination written so far.  Latency (a chain of dependent loads: lengths and
// counts, keep, page entries, data; a batch is one round of it): 32 layers x 8 heads of one 16-row tree 3.2 us, 64 trees of 48 rows in
// 16 layers x 8 heads, 2 to 6 rows kept, 7.5 us, one round in 8192 warps (0.4 of the issue slots, loads are what is waited for).
constexpr int kCompactThreads = 128, kCompactBatch = 4;

template <int D>
__global__ void __launch_bounds__(kCompactThreads)
kv_compact_kernel(KvView c, KvSeqs s, int layers, int64_t layer_bytes, const int32_t *keep, const int32_t *kept, int32_t *lens_out) {
    using T = KvTile<D>;
    constexpr int kNb = T::kNb, kPieces = D / 16 + 2;   // 16 bytes each of K and V codes; K scales; V scales
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (kCompactThreads / 32) + (threadIdx.x >> 5);
    const int b = (int)(unit / ((int64_t)layers * c.heads)), rest = (int)(unit - (int64_t)b * layers * c.heads);
    const int layer = rest / c.heads, head = rest - layer * c.heads;
    if (b >= s.B) return;
    pdl_wait();
    const int len = s.len(b), rows = min(s.nrows(b), len), first = len - rows;
    const int count = min(max((int)ld_dep_u32(MXQ_AT(kept + b, 4, kept, (size_t)s.B * 4)), 0), rows);
    if (rest == 0 && lane == 0) *MXQ_AT(lens_out + b, 4, lens_out, (size_t)s.B * 4) = first + count;
    c.base += (int64_t)layer * layer_bytes;

    // piece e of a token: its address for an access of the piece's kind
    auto tile_of = [&](int pos) -> uint8_t * {
        const int page = s.page(b, pos >> c.page_shift);
        return kv_page_ok(c, page) ? kv_tile<D>(c, page, pos & ((1 << c.page_shift) - 1), head) : nullptr;
    };
    for (int base = 0; base < count * kPieces; base += 32 * kCompactBatch) {
        uint4 v[kCompactBatch];
        uint8_t *to[kCompactBatch];
#pragma unroll
        for (int u = 0; u < kCompactBatch; ++u) {
            const int p = base + u * 32 + lane, j = p / kPieces, e = p - j * kPieces;
            to[u] = nullptr;
            if (j >= count) continue;
            const int from = (int)ld_dep_u32(MXQ_AT(keep + (int64_t)b * s.m + j, 4, keep, (size_t)s.B * s.m * 4));
            if (from <= j || from >= rows) continue;   // in place already, or not a row
            const uint8_t *src = tile_of(first + from);
            uint8_t *dst = tile_of(first + j);
            if (src == nullptr || dst == nullptr) continue;
            to[u] = dst;
            const int ts = (first + from) & 31;
            if (e < D / 16) {
                const int half = e / (D / 32), q = e - half * (D / 32);
                v[u] = ld_dep_u4(MXQ_AT(src + half * T::kV + ts * T::kRow + 16 * q, 16, c.pool, c.pool_bytes));
            } else {
                v[u].x = 0;
#pragma unroll
                for (int blk = 0; blk < kNb; ++blk) {
                    const uint8_t *a = src + (e == D / 16 ? T::kKs + ts * kNb + blk : T::vs(ts, blk));
                    unsigned short byte;
                    asm volatile("ld.global.cg.u8 %0, [%1];" : "=h"(byte) : "l"(MXQ_AT(a, 1, c.pool, c.pool_bytes)) : "memory");
                    v[u].x |= (uint32_t)byte << (8 * blk);
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kCompactBatch; ++u) {
            if (to[u] == nullptr) continue;
            const int p = base + u * 32 + lane, j = p / kPieces, e = p - j * kPieces, ts = (first + j) & 31;
            if (e < D / 16) {
                const int half = e / (D / 32), q = e - half * (D / 32);
                *reinterpret_cast<uint4 *>(MXQ_AT(to[u] + half * T::kV + ts * T::kRow + 16 * q, 16, c.pool, c.pool_bytes)) = v[u];
            } else {
#pragma unroll
                for (int blk = 0; blk < kNb; ++blk)
                    *MXQ_AT(to[u] + (e == D / 16 ? T::kKs + ts * kNb + blk : T::vs(ts, blk)), 1, c.pool, c.pool_bytes) = (uint8_t)(v[u].x >> (8 * blk));
            }
        }
        __syncwarp();
    }
}

MXQ_BOUNDS_TU(bounds_take_kv_pages)

// ---- host ---------------------------------------------------------------------------------------------------------------

// shared memory for the largest call: 24 bytes per sequence
static int book_smem_ready(const void *kernel) {
    static const void *ready[64][2];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return MXQ_ERR_CUDA;
    const void **slot = kernel == (const void *)kv_resize_kernel ? &ready[dev][0] : &ready[dev][1];
    if (*slot != kernel) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MXQ_KV_MAX_SEQS * 24) != cudaSuccess) {
            (void)cudaGetLastError();
            return MXQ_ERR_CUDA;
        }
        *slot = kernel;
    }
    return MXQ_OK;
}

static Book book_of(const mxq_kv_cache *c, int B, int32_t *tables, int W, int32_t *lens) {
    Book k;
    k.refs = c->refs, k.tables = tables, k.lens = lens;
    k.num_pages = (int32_t)c->num_pages, k.B = B, k.W = W;
    k.page_shift = kv_view(c, 0).page_shift;
    return k;
}

}  // namespace mxq

extern "C" {
#pragma GCC visibility push(default)

int mxq_kv_resize(const mxq_kv_cache *cache, int B, int32_t *tables, int W, int32_t *lens, const int32_t *new_lens, void *stream) {
    if (!new_lens) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, 0);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    if (!mxq::aligned_to(new_lens, 4)) return MXQ_ERR_ALIGN;
    rc = mxq::book_smem_ready((const void *)mxq::kv_resize_kernel);
    if (rc != MXQ_OK) return rc;
    const mxq::KvView c = mxq::kv_view(cache, 0);
    return mxq::kv_launch(mxq::kv_resize_kernel, dim3(1), mxq::kBookThreads, (size_t)B * 16, (cudaStream_t)stream,
                          mxq::book_of(cache, B, tables, W, lens), new_lens, c, cache->layers, c.page_bytes * cache->num_pages);
}

size_t mxq_kv_fork_workspace_bytes(int n) { return n < 1 || n > MXQ_KV_MAX_SEQS ? 0 : (size_t)n * sizeof(mxq::ForkJob); }

int mxq_kv_fork(const mxq_kv_cache *cache, int B, int32_t *tables, int W, int32_t *lens, int n, const int32_t *src, const int32_t *dst,
                void *workspace, size_t workspace_bytes, void *stream) {
    if (!src || !dst) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, 0);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    if (n < 1 || n > MXQ_KV_MAX_SEQS) return MXQ_ERR_SHAPE;
    if (!mxq::aligned_to(src, 4) || !mxq::aligned_to(dst, 4) || !mxq::aligned16(workspace)) return MXQ_ERR_ALIGN;
    if (!workspace || workspace_bytes < mxq_kv_fork_workspace_bytes(n)) return MXQ_ERR_WORKSPACE;
    mxq::ForkJob *jobs = (mxq::ForkJob *)workspace;
    rc = mxq::book_smem_ready((const void *)mxq::kv_fork_kernel);
    if (rc != MXQ_OK) return rc;
    rc = mxq::kv_launch(mxq::kv_fork_kernel, dim3(1), mxq::kBookThreads, (size_t)n * 24, (cudaStream_t)stream,
                        mxq::book_of(cache, B, tables, W, lens), n, src, dst, jobs);
    if (rc != MXQ_OK) return rc;
    const mxq::KvView c = mxq::kv_view(cache, 0);
    const int tiles = cache->page_tokens / mxq::kTileTokens;
    const int64_t row_bytes = c.page_bytes / tiles;
    const int pieces = (int)((row_bytes + mxq::kCopyPiece - 1) / mxq::kCopyPiece);
    return mxq::kv_launch(mxq::kv_fork_copy_kernel, dim3((unsigned)n, (unsigned)std::min(cache->layers, mxq::kMaxGridY), (unsigned)(tiles * pieces)), mxq::kCopyThreads,
                          0, (cudaStream_t)stream, (const mxq::ForkJob *)jobs, n, c, cache->layers, c.page_bytes * cache->num_pages, row_bytes, pieces);
}

int mxq_kv_compact(const mxq_kv_cache *cache, int B, int M, const int32_t *tables, int W, const int32_t *lens, const int32_t *rows,
                   const int32_t *keep, const int32_t *kept, int32_t *lens_out, void *stream) {
    if (!keep || !kept || !lens_out) return MXQ_ERR_NULL;
    int rc = mxq::kv_check_cache(cache, 0);
    if (rc == MXQ_OK) rc = mxq::kv_check_seqs(B, W, tables, lens);
    if (rc != MXQ_OK) return rc;
    if (M < 1 || M > MXQ_MAX_T || lens_out == lens) return MXQ_ERR_SHAPE;
    if (!mxq::aligned_to(rows, 4) || !mxq::aligned_to(keep, 4) || !mxq::aligned_to(kept, 4) || !mxq::aligned_to(lens_out, 4)) return MXQ_ERR_ALIGN;
    const int64_t units = (int64_t)B * cache->layers * cache->kv_heads;
    const int64_t grid = (units + mxq::kCompactThreads / 32 - 1) / (mxq::kCompactThreads / 32);
    if (grid > 0x7FFFFFFF) return MXQ_ERR_SHAPE;
    const mxq::KvView c = mxq::kv_view(cache, 0);
    const mxq::KvSeqs s = mxq::kv_seqs(cache, B, M, tables, W, lens, rows);
    return mxq::kv_launch(cache->head_dim == 128 ? mxq::kv_compact_kernel<128> : mxq::kv_compact_kernel<64>, dim3((unsigned)grid),
                          mxq::kCompactThreads, 0, (cudaStream_t)stream, c, s, cache->layers, c.page_bytes * cache->num_pages, keep, kept, lens_out);
}

#pragma GCC visibility pop
}  // extern "C"
