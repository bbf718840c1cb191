// How mxq_kv_attention's work is divided: sizes of items, the parts of a segment, the limits they keep.  Plain C++, used by the kernel
// and checked on the host over all the shapes there are.
//
// A segment (sequence, kv head, row tile) of n 32-token tiles is cut along the tokens into `bigs` big items and then small ones; a
// segment of more than one item is joined by one CTA, whose table of (part, row) pairs lies in the shared memory of its tile rings.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define MXQ_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define MXQ_HOST_DEVICE inline
#endif

namespace mxq {

constexpr int kAttWarps = 4, kAttThreads = 32 * kAttWarps;
constexpr int kAttStages = 2;                  // tiles in a warp's ring
// The sizes of items.  An item costs about two tiles' time by itself, and the last ones leave CTAs idle for up to an item's time.  With
// kTwoSizes tiles or more per CTA, three quarters of every segment go into big items, drawn first, the rest into small ones of a tenth of a
// CTA's share, at least kSmallTiles (2 x 131071 tokens of 32 heads, 591 tiles per CTA, even weights: 249 us; all items of half a share, at
// most kItemTiles tiles: 269; 32 x 16384 tokens of 8 heads: 152 and 157).  A big one is three tenths of a share with one column block
// (4 x 16384 tokens of 32 heads: 87 us; kBigSmalls small ones, two thirds of a share there, 104; 2 x 131071 tokens, peaked weights: 269 and
// 276, even ones 249 and 247), but kBigSmalls small ones with two, whose results are twice as long to put together (even weights,
// 8 x 16384 tokens of 8 heads, 16 rows: 70 us, three tenths 86).
// Below kTwoSizes all items are of half a CTA's share, at most kItemTiles tiles (tree verification, 23 tiles per CTA: 36.5 us, two sizes 43.4;
// it goes the other way for one column block: 32 sequences of 279 to 8047 tokens, 40 per CTA, 39.0 us, two sizes 36.8).
// With less than kOneRound tiles per CTA items have that many, two per warp, the ring's depth: fewer would leave part of it empty.
constexpr uint32_t kTwoSizes = 96, kItemTiles = 48, kSmallTiles = 24, kBigSmalls = 4, kOneRound = 8;

// rows of the flattened (token row, head of the group) index per tile of nt column blocks; CTAs per SM
MXQ_HOST_DEVICE constexpr int att_rows(int nt) { return 8 * nt; }
MXQ_HOST_DEVICE constexpr int att_ctas_per_sm(int d, int nt) { return nt == 1 ? (d == 128 ? 3 : 4) : (d == 128 ? 2 : 3); }
// bytes of shared memory (the rings: a tile of head dimension d has 34 * d bytes); behind the join's table, 8 bytes per (part, row), 16 per
// thread for the sums where several threads share a row; so the most parts a segment may have
MXQ_HOST_DEVICE constexpr int att_smem(int d) { return kAttWarps * kAttStages * 34 * d; }
MXQ_HOST_DEVICE constexpr uint32_t att_max_parts(int d, int nt) { return (uint32_t)((att_smem(d) - kAttThreads * 16) / (att_rows(nt) * 8)); }

// Slots of the workspace, one per part of a cut segment.  No part but a segment's last is smaller than a small item, so a cut segment
// of n tiles has at most 2 n / small of them; a small item is at least a tenth of a CTA's share (rounded down, at least 24), which bounds
// all parts by 22 per CTA.
constexpr uint32_t kAttSlotsPerCta = 24;

struct AttSizes {
    uint32_t small, big;    // tiles of an item; big = 0: no big ones
};
MXQ_HOST_DEVICE AttSizes att_sizes(uint32_t share, int nt) {      // share: tiles of the call per CTA
    AttSizes z;
    if (share >= kTwoSizes) {
        const uint32_t tenth = share / 10 > kSmallTiles ? share / 10 : kSmallTiles;
        z.small = (tenth + kAttWarps - 1) / kAttWarps * kAttWarps;
        const uint32_t three = share * 3u / 10u / kAttWarps * kAttWarps;
        z.big = nt != 1 ? kBigSmalls * z.small : three > z.small ? three : z.small;
    } else {
        const uint32_t half = share / 2 + kAttWarps < kItemTiles ? share / 2 + kAttWarps : kItemTiles;
        z.small = share < kOneRound ? kOneRound : half / kAttWarps * kAttWarps;
        z.big = 0;
    }
    return z;
}

struct AttCut {               // of a segment
    uint32_t small, big;      // tiles of its items
    uint32_t bigs, parts;     // number of its big ones, of all
};
// A segment of n tiles.  Its parts fit the join's table: small items are raised until max_parts of them cover the segment, and as a
// big item is never smaller, it takes the place of one small one at least.  (With few segments a segment is hundreds of shares long:
// in one segment of head dimension 64, big items of three tenths of a share would give 1500 parts where 240 have room.)
MXQ_HOST_DEVICE AttCut att_cut(const AttSizes &z, uint32_t n, uint32_t max_parts) {
    AttCut k;
    const uint32_t least = (n + kAttWarps * max_parts - 1) / (kAttWarps * max_parts) * kAttWarps;
    k.small = z.small > least ? z.small : least;
    k.big = z.big > k.small ? z.big : k.small;
    k.bigs = z.big == 0 ? 0u : (n - n / 4) / k.big;
    const uint32_t rest = (n - k.bigs * k.big + k.small - 1) / k.small;
    k.parts = k.bigs + (rest > 1 ? rest : 1u);
    return k;
}

}  // namespace mxq
