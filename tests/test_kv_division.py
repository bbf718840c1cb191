"""How mxq_kv_attention divides its work (csrc/mxq_kv_division.h), checked on the host over the lengths, segments and GPUs there
can be: the parts of a segment fit the table that joins them, cover every tile once, and fit the workspace."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2503_13565_b200", "csrc", "mxq_kv_division.h")

SOURCE = r"""
#include <algorithm>
#include <random>
#include <vector>
#include "%s"
using namespace mxq;

// one call: segments n[i], times[i] of them; returns 0 or the number of the property that does not hold
static int check(int d, int nt, int sms, const std::vector<uint32_t> &n, const std::vector<uint32_t> &times) {
    const uint64_t grid = (uint64_t)sms * att_ctas_per_sm(d, nt);
    uint64_t work = 0, slots = 0;
    for (size_t i = 0; i < n.size(); ++i) work += (uint64_t)n[i] * times[i];
    const AttSizes z = att_sizes((uint32_t)std::min<uint64_t>(work / grid, 1u << 30), nt);
    if (z.small == 0 || z.small %% kAttWarps || z.big %% kAttWarps) return 1;         // every warp of a CTA has the same share of an item
    for (size_t i = 0; i < n.size(); ++i) {
        const AttCut k = att_cut(z, n[i], att_max_parts(d, nt));
        const uint64_t big = k.big, rows = att_rows(nt);
        if (k.small %% kAttWarps || big %% kAttWarps || k.small < z.small) return 2;
        // table of (maximum, sum) pairs, rounded up to 16 bytes, and the sums of all threads, in the rings' memory
        if ((k.parts * rows * 8 + 15) / 16 * 16 + kAttThreads * 16 > (uint64_t)att_smem(d)) return 3;
        const uint64_t smalls = k.parts - k.bigs, behind = k.bigs * big;
        if (k.bigs > k.parts || smalls < 1 || behind + smalls * k.small < n[i]) return 4;        // every tile in an item
        if (k.parts > 1 && behind + (smalls - 1) * k.small >= n[i]) return 5;                    // and no item without a tile
        if (z.big == 0 && k.bigs) return 6;
        if (k.parts > 1) slots += (uint64_t)k.parts * times[i];
    }
    return slots > kAttSlotsPerCta * grid ? 7 : 0;
}

extern "C" int sweep(int d, int nt, int sms, int64_t *where) {
    std::mt19937 rng(d + nt + sms);
    auto report = [&](int what, uint32_t n, uint32_t segs) { where[0] = n, where[1] = segs; return what; };
    std::vector<uint32_t> lengths;
    for (uint32_t n = 1; n <= 4096; ++n) lengths.push_back(n);
    for (double x = 4096; x < (1 << 26); x *= 1.01) lengths.push_back((uint32_t)x + rng() %% 8);        // (2^26 tiles: 2^31 tokens)
    for (uint32_t n : lengths)
        for (uint32_t segs = 1; segs <= 64; segs += segs < 16 ? 1 : 7)                                  // the same length in every segment
            if (int w = check(d, nt, sms, {n}, {segs})) return report(w, n, segs);
    for (int i = 0; i < 200000; ++i) {                                                                  // batches of different lengths
        const int count = 1 + rng() %% 12;
        std::vector<uint32_t> n, times;
        const uint32_t bits = 2 + rng() %% 21;
        for (int s = 0; s < count; ++s) n.push_back(1 + rng() %% (1u << (1 + rng() %% bits))), times.push_back(1 + rng() %% (i %% 3 ? 4 : 256));
        if (int w = check(d, nt, sms, n, times)) return report(w, n[0], times[0]);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def sweep(tmp_path_factory):
    gxx = shutil.which("g++")
    assert gxx, "the CUDA build needs g++ too"
    where = tmp_path_factory.mktemp("division")
    src, lib = str(where / "sweep.cpp"), str(where / "sweep.so")
    with open(src, "w") as f:
        f.write(SOURCE % HEADER)
    subprocess.run([gxx, "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", src, "-o", lib], check=True)
    return ctypes.CDLL(lib).sweep


WHAT = {1: "a call's item sizes", 2: "a segment's item sizes", 3: "more parts than the join's table holds", 4: "tiles in no item",
        5: "an item without tiles", 6: "big items in a small call", 7: "more parts than the workspace has slots"}


@pytest.mark.parametrize("sms", [132, 148, 160])
@pytest.mark.parametrize("nt", [1, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_parts_cover_the_tiles_and_fit_their_memory(sweep, d, nt, sms):
    where = (ctypes.c_int64 * 2)()
    rc = sweep(d, nt, sms, where)
    assert rc == 0, "%s: %d tiles, %d segments" % (WHAT[rc], where[0], where[1])
