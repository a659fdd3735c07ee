// Which tile a workgroup takes of products whose sizes only the device knows: integer
// arithmetic on the offsets and exchanges between the lanes of a wave. The includer
// declares these (HIP's for the kernels, others where it is built for the host).
#pragma once

#include <stdint.h>

#include "igemm_rows_internal.h"

namespace igemm {
namespace rows {

// Row tiles of a grouped product. Tiles of `bm` rows are numbered group after
// group; `pre` is the number of tiles before the group found, `lo` its first
// position and `cnt` its positions. All lanes of a wave call together and get
// the same answer; total (all row tiles) is what the numbers run up to.
struct Found {
    int group, pre, lo, cnt;
};
__device__ __forceinline__ void group_span(const Product &p, int g, int *lo, int *cnt) {
    if (p.offsets == nullptr) {
        *lo = 0;
        *cnt = p.rows;
        return;
    }
    const int a = min(max(p.offsets[g], 0), p.rows), b = min(max(p.offsets[g + 1], 0), p.rows);
    *lo = a;
    *cnt = max(b - a, 0);
}
// Each lane takes a run of consecutive groups; `mine` are its tiles and `before`
// the tiles of the lanes below it. Offsets that ascend give fewer than kMostTiles;
// the sums of others stop there, before they could wrap to a negative number.
constexpr int kMostTiles = 1 << 27;
constexpr int kMostBlocks = 1 << 24;  // (2^32 threads, 256 a workgroup at least)
__device__ __forceinline__ int wave_tiles(const Product &p, int bm, int per, int lane,
                                          int *before) {
    int mine = 0;
    for (int g = lane * per; g < min((lane + 1) * per, p.groups); ++g) {
        int lo, cnt;
        group_span(p, g, &lo, &cnt);
        mine = min(mine + (cnt + bm - 1) / bm, kMostTiles);
    }
    int sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int up = __shfl_up(sum, d);
        if (lane >= d) sum = min(sum + up, kMostTiles);
    }
    *before = sum - mine;
    return __builtin_amdgcn_readlane(sum, 63);
}
// The group that holds row tile t < total; cnt 0 if offsets that do not ascend leave
// none.
__device__ __forceinline__ Found wave_find(const Product &p, int bm, int per, int lane, int before,
                                           int t) {
    // the last lane whose tiles begin at or before t and that has any
    int next = __shfl_down(before, 1);
    if (lane == 63) next = 0x7fffffff;
    const uint64_t here = __ballot(before <= t && next > t);
    const int owner =
        __builtin_amdgcn_readfirstlane(max(__ffsll((unsigned long long)here) - 1, 0));
    Found f = {0, __builtin_amdgcn_readlane(before, owner), 0, 0};
    for (int g = owner * per; g < min((owner + 1) * per, p.groups); ++g) {
        int lo, cnt;
        group_span(p, g, &lo, &cnt);
        const int tiles = (cnt + bm - 1) / bm;
        if (t < f.pre + tiles) {
            f.group = g;
            f.lo = lo;
            f.cnt = cnt;
            break;
        }
        f.pre += tiles;
    }
    return f;
}

// The tile of workgroup `block`: rows m0 .. of group f's positions, columns n0 .. and k
// slice z; f.cnt 0: none.
struct Place {
    Found f;
    int m0, n0, z;
};
__device__ __forceinline__ Place place_of(const Product &p, int bm, int bn, int slices, int lane,
                                          int block) {
    Place w = {{0, 0, 0, 0}, 0, 0, 0};
    const int tiles_n = (p.n + bn - 1) / bn;
    const int per = (p.groups + 63) / 64;
    int before;
    const int row_tiles = wave_tiles(p, bm, per, lane, &before);
    // Workgroup ids go to the eight XCDs in turn: each takes a contiguous range
    // of the tiles, so that tiles that run together share A and B in its L2.
    // (A grid has fewer than kMostBlocks workgroups, which is what offsets that ascend
    // need at most. Others can make of row_tiles, tiles_n and slices more than an int
    // holds: their tiles stop there, and everything below stays under it.)
    const int total = (int)min((int64_t)row_tiles * tiles_n * slices, (int64_t)kMostBlocks);
    int at;
    {
        const int q = total >> 3, r = total & 7, x = block & 7, i = block >> 3;
        if (i >= q + (x < r)) return w;
        at = x * q + min(x, r) + i;
    }
    w.z = at % slices;
    const int t = at / slices;
    w.f = wave_find(p, bm, per, lane, before, t / tiles_n);
    if (w.f.cnt == 0) return w;
    // Within a group: eight row tiles at a time, over all columns.
    const int mt = (w.f.cnt + bm - 1) / bm;
    const int in = t - w.f.pre * tiles_n, span = 8 * tiles_n;
    const int first = in / span * 8, gsize = min(mt - first, 8);
    const int rest = in - in / span * span;
    w.m0 = (first + rest % gsize) * bm;
    w.n0 = rest / gsize * bn;
    return w;
}

}  // namespace rows
}  // namespace igemm
