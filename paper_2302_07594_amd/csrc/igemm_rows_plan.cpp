// The choices of the products whose rows choose their weights: tile, k slices and
// workspace, by sizes and alignment (host code, no HIP).
#include <stdint.h>

#include "igemm_rows_internal.h"

namespace igemm {
namespace rows {
namespace {

int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

}  // namespace

// What the device will find is taken to be even: `used` groups of `avg` rows.
Choice choose(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters, int64_t rank,
              int num_cu) {
    Choice c = {};
    const int64_t used = groups < rows ? groups : rows;
    const int64_t avg = ceil_div(rows, used);
    auto tiles = [&](int64_t bm, int64_t bn) { return ceil_div(avg, bm) * used * ceil_div(n, bn); };
    // share of the last round of workgroups (`at` at a time) that has work
    auto full = [](int64_t t, int64_t at) { return (double)t / (double)(ceil_div(t, at) * at); };
    if (avg <= 32) {
        c.bm = 32, c.bn = 256;
    } else if (avg <= 64 || tiles(128, 128) < num_cu) {
        c.bm = 64, c.bn = 128;
    } else if (avg >= 192 && (adapters == 0 || rank <= 16) &&
               full(tiles(256, 256), num_cu) >= 0.9 * full(tiles(128, 128), 2 * num_cu)) {
        c.bm = 256, c.bn = 256;
    } else {
        c.bm = 128, c.bn = 128;
    }
    // Fewer tiles than compute units: narrower and shorter ones, then k slices, with
    // adapters for few rows only (join_slices reads `up` once a row).
    c.by_row = adapters > 0 && rank > 0 && rows * rank <= 4096;
    const bool adapt = adapters > 0 && rank > 0;
    int64_t slices = 1;
    if (c.bm <= 64 && tiles(c.bm, c.bn) < num_cu) {
        c.bn = 128;
        if (adapt && !c.by_row) c.bm = 32;
    }
    if (c.bm <= 64 && tiles(c.bm, c.bn) < num_cu && (!adapt || c.by_row)) {
        const int64_t t = tiles(c.bm, 128);
        if (2 * t <= num_cu) slices = num_cu / t;
        if (slices > k / 256) slices = k / 256;
        if (slices > 16) slices = 16;
        if (slices < 1) slices = 1;
    }
    int64_t chunk = ceil_div(ceil_div(k, slices), kStepK) * kStepK;
    if (chunk < kStepK) chunk = kStepK;
    c.kchunk = (int)chunk;
    c.slices = k > 0 ? (int)ceil_div(k, chunk) : 1;
    if (c.slices > 1) c.part_bytes = up256(c.slices * rows * n * 4);
    if (adapt) {
        c.rpad = (int)(ceil_div(rank, 32) * 32);  // (a row's 32 ranks: one line)
        c.ks = c.slices > 1 ? (int)ceil_div(k, kShrinkK) : 1;
        // 32 ranks a workgroup (8192 rows of 4096, rank 64: 49 us, with 16 ranks 55), or
        // 16 where 32 would leave compute units idle.
        c.shrink_ranks =
            rank > 16 && ceil_div(rows, kShrinkRows) * ceil_div(rank, 32) >= num_cu ? 32 : 16;
        c.u_bytes = up256(c.ks * rows * c.rpad * 4);
    }
    return c;
}

int64_t product_workspace(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters,
                          int64_t rank, int num_cu) {
    const Choice c = choose(rows, n, k, groups, adapters, rank, num_cu);
    return c.part_bytes + c.u_bytes;
}

Tile tile_of(const Choice &c, const Product &p, const Adapters &ad, int num_cu) {
    // By DMA where rows start at 4-byte addresses and the offsets of a whole last
    // k-tile stay below 4 GiB; else through registers, in tiles that have the
    // registers for it.
    const bool reg = (uintptr_t)p.A % 4 != 0 || (uintptr_t)p.B % 4 != 0 || p.lda % 4 != 0 ||
                     p.ldb % 4 != 0 || p.stride_b % 4 != 0 ||
                     ((int64_t)p.k + kStepK) * p.ldb > 0xffffffffll ||
                     (ad.adapters > 0 && c.bm == 256 &&
                      ((uintptr_t)ad.up % 4 != 0 || ad.ld_up % 2 != 0 || ad.stride_up % 2 != 0 ||
                       (int64_t)p.rows * c.rpad * 4 > 0x7fffffff));
    int bm = c.bm, bn = c.bn;
    if (reg && bm >= 64) bn = 128;
    if (reg && bm == 256) bm = 128;
    // (through registers a workgroup waits more for its loads: 13 experts, 1554 rows,
    // 1111 x 1777, in 32 rows 20.5 us, in 64 24.0)
    if (reg && bm == 64 && c.slices == 1 &&
        most_tiles(p.rows, p.groups, 64) * ceil_div(p.n, 128) < 2 * num_cu)
        bm = 32;
    return Tile{bm, bn, reg};
}

}  // namespace rows
}  // namespace igemm
