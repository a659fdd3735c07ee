// Device helpers of the products whose rows choose their weights: conversions
// between float and the 16-bit types, and the tile that a workgroup takes of
// products whose sizes only the device knows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_device.h"
#include "igemm_rows_internal.h"

namespace igemm {
namespace rows {

// The 16 bits of x in type T (IGEMM_BF16 or IGEMM_F16), to nearest, ties to even.
template <int T>
__device__ __forceinline__ uint16_t to16(float x) {
    if constexpr (T == IGEMM_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <int T>
__device__ __forceinline__ float from16(uint16_t b) {
    if constexpr (T == IGEMM_BF16) return __builtin_bit_cast(float, (u32)b << 16);
    else return (float)__builtin_bit_cast(_Float16, b);
}

template <int T>
__device__ __forceinline__ void put(void *out, int64_t at, float x) {
    if constexpr (T == IGEMM_F32) ((float *)out)[at] = x;
    else ((uint16_t *)out)[at] = to16<T>(x);
}
template <int T>
__device__ __forceinline__ float get(const void *in, int64_t at) {
    if constexpr (T == IGEMM_F32) return ((const float *)in)[at];
    else return from16<T>(((const uint16_t *)in)[at]);
}
__device__ __forceinline__ void put(int type, void *out, int64_t at, float x) {
    if (type == IGEMM_F32) put<IGEMM_F32>(out, at, x);
    else if (type == IGEMM_BF16) put<IGEMM_BF16>(out, at, x);
    else put<IGEMM_F16>(out, at, x);
}

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

// Position i of a product: its rows of A and out, or -1 where it has none.
__device__ __forceinline__ void rows_of(const Product &p, int i, int *a, int *o) {
    const int s = p.order != nullptr ? p.order[i] : i;
    const int ra = p.slots == 0 ? i : (s >= 0 ? s / p.slots : -1);
    const int ro = p.scatter ? s : i;
    const bool ok = ra >= 0 && ra < p.a_rows && ro >= 0 && ro < p.out_rows && s >= 0;
    *a = ok ? ra : -1;
    *o = ok ? ro : -1;
}

}  // namespace rows
}  // namespace igemm
