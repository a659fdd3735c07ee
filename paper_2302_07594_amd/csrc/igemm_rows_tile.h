// Tile kernel of the experts' products and of the shared projection with
// adapters: out rows = scales * (A rows . B of the row's group) (+ adapters).
//
// The inner product is the ring kernel's (igemm_ring.h): A and B move into
// LDS as they lie, by buffer DMA where rows start at 4-byte addresses, else
// through registers; B is turned k-contiguous by the transpose reads. What
// differs:
//   * the grid covers the most row tiles that the sizes allow, and a workgroup
//     finds its group and rows from the offsets on the device (one wave scan);
//     workgroups past the last tile leave at once, so nothing is read back by
//     the host;
//   * a lane's DMA address takes its row of A from the plan, so gathering rows
//     costs nothing more than reading consecutive ones;
//   * the sums are int32 and exact (k <= 131071); they are scaled in float,
//     turned to rows of 16-byte pieces through LDS and stored once, where the
//     raw sums would cost two more passes over four bytes an element.
// Few rows an expert are bound by reading B (512 tokens of 8 slots, 64 experts of 2048 x
// 1024, bf16: 43 us, 3.6 TB/s). Many are bound by how full their row tiles are (32768 rows,
// 64 experts of 4096 x 2048: 0.81 as routed, 365 us, 1510 TOPS; experts of 512 rows each 320,
// 1710) and by the short k, whose tiles start and end with nothing else under way (one weight,
// 8192 x 11008 x 4096: 1940 TOPS).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_ring.h"
#include "igemm_rows_device.h"

namespace igemm {
namespace rows {

using lds::tr8;
using lds::v2i;
using ring::v4u;

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8hf __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int as_int(float x) { return __builtin_bit_cast(int, x); }
__device__ __forceinline__ float as_float(int x) { return __builtin_bit_cast(float, x); }

// The bits of x with the magnitude one step smaller (0: as it is). Of an infinity it is the
// largest finite number.
__device__ __forceinline__ u32 below(float x, bool nonzero) {
    return __builtin_bit_cast(u32, x) - (nonzero ? 1u : 0u);
}

// 8 values as bf16 parts hi + mid + lo, cut from the value just below x and from what is
// then just below the rest: x exactly (8 leading bits, 8 more, the last ones), and no
// part of a number is 0. An infinite weight therefore makes an infinity of the
// product's sign of each part, where a part of 0 would make NaN; of an infinite x, the
// parts are two finite numbers and an infinity. (|x| of 2^-100 or more: lo is at least
// 2^-32 of it, and bf16 goes down to 2^-133. NaN is NaN in every part.)
__device__ __forceinline__ void split3(const float *x, v8bf &hi, v8bf &mid, v8bf &lo) {
    u32 h[4], m[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        u32 top[2], rest[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const bool nonzero = x[e + q] != 0.0f;
            top[q] = below(x[e + q], nonzero);
            const float r = x[e + q] - __builtin_bit_cast(float, top[q] & 0xffff0000u);
            rest[q] = below(r, nonzero);
            lo[e + q] = (__bf16)(r - __builtin_bit_cast(float, rest[q] & 0xffff0000u));
        }
        h[e / 2] = perm(top[1], top[0], 0x07060302u);
        m[e / 2] = perm(rest[1], rest[0], 0x07060302u);
    }
    hi = __builtin_bit_cast(v8bf, h);
    mid = __builtin_bit_cast(v8bf, m);
}

// 8 float16 values as bf16 parts hi + lo, exactly: their leading 8 bits and the last 3. An
// infinite or NaN value is its hi alone. (lo may be 0: it is multiplied only with the
// upper two parts of split3, which are finite.)
__device__ __forceinline__ void split2(v8hf x, v8bf &hi, v8bf &lo) {
    u32 h[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        u32 top[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float f = (float)x[e + q];
            top[q] = __builtin_bit_cast(u32, f);
            const float r = f - __builtin_bit_cast(float, top[q] & 0xffff0000u);
            lo[e + q] = (__bf16)(r == r ? r : 0.0f);
        }
        h[e / 2] = perm(top[1], top[0], 0x07060302u);
    }
    hi = __builtin_bit_cast(v8bf, h);
}

// 8 consecutive 16-bit values of a row of `len`, from element e0 >= 0; zero from
// `used` (<= len) on. No branch but on len: loads under branches wait for each other.
__device__ __forceinline__ void load8(const uint16_t *row, int e0, int len, int used, u32 w[4]) {
    if (len >= 8) {
        const v4i v = ring::load_edge((const char *)row, 2 * e0, 2 * len, false);
        w[0] = (u32)v.x;
        w[1] = (u32)v.y;
        w[2] = (u32)v.z;
        w[3] = (u32)v.w;
    } else {
        u32 x[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = row[min(e0 + q, max(len - 1, 0))];
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = x[2 * q] | x[2 * q + 1] << 16;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int left = used - e0 - 2 * q;
        w[q] = left >= 2 ? w[q] : (left == 1 ? w[q] & 0xffffu : 0u);
    }
}

__device__ __forceinline__ int rank_of(const Adapters &ad, int which) {
    if (which < 0 || which >= ad.adapters) return 0;
    return ad.ranks != nullptr ? min(max(ad.ranks[which], 0), ad.rank) : ad.rank;
}

// u = scaling scale_a A down^T for few rows or few ranks: row i and k slice z (of
// kslice) by one workgroup, every wave four ranks at a time, 16 bytes of `down` a
// lane. What it reads of `down` is one adapter a row, whichever the row's is, so
// a batch of 16 requests with an adapter each takes as long as one with a shared
// one. Ranks [r0, r0 + 4 WAVES) of the row; those up to rpad that the adapter does not
// have are zeros.
template <int WAVES, int T>
__device__ void shrink_row(const Product &p, const Adapters &ad, float *__restrict__ u, int rpad,
                           int kslice, int i, int z, int block) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int which = ad.ids[i];
    const int rank = rank_of(ad, which), r0 = 4 * (block * WAVES + wave);
    float *row = u + ((int64_t)z * p.rows + i) * rpad;
    if (r0 >= rank) {  // (the whole wave)
        if (rank > 0 && lane < 4 && r0 + lane < rpad) row[r0 + lane] = 0.0f;
        return;
    }
    const int8_t *a = p.A + (int64_t)i * p.lda;
    float f = p.scale_a != nullptr ? p.scale_a[i] : 1.0f;
    if (ad.scaling != nullptr) f *= ad.scaling[which];
    const uint16_t *down = (const uint16_t *)ad.down + which * ad.stride_down;
    const int kb = z * kslice, ke = min(p.k, kb + kslice);
    constexpr int PASS = 2;  // of 64 lanes x 8 k, all their loads in flight together
    float s[4] = {};
    for (int k0 = kb; k0 < ke; k0 += 512 * PASS) {
        u32 x[PASS][2], w[4][PASS][4];
        const bool whole = k0 + 512 * PASS <= ke;
#pragma unroll
        for (int q = 0; q < PASS; ++q) {
            const int e0 = k0 + 512 * q + 8 * lane;
            if (whole) {
                __builtin_memcpy(x[q], a + e0, 8);
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    __builtin_memcpy(w[b][q], down + min(r0 + b, rank - 1) * ad.ld_down + e0, 16);
            } else {
                const v4i v = ring::load_edge((const char *)a, e0, p.k, p.k < 16);
                x[q][0] = (u32)v.x;
                x[q][1] = (u32)v.y;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    load8(down + min(r0 + b, rank - 1) * ad.ld_down, e0, p.k, ke, w[b][q]);
            }
        }
#pragma unroll
        for (int q = 0; q < PASS; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xe = (float)(int8_t)(x[q][e >> 2] >> (8 * (e & 3)));
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const uint16_t v = (uint16_t)(w[b][q][e / 2] >> (16 * (e & 1)));
                    s[b] = fmaf(xe, from16<T>(v), s[b]);
                }
            }
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2)
#pragma unroll
        for (int b = 0; b < 4; ++b) s[b] += __shfl_xor(s[b], o);
    if (lane == 0)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (r0 + b < rpad) row[r0 + b] = r0 + b < rank ? s[b] * f : 0.0f;
}

// BM x BN: the workgroup's tile, WM x WN a wave's; NST ring stages; OCC
// workgroups a compute unit; REG: through registers; PART: the raw sums of k
// slice z go to part[z][position][column] instead; ADAPT: adapters beside, of this
// weight type (0: none), u being rows x rpad floats.
//
// A sliced product's adapters (PART and ADAPT): the first rows x ks x (rank blocks)
// workgroups compute u in ks parts, one a k slice of kshrink (shrink_row), beside the
// product's.
template <int BM, int BN, int WM, int WN, int NST, int OCC, bool REG, bool PART, int ADAPT>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64, OCC *((BM / WM) * (BN / WN)) / 4)
rows_tile(Product p, Adapters ad, float *__restrict__ u, int ks, int kshrink, int rpad,
          int32_t *__restrict__ part, int slices, int kchunk) {
    typedef Mfma<32> M;
    constexpr int TM = WM / 32, TN = WN / 32;
    constexpr int WGN = BN / WN, NW = (BM / WM) * WGN;
    constexpr int BK = kStepK, RA = BK, RB = BN;
    constexpr int APL = BM * RA, BPL = BK * RB, STAGE = APL + BPL;
    constexpr int RPA = 1024 / RA, RPB = 1024 / RB;
    static_assert(APL % (1024 * NW) == 0 && BPL % (1024 * NW) == 0, "1 KB blocks per wave");
    constexpr int DPA = APL / 1024 / NW, DPB = BPL / 1024 / NW, DPW = DPA + DPB;
    static_assert(NST >= 2 && (NST - 2) * DPW < 64, "outstanding DMA count");
    static_assert(!REG || NST == 2, "two stages through registers");
    // A wave's output block: 32 rows x JB blocks of 32 columns at a time (the
    // registers beside the sums), in pieces of 16 bytes.
    constexpr int JB = TN < 2 ? TN : 2, PITCH = 32 * JB * 4 + 16;
    constexpr int SMEM = NST * STAGE > NW * 32 * PITCH ? NST * STAGE : NW * 32 * PITCH;
    static_assert(TN % JB == 0, "whole output blocks");
    static_assert(OCC * (SMEM + 24 * BM + 4 * BN + 16) <= 160 * 1024, "LDS");

    __shared__ __attribute__((aligned(1024))) char smem[SMEM];
    __shared__ __attribute__((aligned(16))) int arow[BM], orow[BM], arow_id[BM];
    __shared__ __attribute__((aligned(16))) float arow_s[BM], bcol_s[PART ? 4 : BN];
    // The adapters of the tile's rows, each once, and their ranks (256 rows).
    constexpr bool XT = ADAPT != 0 && !REG && !PART && BM == 256;
    __shared__ int uniq[XT ? BM : 1], uniq_rank[XT ? BM : 1], uniq_n;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;

    int first = 0;
    if constexpr (PART && ADAPT != 0) {
        const int blocks = rpad / (4 * NW);
        first = p.rows * ks * blocks;
        if ((int)blockIdx.x < first) {
            const int i = (int)blockIdx.x % p.rows, x = (int)blockIdx.x / p.rows;
            shrink_row<NW, ADAPT>(p, ad, u, rpad, kshrink, i, x / blocks, x % blocks);
            return;
        }
    }

    // ---- which tile -----------------------------------------------------------
    const Place at = place_of(p, BM, BN, slices, lane, (int)blockIdx.x - first);
    const Found f = at.f;
    if (f.cnt == 0) return;
    const int m0 = at.m0, n0 = at.n0, z = at.z;
    const int mrows = min(f.cnt - m0, BM);
    const int kbeg = z * kchunk, klen = min(p.k - kbeg, kchunk);
    const int nkt = (klen + BK - 1) / BK;

    // The rows of the tile: the threads that cover them, a wave or two, read the
    // plan while the others already fetch B.
    auto fetch_rows = [&]() __attribute__((always_inline)) {
        for (int r = tid; r < BM; r += NW * 64) {
            int a = -1, o = -1;
            if (r < mrows) rows_of(p, f.lo + m0 + r, &a, &o);
            arow[r] = a;
            orow[r] = o;
            if constexpr (ADAPT != 0 && !PART) {
                const int w = a >= 0 ? ad.ids[a] : -1;
                arow_id[r] = w >= 0 && w < ad.adapters ? w : -1;
            }
        }
    };
    if constexpr (REG) {
        fetch_rows();
        __syncthreads();
    }
    // What the output needs of each row and column, fetched behind the first
    // k-tiles.
    auto terms = [&]() __attribute__((always_inline)) {
        if constexpr (PART) return;
        for (int c = tid; c < BN; c += NW * 64)
            bcol_s[c] = p.scale_b != nullptr && n0 + c < p.n
                            ? p.scale_b[(int64_t)f.group * p.n + n0 + c]
                            : 1.0f;
        for (int r = tid; r < BM; r += NW * 64) {
            const int a = arow[r];
            arow_s[r] = a >= 0 && p.scale_a != nullptr ? p.scale_a[a] : 1.0f;
        }
        if constexpr (XT) {
            if (wave == 0) {
                int n = 0;
                for (int r0 = 0; r0 < mrows; r0 += 64) {
                    int id = r0 + lane < BM ? arow_id[min(r0 + lane, BM - 1)] : -1;
                    for (int q = 0; q < n; ++q) id = id == uniq[q] ? -1 : id;
                    uint64_t todo = __ballot(id >= 0);
                    while (todo != 0) {
                        const int which = __builtin_amdgcn_readlane(
                            id, __ffsll((unsigned long long)todo) - 1);
                        todo &= ~__ballot(id == which);
                        const int rank = rank_of(ad, which);
                        if (lane == 0 && rank > 0) {
                            uniq[n] = which;
                            uniq_rank[n] = rank;
                        }
                        n += rank > 0;
                    }
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                }
                if (lane == 0) uniq_n = n;
            }
        }
    };

    // ---- staging ----------------------------------------------------------------
    int a_row[DPA], a_lc[DPA], b_row[DPB], b_lc[DPB];
#pragma unroll
    for (int d = 0; d < DPA; ++d) {
        a_row[d] = (wave * DPA + d) * RPA + lane / (RA / 16);
        a_lc[d] = (lane % (RA / 16)) ^ (REG ? 0 : ring::swz_a<RA>(a_row[d]));
    }
#pragma unroll
    for (int d = 0; d < DPB; ++d) {
        b_row[d] = (wave * DPB + d) * RPB + lane / (RB / 16);
        b_lc[d] = (lane % (RB / 16)) ^ (REG ? 0 : ring::swz_b<RB>(b_row[d]));
    }
    const int lda = (int)p.lda, ldb = (int)p.ldb;
    const char *a_base = (const char *)p.A + kbeg;
    const char *b_base = (const char *)p.B + f.group * p.stride_b + (int64_t)kbeg * ldb + n0;
    const u32 lds0 = (u32)(uintptr_t)(const __attribute__((address_space(3))) char *)smem;

    u32 a_vo[DPA], b_vo[DPB];
    v4u Ars = {0u, 0u, 0u, 0u}, Brs = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int d = 0; d < DPB; ++d) b_vo[d] = (u32)b_row[d] * (u32)ldb + 16u * (u32)b_lc[d];
    auto place_a = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DPA; ++d) {
            const int a = arow[a_row[d]];
            a_vo[d] = a >= 0 ? (u32)a * (u32)lda + 16u * (u32)a_lc[d] : 0x80000000u;
        }
    };
    if constexpr (!REG) {
        // B's resource ends with its k range: rows beyond are zeros, so what A
        // has beyond the range, or in rows with nothing to do, never counts.
        Ars = ring::resource(a_base, (u32)(((int64_t)(p.a_rows - 1) * lda + p.k - kbeg + 3) & ~3));
        Brs = ring::resource(b_base, (u32)(((int64_t)(klen - 1) * ldb + p.n - n0 + 3) & ~3));
    }
    // The adapters' k-tiles follow the product's: two units of 16 ranks of one adapter
    // each (of different ones, where one ends), u (floats, 64 bytes a row and unit, as
    // half a row of A) against `up` (32 bytes a column and unit).
    struct Unit {
        int q, e0;        // adapter uniq[q], first rank
        int which, rank;  // that adapter and its rank; which -2: no more units
    };
    auto unit_of = [&](int q) __attribute__((always_inline)) -> Unit {
        Unit x = {q, 0, -2, 0};
        if constexpr (XT) {
            if (q < __builtin_amdgcn_readfirstlane(uniq_n)) {
                x.which = __builtin_amdgcn_readfirstlane(uniq[q]);
                x.rank = __builtin_amdgcn_readfirstlane(uniq_rank[q]);
            }
        }
        return x;
    };
    auto next = [&](Unit x) __attribute__((always_inline)) -> Unit {
        x.e0 += 16;
        return x.e0 < x.rank || x.which < 0 ? x : unit_of(x.q + 1);
    };
    auto issue_extra = [&](Unit x, int s) __attribute__((always_inline)) {
        if constexpr (XT) {
            const Unit y = next(x);
            const int w0 = x.which, w1 = y.which;
            const v4u ur = ring::resource((const char *)u,
                                          w0 >= 0 ? (u32)(p.rows * rpad * 4) : 0u);
            const u32 up_bytes = (u32)((((int64_t)(p.n - 1) * ad.ld_up + ad.rank) * 2 + 3) & ~3);
            const u32 base = lds0 + (u32)(s * STAGE);
#pragma unroll
            for (int d = 0; d < DPB; ++d) {
                // 1 KB: 32 columns of two 16-byte chunks, unit after unit
                const int b = wave * DPB + d;
                const bool second = b >= BN / 32;
                const int w = second ? w1 : w0, e0 = second ? y.e0 : x.e0;
                const int col = (b * 32 + (lane >> 1)) % BN;
                const int lc = (lane & 1) ^ ((col >> 3) & 1);
                const v4u br = ring::resource(
                    (const char *)((const uint16_t *)ad.up + max(w, 0) * ad.stride_up),
                    w >= 0 && b < BN / 16 ? up_bytes : 0u);
                ring::dma((u32)min(n0 + col, p.n - 1) * (u32)(ad.ld_up * 2) +
                              (u32)(e0 * 2 + 16 * lc),
                          br, base + (u32)(APL + b * 1024));
            }
#pragma unroll
            for (int d = 0; d < DPA; ++d) {
                const int r = a_row[d], w = a_lc[d] < 4 ? w0 : w1;
                const int e = (a_lc[d] < 4 ? x.e0 : y.e0) + 4 * (a_lc[d] & 3);
                ring::dma(arow_id[r] == w ? (u32)max(arow[r], 0) * (u32)(rpad * 4) + 4u * (u32)e
                                          : 0x80000000u,
                          ur, base + (u32)((wave * DPA + d) * 1024));
            }
        }
    };
    // k-tile kt into stage s. Tiles past the range are issued too, on empty
    // resources, so that every wave counts DPB + DPA DMAs a tile.
    auto issue_b = [&](int kt, int s) __attribute__((always_inline)) {
        v4u br = Brs;
        br.z = kt < nkt ? br.z : 0u;
        const u32 bs = kt < nkt ? (u32)(kt * BK) * (u32)ldb : 0u;
        const u32 base = lds0 + (u32)(s * STAGE);
#pragma unroll
        for (int d = 0; d < DPB; ++d)
            ring::dma(b_vo[d] + bs, br, base + (u32)(APL + (wave * DPB + d) * 1024));
    };
    auto issue_a = [&](int kt, int s) __attribute__((always_inline)) {
        v4u ar = Ars;
        ar.z = kt < nkt ? ar.z : 0u;
        const u32 as = kt < nkt ? (u32)(kt * BK) : 0u;
        const u32 base = lds0 + (u32)(s * STAGE);
#pragma unroll
        for (int d = 0; d < DPA; ++d)
            ring::dma(a_vo[d] + as, ar, base + (u32)((wave * DPA + d) * 1024));
    };
    auto issue = [&](int kt, int s) __attribute__((always_inline)) {
        issue_b(kt, s);
        issue_a(kt, s);
    };

    // Through registers: bounded loads of any alignment.
    typedef v4i regs_a[REG ? DPA : 1];
    typedef v4i regs_b[REG ? DPB : 1];
    auto load = [&](regs_a &va, regs_b &vb, int kt) __attribute__((always_inline)) {
        if constexpr (REG) {
            const int k0 = kt * BK, left = klen - k0;
            const char *bk = b_base + (int64_t)k0 * ldb;
            // A k-tile inside both matrices takes plain loads, all in flight at
            // once. (What A's rows have past the k range meets zeros of B.)
            const bool inside = k0 + BK <= klen &&
                                (int64_t)(kbeg + k0 + BK - 1) * ldb + n0 + BN <=
                                    (int64_t)(p.k - 1) * ldb + p.n;
            if (inside) {
#pragma unroll
                for (int d = 0; d < DPA; ++d)
                    va[d] = ring::load_u16(a_base + (u32)(max(arow[a_row[d]], 0) * lda + k0 +
                                                          16 * a_lc[d]));
#pragma unroll
                for (int d = 0; d < DPB; ++d)
                    vb[d] = ring::load_u16(bk + (u32)(b_row[d] * ldb + 16 * b_lc[d]));
                return;
            }
            const int a_end = (int)((int64_t)(p.a_rows - 1) * lda + p.k - kbeg);
            const bool a_tiny = (int64_t)(p.a_rows - 1) * lda + p.k < 16;
            const bool b_tiny = (int64_t)(p.k - 1) * ldb + p.n < 16;
            const int b_end =
                (int)min((int64_t)(p.k - 1 - kbeg - k0) * ldb + p.n - n0, (int64_t)0x7fffffff);
#pragma unroll
            for (int d = 0; d < DPA; ++d) {
                const int a = max(arow[a_row[d]], 0);
                va[d] = ring::load_edge(a_base, a * lda + k0 + 16 * a_lc[d], a_end, a_tiny);
            }
#pragma unroll
            for (int d = 0; d < DPB; ++d) {
                const int off = min(b_row[d], left - 1) * ldb + 16 * b_lc[d];
                vb[d] = ring::load_edge(bk, off, b_end, b_tiny);
                if (b_row[d] >= left) vb[d] = v4i{0, 0, 0, 0};
            }
        }
    };
    auto store = [&](const regs_a &va, const regs_b &vb, int s) __attribute__((always_inline)) {
        if constexpr (REG) {
            char *sa = smem + s * STAGE, *sb = sa + APL;
#pragma unroll
            for (int d = 0; d < DPA; ++d)
                *(v4i *)(sa + a_row[d] * RA + 16 * (a_lc[d] ^ ring::swz_a<RA>(a_row[d]))) = va[d];
#pragma unroll
            for (int d = 0; d < DPB; ++d)
                *(v4i *)(sb + b_row[d] * RB + 16 * (b_lc[d] ^ ring::swz_b<RB>(b_row[d]))) = vb[d];
        }
    };

    // ---- fragments and matrix instructions (as the ring kernel's) -----------------
    constexpr int KS = BK / 32;
    const int fr = lane & 31, gq = lane >> 4, ul = lane & 15;
    int a_rd[KS], b_rd[TN];
    {
        const int row = wm0 + fr, krow = 16 * (gq >> 1) + (ul >> 1);
#pragma unroll
        for (int s = 0; s < KS; ++s)
            a_rd[s] = row * RA + 16 * ((2 * s + (lane >> 5)) ^ ring::swz_a<RA>(row));
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int cb = wn0 + 32 * j + 16 * (gq & 1) + 8 * (ul & 1);
            b_rd[j] = APL + krow * RB + 16 * ((cb >> 4) ^ ring::swz_b<RB>(krow)) + (cb & 15);
        }
    }
    v16i acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    // B's fragment is the left operand: a lane then holds one row of the block (lane %
    // 32) and, register by register, columns 8 (r / 4) + 4 (lane / 32) + r % 4, four
    // consecutive ones that leave in one write; scales and adapters of a row are a
    // lane's own.
    // A wave whose rows or columns all lie outside leaves the matrix cores to the
    // others (the last row tile of a group is part empty).
    const bool busy = wm0 < mrows && n0 + wn0 < p.n;
    auto tile = [&](int s) __attribute__((always_inline)) {
        if (!busy) return;
        const char *st = smem + s * STAGE;
#pragma unroll
        for (int q = 0; q < KS; ++q) {
            v4i a[TM], b[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const char *at_b = st + b_rd[j] + q * 32 * RB;
                const v2i x = tr8(at_b), y = tr8(at_b + 8 * RB);
                b[j] = v4i{x.x, x.y, y.x, y.y};
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = *(const v4i *)(st + a_rd[q] + i * 32 * RA);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = M::mma(b[j], a[i], acc[i][j]);
        }
    };
    // The scaled sums take the places of the raw ones.
    auto scale = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const float sa = arow_s[wm0 + 32 * i + fr];
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 s =
                        *(const float4 *)(bcol_s + wn0 + 32 * j + M::out_row(lane, r));
                    const float sb[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[i][j][r + q] = as_int((float)acc[i][j][r + q] * sa * sb[q]);
                }
        }
    };
    auto tile_extra = [&](Unit x, int s) __attribute__((always_inline)) {
        if constexpr (XT) {
            if (!busy) return;
            const char *st = smem + s * STAGE;
            const int half = lane >> 5;
#pragma unroll 1
            for (int h = 0; h < 2 && x.which >= 0; ++h, x = next(x)) {
                const int which = x.which, left = x.rank - x.e0;
                // what lies beyond the adapter's rank does not count
                const int have = left - 8 * half;
                v8bf v1[TN], v2[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int col = wn0 + 32 * j + fr;
                    v4i b = *(const v4i *)(st + APL + h * (BN * 32) + col * 32 +
                                           16 * (half ^ ((col >> 3) & 1)));
                    if (left < 16) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            b[q] = have >= 2 * q + 2 ? b[q] : (have == 2 * q + 1 ? b[q] & 0xffff : 0);
                    }
                    v1[j] = __builtin_bit_cast(v8bf, b);
                    if constexpr (ADAPT == IGEMM_F16)
                        split2(__builtin_bit_cast(v8hf, b), v1[j], v2[j]);
                }
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int row = wm0 + 32 * i + fr;
                    const bool it = arow_id[row] == which;
                    const uint64_t own = __ballot(it);
                    if (own == 0) continue;
                    const int ch = 4 * h + 2 * half;
                    const float4 lo =
                        *(const float4 *)(st + row * RA + 16 * (ch ^ ring::swz_a<RA>(row)));
                    const float4 hi =
                        *(const float4 *)(st + row * RA + 16 * ((ch + 1) ^ ring::swz_a<RA>(row)));
                    const float uv[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                    v8bf u1, u2, u3;
                    split3(uv, u1, u2, u3);
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        auto product = [&](v16f y) __attribute__((always_inline)) -> v16f {
                            if constexpr (ADAPT == IGEMM_F16) {
                                y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v2[j], u2, y, 0, 0, 0);
                                y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v2[j], u1, y, 0, 0, 0);
                            }
                            y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1[j], u3, y, 0, 0, 0);
                            y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1[j], u2, y, 0, 0, 0);
                            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1[j], u1, y, 0, 0, 0);
                        };
                        if (~own == 0) {
                            acc[i][j] =
                                __builtin_bit_cast(v16i, product(__builtin_bit_cast(v16f, acc[i][j])));
                        } else {
                            v16f y;
#pragma unroll
                            for (int r = 0; r < 16; ++r) y[r] = 0.0f;
                            y = product(y);
                            // Rows of other adapters keep what they have: nothing of
                            // this one, infinities and NaN included, reaches them.
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const int old = acc[i][j][r];
                                acc[i][j][r] = it ? as_int(as_float(old) + y[r]) : old;
                            }
                        }
                    }
                }
            }
        }
    };
    if constexpr (!REG) {
        // (the compiler's waits do not know of the DMAs: the rows are read, and waited
        // for, before this wave's first one)
        fetch_rows();
#pragma unroll
        for (int s = 0; s < NST - 1; ++s) issue_b(s, s);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        place_a();
#pragma unroll
        for (int s = 0; s < NST - 1; ++s) issue_a(s, s);
        terms();
        // (the k loop's first barrier publishes what terms() leaves in LDS)
        // The adapters' tiles follow tile nkm - 1: with fewer k-tiles than the ring
        // holds, the empty ones that were issued above are multiplied too.
        const int nkm = XT ? max(nkt, NST - 1) : nkt;
        int s = 0;
        // Tile kt has landed when at most the NST - 2 later ones are out; of the first
        // tiles, whose A was issued after all of their B, when at most NST - 2 tiles'
        // A is.
        auto arrived = [&](int kt) __attribute__((always_inline)) {
            if (kt < NST - 2)
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NST - 2) * DPA) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NST - 2) * DPW) : "memory");
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };
        auto turn = [&]() __attribute__((always_inline)) { s = s == NST - 1 ? 0 : s + 1; };
        if constexpr (!XT) {
            for (int kt = 0; kt < nkm; ++kt) {
                arrived(kt);
                issue(kt + NST - 1, s == 0 ? NST - 1 : s - 1);
                tile(s);
                turn();
            }
        } else {
            // (the last tiles apart: what only they need is not kept over the others)
            int kt = 0;
            for (; kt < nkm - (NST - 1); ++kt) {
                arrived(kt);
                issue(kt + NST - 1, s == 0 ? NST - 1 : s - 1);
                tile(s);
                turn();
            }
            Unit ahead = {0, 0, -2, 0};
            for (int x = 0; x < NST - 1; ++x) {
                arrived(kt + x);
                if (x == 0) ahead = unit_of(0);  // (listed before this barrier)
                issue_extra(ahead, s == 0 ? NST - 1 : s - 1);
                ahead = next(next(ahead));
                tile(s);
                turn();
            }
            scale();
            Unit now = unit_of(0);
            while (now.which >= 0) {
                arrived(nkm);
                issue_extra(ahead, s == 0 ? NST - 1 : s - 1);
                ahead = next(next(ahead));
                tile_extra(now, s);
                turn();
                now = next(next(now));
            }
        }
        // no DMA may land in LDS that is used anew below
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
        regs_a va;
        regs_b vb;
        if (nkt > 0) {
            load(va, vb, 0);
            store(va, vb, 0);
        }
        terms();
        for (int kt = 0; kt < nkt; ++kt) {
            __syncthreads();
            if (kt + 1 < nkt) load(va, vb, kt + 1);
            tile(kt & 1);
            if (kt + 1 < nkt) store(va, vb, 1 - (kt & 1));
        }
    }

    // ---- raw sums of a slice ----------------------------------------------------------
    if constexpr (PART) {
        int32_t *dst = part + ((int64_t)z * p.rows + f.lo + m0) * p.n + n0;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int lr = wm0 + 32 * i + fr;
            if (lr >= mrows) continue;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int c = wn0 + 32 * j + M::out_row(lane, r);
                    int32_t *at = dst + (int64_t)lr * p.n + c;
                    const v4i v = {acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2],
                                   acc[i][j][r + 3]};
                    if (n0 + c + 4 <= p.n) {
                        __builtin_memcpy(at, &v, 16);
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (n0 + c + q < p.n) at[q] = v[q];
                    }
                }
        }
        return;
    }

    // ---- scales, adapters, output -------------------------------------------------------
    __syncthreads();  // the ring becomes the waves' output blocks
    char *blk = smem + wave * 32 * PITCH;
    if (!busy) return;
    if constexpr (!XT) scale();
    if constexpr (ADAPT != 0 && !PART && !XT) {
        // The adapters from memory: fragments of u and `up` straight into registers, the
        // next 16 ranks' on their way while these are multiplied (all blocks' first
        // ones from the start; staged as k-tiles, which is the 256-row tiles' way, 2048 x
        // 4096 x 4096 with rank 64, 54 us, took 4 us more).
        struct Piece {
            float u[8];
            u32 w[TN][4];
        };
        const int e1 = 8 * (lane >> 5);
        int mine[TM], ranks[TM], urow[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            mine[i] = arow_id[wm0 + 32 * i + fr];
            urow[i] = max(arow[wm0 + 32 * i + fr], 0);
            ranks[i] = rank_of(ad, mine[i]);
        }
        auto fetch = [&](int i, int which, int rank, int e0, Piece &f) __attribute__((always_inline)) {
            const float4 *src = (const float4 *)(u + (int64_t)urow[i] * rpad + e0 + e1);
            const float4 lo = src[0], hi = src[1];
            const float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int q = 0; q < 8; ++q) f.u[q] = x[q];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int c = min(n0 + wn0 + 32 * j + fr, p.n - 1);
                const uint16_t *row =
                    (const uint16_t *)ad.up + which * ad.stride_up + c * ad.ld_up;
                if (ad.rank % 8 == 0 && e0 + 16 <= rank)
                    __builtin_memcpy(f.w[j], row + e0 + e1, 16);
                else
                    load8(row, e0 + e1, ad.rank, rank, f.w[j]);
            }
        };
        // The block's adapters, one after the other: every row is multiplied with
        // each, and takes its own one's result. (A row of a matrix product depends on
        // its own row of u alone, so other rows' values cannot reach it.)
        auto first_of = [&](int i, uint64_t todo, int *rank) __attribute__((always_inline)) -> int {
            const int l = __ffsll((unsigned long long)todo) - 1;
            *rank = __builtin_amdgcn_readlane(ranks[i], l);
            return __builtin_amdgcn_readlane(mine[i], l);
        };
        Piece head[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint64_t todo = __ballot(ranks[i] > 0);
            if (todo != 0) {
                int rank;
                const int which = first_of(i, todo, &rank);
                fetch(i, which, rank, 0, head[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            uint64_t todo = __ballot(ranks[i] > 0);
            if (todo == 0) continue;
            int rank, e0 = 0, which = first_of(i, todo, &rank);
            todo &= ~__ballot(mine[i] == which);
            v16f y[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) y[j][r] = 0.0f;
            Piece f = head[i];
            for (;;) {
                // the next piece: more ranks, or the next adapter's first
                Piece ahead;
                const bool more = e0 + 16 < rank, last = !more && todo == 0;
                int next_which = which, next_rank = rank, next_e0 = e0 + 16;
                if (!more && todo != 0) {
                    next_which = first_of(i, todo, &next_rank);
                    next_e0 = 0;
                }
                if (!last) fetch(i, next_which, next_rank, next_e0, ahead);
                v8bf u1, u2, u3;
                split3(f.u, u1, u2, u3);
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const v4u b4 = {f.w[j][0], f.w[j][1], f.w[j][2], f.w[j][3]};
                    v8bf v1 = __builtin_bit_cast(v8bf, b4), v2;
                    if constexpr (ADAPT == IGEMM_F16) {
                        split2(__builtin_bit_cast(v8hf, b4), v1, v2);
                        y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v2, u2, y[j], 0, 0, 0);
                        y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v2, u1, y[j], 0, 0, 0);
                    }
                    y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, u3, y[j], 0, 0, 0);
                    y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, u2, y[j], 0, 0, 0);
                    y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, u1, y[j], 0, 0, 0);
                }
                if (!more) {
                    // the adapter is done: its rows take the result
                    const bool it = mine[i] == which;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
#pragma unroll
                        for (int j = 0; j < TN; ++j) {
                            const int old = acc[i][j][r];
                            acc[i][j][r] = it ? as_int(as_float(old) + y[j][r]) : old;
                            y[j][r] = 0.0f;
                        }
                    }
                    if (last) break;
                    todo &= ~__ballot(mine[i] == next_which);
                }
                which = next_which;
                rank = next_rank;
                e0 = next_e0;
                f = ahead;
            }
        }
    }
    auto emit = [&](auto type_c) __attribute__((always_inline)) {
        constexpr int T = decltype(type_c)::value;
        constexpr int ES = T == IGEMM_F32 ? 4 : 2, V = 16 / ES, LPR = 32 * JB / V;  // lanes a row
        // (rows 34 or 68 words apart: a write of 32 rows covers all banks)
        constexpr int P = 32 * JB * ES + (ES == 2 ? 8 : 16);
#pragma unroll
        for (int ij = 0; ij < TM * (TN / JB); ++ij) {
            const int i = ij / (TN / JB), jb = ij % (TN / JB) * JB;
            const int r0 = wm0 + 32 * i, c0 = n0 + wn0 + 32 * jb;
#pragma unroll
            for (int j = 0; j < JB; ++j)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    float x[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int bits = acc[i][jb + j][r + q];
                        x[q] = as_float(bits);
                    }
                    char *at = blk + fr * P + (32 * j + M::out_row(lane, r)) * ES;
                    if constexpr (ES == 4) {
                        *(float4 *)at = make_float4(x[0], x[1], x[2], x[3]);
                    } else {
                        uint2 w;
                        w.x = (u32)to16<T>(x[0]) | (u32)to16<T>(x[1]) << 16;
                        w.y = (u32)to16<T>(x[2]) | (u32)to16<T>(x[3]) << 16;
                        *(uint2 *)at = w;
                    }
                }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            const int c = (lane % LPR) * V, col = c0 + c;
#pragma unroll
            for (int q = 0; q < 32; q += 64 / LPR) {
                const int lr = q + lane / LPR;
                const int o = orow[r0 + lr];
                if (o < 0) continue;
                const char *src = blk + lr * P + c * ES;
                char *dst = (char *)p.out + ((int64_t)o * p.ldo + col) * ES;
                if (col + V <= p.n) {
                    // (src lies at a multiple of 8)
                    const uint2 lo = *(const uint2 *)src, hi = *(const uint2 *)(src + 8);
                    const v4i v = {(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
                    __builtin_memcpy(dst, &v, 16);
                } else {
                    for (int e = 0; col + e < p.n; ++e)
                        if constexpr (ES == 4) ((float *)dst)[e] = ((const float *)src)[e];
                        else ((uint16_t *)dst)[e] = ((const uint16_t *)src)[e];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (p.type == IGEMM_F32) emit(ic<IGEMM_F32>{});
    else if (p.type == IGEMM_BF16) emit(ic<IGEMM_BF16>{});
    else emit(ic<IGEMM_F16>{});
}

}  // namespace rows
}  // namespace igemm
