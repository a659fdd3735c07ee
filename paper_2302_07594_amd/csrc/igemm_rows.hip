// The experts' products, the shared projection with adapters, and the sum of a
// token's slots: the kernels beside the tile kernel (igemm_rows_tile.h), the
// choice of tile and slices, the launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_rows_tile.h"

namespace igemm {
namespace rows {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int byte_of(u32 w, int b) { return (int)(int8_t)(w >> (8 * b)); }

// 16 int8 of a row of `len` from e0, zero beyond it.
__device__ __forceinline__ v4i load_row16(const int8_t *row, int e0, int len) {
    if (e0 + 16 <= len) return ring::load_u16((const char *)row + e0);
    return load_elems<1>(row, e0, len);
}

// ---- u = scaling scale_a A down^T -------------------------------------------------

// Few rows or few ranks, where the product is not sliced (shrink_row).
__global__ void __launch_bounds__(256)
shrink_rows(Product p, Adapters ad, float *__restrict__ u, int rpad) {
    shrink_row<4>(p, ad, u, rpad, blockIdx.x, blockIdx.y);
}

// Many rows: 32 rows x 32 ranks a workgroup on the matrix cores, k over its eight
// waves, whose sums meet in LDS. int8 values are exact in both 16-bit types.
// The block's adapters are taken one after the other, as in the tile kernel.
template <int T>
__global__ void __launch_bounds__(512)
shrink_tiles(Product p, Adapters ad, float *__restrict__ u, int rpad) {
    __shared__ float red[8][32][33];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i0 = blockIdx.x * 32, r0 = blockIdx.y * 32;
    const int row = min(i0 + (lane & 31), p.rows - 1), half = lane >> 5;
    int mine = i0 + (lane & 31) < p.rows ? ad.ids[row] : -1;
    if (mine >= ad.adapters) mine = -1;
    const int8_t *a = p.A + (int64_t)row * p.lda;
    const int span = ((p.k + 7) / 8 + 31) / 32 * 32;  // k of a wave
    const int kb = wave * span, ke = min(kb + span, p.k);
    uint64_t todo = __ballot(mine >= 0);
    while (todo != 0) {
        const int which =
            __builtin_amdgcn_readlane(mine, __ffsll((unsigned long long)todo) - 1);
        todo &= ~__ballot(mine == which);
        const int rank = rank_of(ad, which);
        if (r0 >= rank) continue;
        const int r = min(r0 + (lane & 31), rank - 1);
        const uint16_t *d =
            (const uint16_t *)ad.down + which * ad.stride_down + r * ad.ld_down;
        v16f acc;
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[q] = 0.0f;
        // 32 k in two instructions: lane half h holds k 16 h .. 16 h + 15 of both
        // operands, eight at a time.
        auto step = [&](v4i av, const v4i (&dv)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if constexpr (T == IGEMM_BF16) {
                    v8bf x;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = (__bf16)(float)byte_of((u32)av[2 * q + e / 4], e & 3);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        x, __builtin_bit_cast(v8bf, dv[q]), acc, 0, 0, 0);
                } else {
                    v8h x;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = (_Float16)(float)byte_of((u32)av[2 * q + e / 4], e & 3);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                        x, __builtin_bit_cast(v8h, dv[q]), acc, 0, 0, 0);
                }
            }
        };
        // Four steps' loads before the first is used; the last k apart, bounded.
        int k0 = kb;
        constexpr int AHEAD = 4;
        for (; k0 + 32 * AHEAD <= ke; k0 += 32 * AHEAD) {
            v4i av[AHEAD], dv[AHEAD][2];
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) {
                const int e0 = k0 + 32 * x + 16 * half;
                av[x] = ring::load_u16((const char *)a + e0);
                dv[x][0] = ring::load_u16((const char *)(d + e0));
                dv[x][1] = ring::load_u16((const char *)(d + e0 + 8));
            }
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) step(av[x], dv[x]);
        }
        for (; k0 < ke; k0 += 32) {
            const int e0 = k0 + 16 * half;
            v4i dv[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                u32 w[4];
                load8(d, e0 + 8 * q, p.k, p.k, w);
                dv[q] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
            }
            step(load_row16(a, e0, p.k), dv);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 16; ++q)
            red[wave][Mfma<32>::out_row(lane, q)][lane & 31] = acc[q];
        __syncthreads();
        const float f = ad.scaling != nullptr ? ad.scaling[which] : 1.0f;
        for (int e = threadIdx.x; e < 1024; e += 512) {
            const int lr = e >> 5, c = e & 31, i = i0 + lr;
            if (i < p.rows && r0 + c < rank && ad.ids[i] == which) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) s += red[w][lr][c];
                u[(int64_t)i * rpad + r0 + c] = s * (p.scale_a != nullptr ? p.scale_a[i] : 1.0f) * f;
            }
        }
    }
}

// ---- the slices of few rows joined ---------------------------------------------------
//
// A workgroup a position and 256 columns: the raw sums of the k slices added up
// (exactly), scaled, with the adapter's part in plain float arithmetic.
__global__ void __launch_bounds__(256)
join_slices(Product p, Adapters ad, const float *__restrict__ u, int ks, int rpad,
            const int32_t *__restrict__ part, int slices) {
    __shared__ float us[1024];
    const int i = blockIdx.y, lane = threadIdx.x & 63;
    const int c = blockIdx.x * 256 + threadIdx.x;
    int sum = 0;
    if (c < p.n) {
#pragma unroll 8
        for (int z = 0; z < slices; ++z) sum += part[((int64_t)z * p.rows + i) * p.n + c];
    }
    int g = 0;
    if (p.offsets != nullptr) {
        int below = 0;
        for (int x = lane; x <= p.groups; x += 64) below += p.offsets[x] <= i;
#pragma unroll
        for (int o = 32; o > 0; o /= 2) below += __shfl_xor(below, o);
        g = below - 1;
        if (g < 0 || g >= p.groups) return;
    }
    int a, o;
    rows_of(p, i, &a, &o);
    if (o < 0) return;
    int rank = 0, which = -1;
    if (ad.adapters > 0) {
        which = ad.ids[a];
        rank = rank_of(ad, which);
        for (int r = threadIdx.x; r < rank; r += 256) {
            float s = 0.0f;
            for (int q = 0; q < ks; ++q) s += u[((int64_t)q * p.rows + a) * rpad + r];
            us[r] = s;
        }
        __syncthreads();
    }
    if (c >= p.n) return;
    float x = (float)sum * (p.scale_a != nullptr ? p.scale_a[a] : 1.0f);
    if (p.scale_b != nullptr) x *= p.scale_b[(int64_t)g * p.n + c];
    if (rank > 0) {
        const uint16_t *up = (const uint16_t *)ad.up + which * ad.stride_up + c * ad.ld_up;
        float y = 0.0f;
        for (int r = 0; r < rank; r += 8) {
            u32 w[4];
            load8(up, r, ad.rank, rank, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint16_t b = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
                const float v = ad.type == IGEMM_BF16 ? from16<IGEMM_BF16>(b) : from16<IGEMM_F16>(b);
                if (r + e < rank) y = fmaf(us[r + e], v, y);
            }
        }
        x += y;
    }
    put(p.type, p.out, (int64_t)o * p.ldo + c, x);
}

// ---- the sum of a token's slots ---------------------------------------------------

// One pass over Z. A thread takes 16 bytes of a row, eight slots' loads at a time
// before the first is used; a group of `lanes` threads (a power of two) covers a
// row, or 16 * lanes bytes of it. Slots left out read the token's first slot's
// row instead, which is at hand, so that no load waits for an id's branch.
template <int T, bool WAVE>
__global__ void __launch_bounds__(256)
combine_slots(int64_t tokens, int top_k, int n, const char *Z, int64_t ldz,
              const float *__restrict__ weights, const int32_t *__restrict__ ids,
              const char *base, int64_t ld_base, char *out, int64_t ldo, int lanes,
              int pieces) {
    constexpr int ES = T == IGEMM_F32 ? 4 : 2, V = 16 / ES;
    const int tid = threadIdx.x, per = (int)blockDim.x / lanes;
    const u32 at = blockIdx.x * per + tid / lanes, row = at / (u32)pieces;
    int64_t t = row;
    const int c = ((int)(at - row * (u32)pieces) * lanes + tid % lanes) * V;
    if constexpr (WAVE)  // the whole wave has one token: its weights are scalars
        t = (int64_t)__builtin_amdgcn_readfirstlane((int)t);
    if (t >= tokens || c >= n) return;
    const bool whole = c + V <= n;
    auto fetch = [&](const char *row) -> v4i {
        if (whole) return ring::load_u16(row + (int64_t)c * ES);
        return load_elems<ES == 4 ? 1 : 2>(row + (int64_t)c * ES, 0, ES == 4 ? (n - c) * 4 : n - c);
    };
    auto value = [&](v4i v, int e) -> float {
        const int word = v[ES == 4 ? e : e / 2];
        if constexpr (ES == 4) return __builtin_bit_cast(float, word);
        else return from16<T>((uint16_t)((u32)word >> (16 * (e & 1))));
    };
    float x[V] = {};
    if (base != nullptr) {
        const v4i b = fetch(base + t * ld_base * ES);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = value(b, e);
    }
    const int64_t s0 = t * top_k;
    for (int j0 = 0; j0 < top_k; j0 += 8) {
        v4i z[8];
        float w[8];
        bool on[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = j0 + j < top_k;
            const int64_t s = s0 + (in ? j0 + j : 0);
            on[j] = in && (ids == nullptr || ids[s] >= 0);
            w[j] = weights[s];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = fetch(Z + (on[j] ? s0 + j0 + j : s0) * ldz * ES);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = on[j] ? fmaf(w[j], value(z[j], e), x[e]) : x[e];
    }
    char *dst = out + (t * ldo + c) * ES;
    if (whole) {
        v4i r;
        if constexpr (ES == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = __builtin_bit_cast(int, x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                r[e] = (int)((u32)to16<T>(x[2 * e]) | (u32)to16<T>(x[2 * e + 1]) << 16);
        }
        __builtin_memcpy(dst, &r, 16);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < n) put<T>(dst, e, x[e]);
    }
}

// ---- choices --------------------------------------------------------------------------

struct Choice {
    int bm, bn;       // tile
    int slices, kchunk;
    bool by_row;      // u: a workgroup a row (ks k slices), else 32 x 32 blocks
    int ks, rpad;
    int64_t u_bytes, part_bytes;
};

int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// By sizes alone, so that the workspace can be sized before the operands exist.
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
        c.bm = 64, c.bn = 256;
    } else if (avg >= 192 &&
               full(tiles(256, 256), num_cu) >= 0.9 * full(tiles(128, 128), 2 * num_cu)) {
        c.bm = 256, c.bn = 256;
    } else {
        c.bm = 128, c.bn = 128;
    }
    // Fewer tiles than compute units: narrower ones, then k slices.
    int64_t slices = 1;
    if (c.bm <= 64 && tiles(c.bm, 256) < num_cu) {
        c.bn = 128;
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
    if (adapters > 0 && rank > 0) {
        c.rpad = (int)(ceil_div(rank, 16) * 16);
        c.by_row = c.slices > 1 || rows * rank <= 4096;
        c.ks = c.by_row ? (int)ceil_div(k, kShrinkK) : 1;
        c.u_bytes = up256(c.ks * rows * c.rpad * 4);
    }
    return c;
}

// Row tiles at most: every group with rows may end inside one.
int64_t most_tiles(int64_t rows, int64_t groups, int64_t bm) {
    const int64_t used = groups < rows ? groups : rows;
    return (rows + used * (bm - 1)) / bm;
}

template <int BM, int BN, int WM, int WN, int NST, int OCC, bool REG>
const void *pick_epi(bool part, bool adapt) {
    if (part) {
        if constexpr (BM <= 64 && BN == 128)
            return adapt ? (const void *)rows_tile<BM, BN, WM, WN, NST, OCC, REG, true, true>
                         : (const void *)rows_tile<BM, BN, WM, WN, NST, OCC, REG, true, false>;
        return nullptr;
    }
    return adapt ? (const void *)rows_tile<BM, BN, WM, WN, NST, OCC, REG, false, true>
                 : (const void *)rows_tile<BM, BN, WM, WN, NST, OCC, REG, false, false>;
}
// The tile's kernel and its threads. (us, random operands that are not cached:
// 64 rows of 64 experts, 1024 x 2048: 32 x 256 20.5, 32 x 128 23.5; 4096 rows,
// 2048 x 1024: 64 x 256 41.9, 64 x 128 42.4, 128 x 128 47.9; 32768 rows, 4096 x 2048:
// 256 x 256 358, 128 x 256 404, 128 x 128 442; one weight, 8192 x 11008 x 4096: 351,
// 377, 391; 2048 x 4096 x 4096, 128 tiles of 256 x 256: 53, else 38.)
const void *pick(int bm, int bn, bool reg, bool part, bool adapt, int *threads) {
    *threads = bm == 256 || (bm == 64 && bn == 256 && !reg) ? 512 : 256;
    if (reg)
        return bm == 32    ? (bn == 256 ? pick_epi<32, 256, 32, 64, 2, 2, true>(part, adapt)
                                        : pick_epi<32, 128, 32, 32, 2, 2, true>(part, adapt))
               : bm == 64  ? pick_epi<64, 128, 32, 64, 2, 2, true>(part, adapt)
                           : pick_epi<128, 128, 64, 64, 2, 2, true>(part, adapt);
    return bm == 32    ? (bn == 256 ? pick_epi<32, 256, 32, 64, 4, 1, false>(part, adapt)
                                    : pick_epi<32, 128, 32, 32, 3, 2, false>(part, adapt))
           : bm == 64  ? (bn == 256 ? pick_epi<64, 256, 32, 64, 3, 1, false>(part, adapt)
                                    : pick_epi<64, 128, 32, 64, 3, 2, false>(part, adapt))
           : bm == 128 ? pick_epi<128, 128, 64, 64, 2, 2, false>(part, adapt)
                       : pick_epi<256, 256, 128, 64, 2, 1, false>(part, adapt);
}

}  // namespace

int64_t product_workspace(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters,
                          int64_t rank, int num_cu) {
    const Choice c = choose(rows, n, k, groups, adapters, rank, num_cu);
    return c.part_bytes + c.u_bytes;
}

int launch_product(const Product &p, const Adapters &ad, int num_cu, void *workspace,
                   void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const Choice c = choose(p.rows, p.n, p.k, p.groups, ad.adapters, ad.rank, num_cu);
    int32_t *part = (int32_t *)workspace;
    float *u = (float *)((char *)workspace + c.part_bytes);
    const bool sliced = c.slices > 1, adapt = ad.adapters > 0;
    // By DMA where rows start at 4-byte addresses and the offsets of a whole last
    // k-tile stay below 4 GiB; else through registers, in tiles that have the
    // registers for it.
    const bool reg = (uintptr_t)p.A % 4 != 0 || (uintptr_t)p.B % 4 != 0 || p.lda % 4 != 0 ||
                     p.ldb % 4 != 0 || p.stride_b % 4 != 0 ||
                     ((int64_t)p.k + kStepK) * p.ldb > 0xffffffffll;
    int bm = c.bm, bn = c.bn, threads = 0;
    if (reg && bm >= 64) bn = 128;
    if (reg && bm == 256) bm = 128;
    const void *fn = pick(bm, bn, reg, sliced, adapt, &threads);
    const int64_t first = sliced && adapt ? (int64_t)p.rows * c.ks : 0;
    const int64_t grid = first + most_tiles(p.rows, p.groups, bm) * ceil_div(p.n, bn) * c.slices;
    if (fn == nullptr || grid > 0x7fffffff) return IGEMM_ENOTSUP;
    if (adapt && !sliced) {
        if (c.by_row) {
            const dim3 g((unsigned)p.rows, (unsigned)c.ks);
            shrink_rows<<<g, 256, 0, stream>>>(p, ad, u, c.rpad);
        } else {
            const dim3 g((unsigned)((p.rows + 31) / 32), (unsigned)((ad.rank + 31) / 32));
            if (ad.type == IGEMM_BF16)
                shrink_tiles<IGEMM_BF16><<<g, 512, 0, stream>>>(p, ad, u, c.rpad);
            else
                shrink_tiles<IGEMM_F16><<<g, 512, 0, stream>>>(p, ad, u, c.rpad);
        }
        if (hipGetLastError() != hipSuccess) return IGEMM_EHIP;
    }
    Product pp = p;
    Adapters aa = ad;
    int ks = c.ks, rpad = c.rpad, slices = c.slices, kchunk = c.kchunk;
    void *args[] = {&pp, &aa, &u, &ks, &rpad, &part, &slices, &kchunk};
    if (hipLaunchKernel(fn, dim3((unsigned)grid), dim3((unsigned)threads), args, 0, stream) !=
        hipSuccess)
        return IGEMM_EHIP;
    if (sliced)
        join_slices<<<dim3((unsigned)((p.n + 255) / 256), (unsigned)p.rows), 256, 0, stream>>>(
            p, ad, u, c.ks, c.rpad, part, c.slices);
    return hipGetLastError() == hipSuccess ? IGEMM_OK : IGEMM_EHIP;
}

int launch_combine(int64_t tokens, int64_t top_k, int64_t n, int type, const void *Z, int64_t ldz,
                   const float *weights, const int32_t *ids, const void *base, int64_t ld_base,
                   void *out, int64_t ldo, void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const int vec = type == IGEMM_F32 ? 4 : 8;
    // Few values: workgroups of one wave, so that more compute units share them.
    const int threads = tokens * n >= (int64_t)num_cu_of_current_device() * 4 * 256 * vec ? 256 : 64;
    int lanes = 1;
    while (lanes < threads && (int64_t)lanes * vec < n) lanes *= 2;
    int pieces = (int)((n + (int64_t)lanes * vec - 1) / ((int64_t)lanes * vec));
    const int64_t per = threads / lanes, blocks = (tokens * pieces + per - 1) / per;
    if (tokens * pieces > 0x7fffffff) return IGEMM_ENOTSUP;
    const bool wave = lanes >= 64;
#define IGEMM_COMBINE(t)                                           \
    (wave ? (const void *)combine_slots<t, true> : (const void *)combine_slots<t, false>)
    const void *fn = type == IGEMM_F32    ? IGEMM_COMBINE(IGEMM_F32)
                     : type == IGEMM_BF16 ? IGEMM_COMBINE(IGEMM_BF16)
                                          : IGEMM_COMBINE(IGEMM_F16);
#undef IGEMM_COMBINE
    int ki = (int)top_k, ni = (int)n;
    void *args[] = {&tokens, &ki,  &ni, (void *)&Z, &ldz,   (void *)&weights, (void *)&ids,
                    (void *)&base, &ld_base, &out,  &ldo, &lanes, &pieces};
    return hipLaunchKernel(fn, dim3((unsigned)blocks), dim3((unsigned)threads), args, 0, stream) ==
                   hipSuccess
               ? IGEMM_OK
               : IGEMM_EHIP;
}

}  // namespace rows
}  // namespace igemm
