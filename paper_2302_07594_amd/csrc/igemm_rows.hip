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
//
// Few rows, or few ranks: a workgroup a row and k slice, every wave one rank in
// four at a time, 16 bytes of `down` a lane. What it reads of `down` is one
// adapter a row, whichever the row's is, so a batch of 16 requests with an
// adapter each takes as long as one with a shared adapter.
constexpr int kShrinkK = 1024;  // k a workgroup: two passes of 64 lanes x 8

template <int T>
__global__ void __launch_bounds__(256)
shrink_rows(Product p, Adapters ad, float *__restrict__ u, int rpad) {
    const int i = blockIdx.x, z = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int which = ad.ids[i];
    const int rank = rank_of(ad, which);
    if (rank == 0) return;
    const int8_t *a = p.A + (int64_t)i * p.lda;
    constexpr int PASS = kShrinkK / 512;
    float x[PASS][8];
#pragma unroll
    for (int q = 0; q < PASS; ++q) {
        const int e0 = z * kShrinkK + 512 * q + 8 * lane;
        u32 w[2] = {0u, 0u};
        if (e0 + 8 <= p.k) {
            __builtin_memcpy(w, a + e0, 8);
        } else {
            for (int e = 0; e < 8 && e0 + e < p.k; ++e)
                w[e >> 2] |= (u32)(uint8_t)a[e0 + e] << (8 * (e & 3));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[q][e] = (float)byte_of(w[e >> 2], e & 3);
    }
    float f = p.scale_a != nullptr ? p.scale_a[i] : 1.0f;
    if (ad.scaling != nullptr) f *= ad.scaling[which];
    const uint16_t *down = (const uint16_t *)ad.down + which * ad.stride_down;
    for (int r = wave; r < rank; r += 4) {
        const uint16_t *d = down + r * ad.ld_down;
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < PASS; ++q) {
            const int e0 = z * kShrinkK + 512 * q + 8 * lane;
            if (e0 >= p.k) continue;
            u32 w[4];
            load8(d, e0, p.k, p.k, w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s = fmaf(x[q][e], from16<T>((uint16_t)(w[e / 2] >> (16 * (e & 1)))), s);
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) s += __shfl_xor(s, o);
        if (lane == 0) u[((int64_t)z * p.rows + i) * rpad + r] = s * f;
    }
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
        for (int k0 = kb; k0 < ke; k0 += 32) {
            // 32 k in two instructions: lane half h holds k 16 h .. 16 h + 15 of
            // both operands, eight at a time.
            const int e0 = k0 + 16 * half;
            const v4i av = load_row16(a, e0, p.k);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                u32 w[4];
                load8(d, e0 + 8 * q, p.k, p.k, w);
                const v4u w4 = {w[0], w[1], w[2], w[3]};
                if constexpr (T == IGEMM_BF16) {
                    v8bf x;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = (__bf16)(float)byte_of((u32)av[2 * q + e / 4], e & 3);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        x, __builtin_bit_cast(v8bf, w4), acc, 0, 0, 0);
                } else {
                    v8h x;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = (_Float16)(float)byte_of((u32)av[2 * q + e / 4], e & 3);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                        x, __builtin_bit_cast(v8h, w4), acc, 0, 0, 0);
                }
            }
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
    int sum = 0;
    for (int z = 0; z < slices; ++z) sum += part[((int64_t)z * p.rows + i) * p.n + c];
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
    int bm;           // rows of a tile; 128 columns
    int slices, kchunk;
    bool by_row;      // u: a workgroup a row (ks k slices), else 32 x 32 blocks
    int ks, rpad;
    int64_t u_bytes, part_bytes;
};

int64_t up256(int64_t b) { return (b + 255) / 256 * 256; }

// By sizes alone, so that the workspace can be sized before the operands exist.
Choice choose(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters, int64_t rank,
              int num_cu) {
    Choice c = {};
    const int64_t used = groups < rows ? groups : rows;   // groups that may have rows
    const int64_t avg = (rows + used - 1) / used;
    c.bm = avg <= 32 ? 32 : avg <= 64 ? 64 : 128;
    const int64_t tiles = (avg + c.bm - 1) / c.bm * used * ((n + 127) / 128);
    int64_t slices = 1;
    if (2 * tiles <= num_cu) {
        slices = num_cu / tiles;
        if (slices > k / 256) slices = k / 256;
        if (slices > 16) slices = 16;
        if (slices < 1) slices = 1;
    }
    int64_t chunk = ((k + slices - 1) / slices + kStepK - 1) / kStepK * kStepK;
    if (chunk < kStepK) chunk = kStepK;
    c.kchunk = (int)chunk;
    c.slices = k > 0 ? (int)((k + chunk - 1) / chunk) : 1;
    if (c.slices > 1) c.part_bytes = up256(c.slices * rows * n * 4);
    if (adapters > 0 && rank > 0) {
        c.rpad = (int)((rank + 15) / 16 * 16);
        c.by_row = rows * rank <= 4096;
        c.ks = c.by_row ? (int)((k + kShrinkK - 1) / kShrinkK) : 1;
        c.u_bytes = up256(c.ks * rows * c.rpad * 4);
    }
    return c;
}

// Row tiles at most: every group with rows may end inside one.
int64_t most_tiles(int64_t rows, int64_t groups, int64_t bm) {
    const int64_t used = groups < rows ? groups : rows;
    return (rows + used * (bm - 1)) / bm;
}

template <int BM, int WM, int WN, int NST, int OCC>
const void *pick(bool reg, bool part, bool adapt) {
    if (reg)
        return part    ? (const void *)rows_tile<BM, 128, WM, WN, 2, OCC, true, true, false>
               : adapt ? (const void *)rows_tile<BM, 128, WM, WN, 2, OCC, true, false, true>
                       : (const void *)rows_tile<BM, 128, WM, WN, 2, OCC, true, false, false>;
    return part    ? (const void *)rows_tile<BM, 128, WM, WN, NST, OCC, false, true, false>
           : adapt ? (const void *)rows_tile<BM, 128, WM, WN, NST, OCC, false, false, true>
                   : (const void *)rows_tile<BM, 128, WM, WN, NST, OCC, false, false, false>;
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
    const int tiles_n = (p.n + 127) / 128;
    const int64_t grid = most_tiles(p.rows, p.groups, c.bm) * tiles_n * c.slices;
    if (grid > 0x7fffffff) return IGEMM_ENOTSUP;
    if (ad.adapters > 0) {
        if (c.by_row) {
            const dim3 g((unsigned)p.rows, (unsigned)c.ks);
            if (ad.type == IGEMM_BF16)
                shrink_rows<IGEMM_BF16><<<g, 256, 0, stream>>>(p, ad, u, c.rpad);
            else
                shrink_rows<IGEMM_F16><<<g, 256, 0, stream>>>(p, ad, u, c.rpad);
        } else {
            const dim3 g((unsigned)((p.rows + 31) / 32), (unsigned)((ad.rank + 31) / 32));
            if (ad.type == IGEMM_BF16)
                shrink_tiles<IGEMM_BF16><<<g, 512, 0, stream>>>(p, ad, u, c.rpad);
            else
                shrink_tiles<IGEMM_F16><<<g, 512, 0, stream>>>(p, ad, u, c.rpad);
        }
        if (hipGetLastError() != hipSuccess) return IGEMM_EHIP;
    }
    // By DMA where rows start at 4-byte addresses and the offsets of a whole last
    // k-tile stay below 4 GiB.
    const bool reg = (uintptr_t)p.A % 4 != 0 || (uintptr_t)p.B % 4 != 0 || p.lda % 4 != 0 ||
                     p.ldb % 4 != 0 || p.stride_b % 4 != 0 ||
                     ((int64_t)p.k + kStepK) * p.ldb > 0xffffffffll;
    const bool sliced = c.slices > 1, adapt = ad.adapters > 0 && !sliced;
    const void *fn = c.bm == 32   ? pick<32, 32, 32, 3, 2>(reg, sliced, adapt)
                     : c.bm == 64 ? pick<64, 32, 64, 3, 2>(reg, sliced, adapt)
                                  : pick<128, 64, 64, 2, 2>(reg, sliced, adapt);
    Product pp = p;
    Adapters aa = ad;
    const float *uc = u;
    int ks = c.ks, rpad = c.rpad, slices = c.slices, kchunk = c.kchunk;
    void *args[] = {&pp, &aa, &uc, &ks, &rpad, &part, &slices, &kchunk};
    if (hipLaunchKernel(fn, dim3((unsigned)grid), dim3(256), args, 0, stream) != hipSuccess)
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
