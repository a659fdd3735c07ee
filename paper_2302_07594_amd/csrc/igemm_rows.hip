// The experts' products, the shared projection with adapters, and the sum of a
// token's slots: the kernels beside the tile kernel (igemm_rows_tile.h), the
// choice of tile and slices, the launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_rows_tile.h"

namespace igemm {
namespace rows {
namespace {

typedef v8hf v8h;
typedef short v8s __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int byte_of(u32 w, int b) { return (int)(int8_t)(w >> (8 * b)); }

// ---- u = scaling scale_a A down^T -------------------------------------------------

// Few rows or few ranks, where the product is not sliced (shrink_row).
template <int T>
__global__ void __launch_bounds__(256)
shrink_rows(Product p, Adapters ad, float *__restrict__ u, int rpad) {
    shrink_row<4, T>(p, ad, u, rpad, p.k, blockIdx.x, 0, blockIdx.y);
}

// Many rows: 32 rows x 16 NR ranks a workgroup, on the matrix cores (int8 values are
// exact in both 16-bit types): two waves of 16 rows for each of four k groups of
// 128 k at a time, whose sums meet in LDS at the end. Both operands pass through LDS,
// read along their rows: fragments read straight from memory take 32 rows a load,
// which at a row stride of a power of two all lie in one channel of the cache
// (8192 x 4096, rank 16, 24 adapters: 31 us, against 20 here). Bound by
// the latency of the k-tiles: two are under way, and with 16 ranks two workgroups share
// a compute unit (at least 8 us of reading A there). The block's adapters are shared
// out to gridDim.z workgroups, each of which takes its own one after the other:
// where one request ends and the next begins, a block has two.
constexpr int kShrinkTile = 512, kShrinkTurns = 3;
template <int T, int NR>
__global__ void __launch_bounds__(512, NR == 1 ? 4 : 2)
shrink_tiles(Product p, Adapters ad, float *__restrict__ u, int rpad) {
    constexpr int DR = 16 * NR;  // ranks
    __shared__ __attribute__((aligned(16))) char sa[2][4][kShrinkRows * 128];
    __shared__ __attribute__((aligned(16))) char sd[2][4][DR * 256];
    __shared__ __attribute__((aligned(16))) v4f red[3][2][NR][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i0 = blockIdx.x * kShrinkRows, r0 = blockIdx.y * DR;
    const int at = i0 + (lane & 31);
    int mine = at < p.rows ? ad.ids[at] : -1;
    if (mine >= ad.adapters) mine = -1;
    uint64_t todo = __ballot(mine >= 0);
    const int q = lane >> 4, c = lane & 15;
    const int kg = wave >> 1, rw = wave & 1;  // k group, row block
    int turn = 0;
    while (todo != 0) {
        const int which =
            __builtin_amdgcn_readlane(mine, __ffsll((unsigned long long)todo) - 1);
        todo &= ~__ballot(mine == which);
        if (turn++ % (int)gridDim.z != (int)blockIdx.z) continue;
        const int rank = rank_of(ad, which);
        const uint16_t *down = (const uint16_t *)ad.down + which * ad.stride_down;
        // Sixteen lanes a row of A, thirty-two a row of `down`. Rows past the end and
        // ranks past the adapter's read the last one: nothing comes of them. Whole
        // k-tiles are loaded without a branch (behind one, the wait for a tile is a wait
        // for every load under way), what is left of k at the end.
        v4i av[2][2], dv[2][2 * NR];  // two k-tiles on their way
        const int8_t *arow = p.A + (int64_t)min(i0 + (tid >> 4), p.rows - 1) * p.lda;
        const uint16_t *drow[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n)
            drow[n] = down + max(min(r0 + 16 * n + (tid >> 5), rank - 1), 0) * ad.ld_down;
        auto load = [&](auto set, int kt) __attribute__((always_inline)) {
            constexpr int S = decltype(set)::value;
#pragma unroll
            for (int x = 0; x < 2; ++x)
                av[S][x] = ring::load_u16((const char *)arow + kt * kShrinkTile + 256 * x +
                                          16 * (tid & 15));
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    dv[S][2 * n + x] = ring::load_u16(
                        (const char *)(drow[n] + kt * kShrinkTile + 256 * x + 8 * (tid & 31)));
        };
        auto load_rest = [&](int kt) __attribute__((always_inline)) {
            // (addresses of the loop over the adapters' every round are not worth
            // registers all along)
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));
#pragma unroll
            for (int x = 0; x < 2; ++x)
                av[0][x] = ring::load_edge((const char *)arow,
                                           kt * kShrinkTile + 256 * x + 16 * (tid & 15), p.k,
                                           p.k < 16);
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    u32 w[4];
                    load8(drow[n], kt * kShrinkTile + 256 * x + 8 * (tid & 31), p.k, p.k, w);
                    dv[0][2 * n + x] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
                }
        };
        auto store = [&](auto set) __attribute__((always_inline)) {
            constexpr int s = decltype(set)::value;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int row = tid >> 4, ch = 16 * x + (tid & 15);
                *(v4i *)(sa[s][ch >> 3] + row * 128 + 16 * ((ch & 7) ^ (row & 7))) = av[s][x];
            }
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 16 * n + (tid >> 5), ch = 32 * x + (tid & 31);
                    *(v4i *)(sd[s][ch >> 4] + row * 256 + 16 * ((ch & 15) ^ (row & 15))) =
                        dv[s][2 * n + x];
                }
        };
        v4f acc[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] = 0.0f;
        auto multiply = [&](auto set) __attribute__((always_inline)) {
            constexpr int s = decltype(set)::value;
            // 32 k an instruction: lane group q holds k 8 q .. 8 q + 7 of both.
            const int row = 16 * rw + c;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const int chunk = 2 * ks + (q >> 1);
                const u32 *src = (const u32 *)(sa[s][kg] + row * 128 +
                                               16 * (chunk ^ (row & 7)) + 8 * (q & 1));
                const u32 w[2] = {src[0], src[1]};
                v8s x;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = (short)to16<T>((float)byte_of(w[e >> 2], e & 3));
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const v4i d = *(const v4i *)(sd[s][kg] + (16 * n + c) * 256 +
                                                 16 * ((4 * ks + q) ^ c));
                    if constexpr (T == IGEMM_BF16)
                        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, d), acc[n], 0, 0,
                            0);
                    else
                        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                            __builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, d), acc[n], 0, 0,
                            0);
                }
            }
        };
        if (rank > r0) {
            const int whole = p.k / kShrinkTile;
            // k-tile kt from stage s; ahead: the loads of the next but one are issued,
            // after: the next one goes to the other stage.
            auto step = [&](auto set, int kt, auto ahead, auto after)
                __attribute__((always_inline)) {
                constexpr int s = decltype(set)::value;
                __syncthreads();
                if constexpr (decltype(ahead)::value) load(ic<s>{}, kt + 2);
                multiply(set);
                if constexpr (decltype(after)::value) store(ic<1 - s>{});
            };
            if (whole > 0) {
                load(ic<0>{}, 0);
                load(ic<1>{}, min(1, whole - 1));
                store(ic<0>{});
                int kt = 0;
                for (; kt + 3 < whole; kt += 2) {
                    step(ic<0>{}, kt, ic<1>{}, ic<1>{});
                    step(ic<1>{}, kt + 1, ic<1>{}, ic<1>{});
                }
                if (whole - kt == 3) {
                    step(ic<0>{}, kt, ic<1>{}, ic<1>{});
                    step(ic<1>{}, kt, ic<0>{}, ic<1>{});
                    step(ic<0>{}, kt, ic<0>{}, ic<0>{});
                } else if (whole - kt == 2) {
                    step(ic<0>{}, kt, ic<0>{}, ic<1>{});
                    step(ic<1>{}, kt, ic<0>{}, ic<0>{});
                } else {
                    step(ic<0>{}, kt, ic<0>{}, ic<0>{});
                }
            }
            if (whole * kShrinkTile < p.k) {
                load_rest(whole);
                __syncthreads();
                store(ic<0>{});
                __syncthreads();
                multiply(ic<0>{});
            }
        }
        __syncthreads();
        if (kg > 0)
#pragma unroll
            for (int n = 0; n < NR; ++n) red[kg - 1][rw][n][lane] = acc[n];
        __syncthreads();
        if (kg > 0) continue;
        const float f = ad.scaling != nullptr ? ad.scaling[which] : 1.0f;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int g = 0; g < 3; ++g) acc[n] += red[g][rw][n][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int lr = 16 * rw + 4 * q + e, i = i0 + lr;
            if (__shfl(mine, lr) != which) continue;
            const float sc = p.scale_a != nullptr ? p.scale_a[i] : 1.0f;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const int r = r0 + 16 * n + c;
                if (r < rpad)
                    u[(int64_t)i * rpad + r] = r < rank ? acc[n][e] * sc * f : 0.0f;
            }
        }
    }
}

// ---- the slices of few rows joined ---------------------------------------------------
//
// A workgroup a position and 256 columns: the raw sums of the k slices added up
// (exactly), scaled, with the adapter's part in plain float arithmetic (`up` is read
// once a row; 16 x 4096, rank 16: 4.7 us, a launch and two rounds of loads).
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
        const bool whole = ad.rank % 8 == 0 && rank % 8 == 0;
#pragma unroll 2
        for (int r = 0; r < rank; r += 8) {
            u32 w[4];
            if (whole) __builtin_memcpy(w, up + r, 16);
            else load8(up, r, ad.rank, rank, w);
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

// One pass over Z, bound by memory (4096 tokens of 8 slots of 4096, bf16: 61 us, 5.5 TB/s;
// 16 tokens: 4 us, a launch and one round of loads). A thread takes 16 bytes of a row, eight slots' loads at a time
// before the first is used; a group of `lanes` threads (a power of two) covers a
// row, or 16 * lanes bytes of it. Slots left out read the token's first slot's
// row instead, which is at hand, so that no load waits for an id's branch.
// Whether the v elements from c on lie in a row of n, 0 <= c < n. (c + v may pass an int:
// the last 16 bytes of a row of 2^31 - 1 elements begin at 2^31 - 8.)
constexpr __host__ __device__ bool whole_from(int c, int v, int n) { return c <= n - v; }
static_assert(!whole_from(0x7ffffff8, 8, 0x7fffffff) && whole_from(0x7ffffff0, 8, 0x7fffffff) &&
                  !whole_from(0x7ffffffc, 4, 0x7fffffff) && !whole_from(0, 8, 7) &&
                  whole_from(0, 8, 8) && !whole_from(0, 8, 1),
              "the ends of rows");

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
    const bool whole = whole_from(c, V, n);
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
    int64_t s8 = s0;  // the next eight slots; (counted down: j0 + 8 may pass an int)
    for (int left = top_k; left > 0; left -= 8, s8 += 8) {
        v4i z[8];
        float w[8];
        bool on[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = j < left;
            const int64_t s = in ? s8 + j : s0;
            on[j] = in && (ids == nullptr || ids[s] >= 0);
            w[j] = weights[s];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = fetch(Z + (on[j] ? s8 + j : s0) * ldz * ES);
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

// A grid has fewer than 2^32 threads.
bool launchable(int64_t blocks, int threads) { return blocks <= 0xffffffffll / threads; }

template <int BM, int BN, int WM, int WN, int NST, int OCC, bool REG, int ADAPT>
const void *pick_part(bool part) {
    if (!part) return (const void *)rows_tile<BM, BN, WM, WN, NST, OCC, REG, false, ADAPT>;
    if constexpr (BM <= 64 && BN == 128)
        return (const void *)rows_tile<BM, BN, WM, WN, NST, OCC, REG, true, ADAPT>;
    return nullptr;
}
// adapt: the adapters' weight type, 0 for none.
template <int BM, int BN, int WM, int WN, int NST, int OCC, bool REG>
const void *pick_epi(bool part, int adapt) {
    return adapt == 0            ? pick_part<BM, BN, WM, WN, NST, OCC, REG, 0>(part)
           : adapt == IGEMM_BF16 ? pick_part<BM, BN, WM, WN, NST, OCC, REG, IGEMM_BF16>(part)
                                 : pick_part<BM, BN, WM, WN, NST, OCC, REG, IGEMM_F16>(part);
}
// The tile's kernel and its threads. (us, random operands that are not cached:
// 64 rows of 64 experts, 1024 x 2048: 32 x 256 20.4, 64 x 128 20.9; 4096 rows,
// 2048 x 1024: 64 x 128 40.7, 128 x 128 46.9; 32768 rows, 4096 x 2048: 256 x 256 360,
// 128 x 128 410; one weight, 8192 x 11008 x 4096: 365, 370, with adapters of rank 16 394,
// 406, of rank 64 552, 514 (two waves a SIMD have no other work while the adapters' tiles
// arrive); 2048 x 4096 x 4096, 128 tiles of 256 x 256: 54, else 39.)
const void *pick(int bm, int bn, bool reg, bool part, int adapt, int *threads) {
    *threads = bm == 256 ? 512 : 256;
    if (reg)
        return bm == 32    ? (bn == 256 ? pick_epi<32, 256, 32, 64, 2, 2, true>(part, adapt)
                                        : pick_epi<32, 128, 32, 32, 2, 2, true>(part, adapt))
               : bm == 64  ? pick_epi<64, 128, 32, 64, 2, 2, true>(part, adapt)
                           : pick_epi<128, 128, 64, 64, 2, 2, true>(part, adapt);
    return bm == 32    ? (bn == 256 ? pick_epi<32, 256, 32, 64, 4, 1, false>(part, adapt)
                                    : pick_epi<32, 128, 32, 32, 3, 2, false>(part, adapt))
           : bm == 64  ? pick_epi<64, 128, 32, 64, 2, 3, false>(part, adapt)
           : bm == 128 ? pick_epi<128, 128, 64, 64, 2, 2, false>(part, adapt)
                       : pick_epi<256, 256, 64, 128, 2, 1, false>(part, adapt);
}

}  // namespace

int launch_product(const Product &p, const Adapters &ad, int num_cu, void *workspace,
                   void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const Choice c = choose(p.rows, p.n, p.k, p.groups, ad.adapters, ad.rank, num_cu);
    int32_t *part = (int32_t *)workspace;
    float *u = (float *)((char *)workspace + c.part_bytes);
    const bool sliced = c.slices > 1, adapt = ad.adapters > 0;
    const Tile t = tile_of(c, p, ad, num_cu);
    int threads = 0;
    const void *fn = pick(t.bm, t.bn, t.reg, sliced, adapt ? ad.type : 0, &threads);
    const int64_t first = sliced && adapt ? (int64_t)p.rows * c.ks * (c.rpad / 16) : 0;
    const int64_t grid = first + most_tiles(p.rows, p.groups, t.bm) * ceil_div(p.n, t.bn) * c.slices;
    if (fn == nullptr || !launchable(grid, threads) ||
        (adapt && !launchable(ceil_div(p.rows, kShrinkRows), 512)))
        return IGEMM_ENOTSUP;
    if (adapt && !sliced) {
        if (c.by_row) {
            const dim3 g((unsigned)p.rows, (unsigned)(c.rpad / 16));
            if (ad.type == IGEMM_BF16)
                shrink_rows<IGEMM_BF16><<<g, 256, 0, stream>>>(p, ad, u, c.rpad);
            else
                shrink_rows<IGEMM_F16><<<g, 256, 0, stream>>>(p, ad, u, c.rpad);
        } else {
            const bool two = c.shrink_ranks == 32;
            const dim3 g((unsigned)ceil_div(p.rows, kShrinkRows),
                         (unsigned)ceil_div(ad.rank, c.shrink_ranks), kShrinkTurns);
            const bool bf = ad.type == IGEMM_BF16;
            const void *sh = two ? bf ? (const void *)shrink_tiles<IGEMM_BF16, 2>
                                      : (const void *)shrink_tiles<IGEMM_F16, 2>
                             : bf ? (const void *)shrink_tiles<IGEMM_BF16, 1>
                                  : (const void *)shrink_tiles<IGEMM_F16, 1>;
            Product sp = p;
            Adapters sad = ad;
            int rpad = c.rpad;
            void *args[] = {&sp, &sad, &u, &rpad};
            if (hipLaunchKernel(sh, g, dim3(512), args, 0, stream) != hipSuccess)
                return IGEMM_EHIP;
        }
        if (hipGetLastError() != hipSuccess) return IGEMM_EHIP;
    }
    Product pp = p;
    Adapters aa = ad;
    int ks = c.ks, kshrink = kShrinkK, rpad = c.rpad, slices = c.slices, kchunk = c.kchunk;
    void *args[] = {&pp, &aa, &u, &ks, &kshrink, &rpad, &part, &slices, &kchunk};
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
    if (tokens * pieces > 0x7fffffff || !launchable(blocks, threads)) return IGEMM_ENOTSUP;
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
