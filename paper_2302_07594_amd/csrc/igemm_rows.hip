// The experts' products and the shared projection with adapters: the plain
// kernels, which take every size, stride and alignment.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_rows_device.h"

namespace igemm {
namespace rows {
namespace {

constexpr int kTile = 64, kStep = 32;

__global__ void __launch_bounds__(256)
product_plain(Product p, Adapters ad, const float *__restrict__ u) {
    __shared__ int8_t sa[kTile][kStep + 4];
    __shared__ int8_t sb[kStep][kTile + 4];
    __shared__ int ra[kTile], ro[kTile];
    const int tid = threadIdx.x, lane = tid & 63;
    const int tiles_n = (p.n + kTile - 1) / kTile;
    const int t = blockIdx.x / tiles_n, n0 = (blockIdx.x - t * tiles_n) * kTile;
    const int per = (p.groups + 63) / 64;
    int before;
    const int total = wave_tiles(p, kTile, per, lane, &before);
    if (t >= total) return;
    const Found f = wave_find(p, kTile, per, lane, before, t);
    const int at = (t - f.pre) * kTile;
    if (tid < kTile) {
        ra[tid] = ro[tid] = -1;
        if (at + tid < f.cnt) rows_of(p, f.lo + at + tid, &ra[tid], &ro[tid]);
    }
    __syncthreads();
    const int8_t *B = p.B + f.group * p.stride_b;
    const int r0 = (tid >> 4) * 4, c0 = (tid & 15) * 4;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < p.k; k0 += kStep) {
        for (int e = tid; e < kTile * kStep; e += 256) {
            const int r = e / kStep, c = e % kStep;
            sa[r][c] = ra[r] >= 0 && k0 + c < p.k ? p.A[(int64_t)ra[r] * p.lda + k0 + c] : 0;
        }
        for (int e = tid; e < kTile * kStep; e += 256) {
            const int r = e / kTile, c = e % kTile;
            sb[r][c] = k0 + r < p.k && n0 + c < p.n ? B[(int64_t)(k0 + r) * p.ldb + n0 + c] : 0;
        }
        __syncthreads();
        for (int c = 0; c < kStep; ++c)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] += (int)sa[r0 + i][c] * (int)sb[c][c0 + j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int a = ra[r0 + i], o = ro[r0 + i];
        if (o < 0) continue;
        const float s = p.scale_a != nullptr ? p.scale_a[a] : 1.0f;
        int which = ad.adapters > 0 ? ad.ids[a] : -1, rank = 0;
        if (which < 0 || which >= ad.adapters) which = -1;
        if (which >= 0)
            rank = ad.ranks != nullptr ? min(max(ad.ranks[which], 0), ad.rank) : ad.rank;
        for (int j = 0; j < 4; ++j) {
            const int c = n0 + c0 + j;
            if (c >= p.n) continue;
            float x = (float)acc[i][j] * s;
            if (p.scale_b != nullptr) x *= p.scale_b[(int64_t)f.group * p.n + c];
            const uint16_t *up = (const uint16_t *)ad.up + which * ad.stride_up + c * ad.ld_up;
            float y = 0.0f;
            for (int r = 0; r < rank; ++r)
                y += u[(int64_t)a * ad.rank + r] *
                     (ad.type == IGEMM_BF16 ? from16<IGEMM_BF16>(up[r]) : from16<IGEMM_F16>(up[r]));
            if (which >= 0) x += y;
            put(p.type, p.out, (int64_t)o * p.ldo + c, x);
        }
    }
}

// u[i, r], a wave each.
__global__ void __launch_bounds__(64) shrink_plain(Product p, Adapters ad, float *__restrict__ u) {
    const int i = blockIdx.x, r = blockIdx.y, lane = threadIdx.x;
    const int which = ad.ids[i];
    if (which < 0 || which >= ad.adapters) return;
    const int rank = ad.ranks != nullptr ? min(max(ad.ranks[which], 0), ad.rank) : ad.rank;
    if (r >= rank) return;
    const uint16_t *d = (const uint16_t *)ad.down + which * ad.stride_down + r * ad.ld_down;
    float x = 0.0f;
    for (int c = lane; c < p.k; c += 64)
        x += (float)p.A[(int64_t)i * p.lda + c] *
             (ad.type == IGEMM_BF16 ? from16<IGEMM_BF16>(d[c]) : from16<IGEMM_F16>(d[c]));
    for (int s = 32; s > 0; s /= 2) x += __shfl_xor(x, s);
    if (p.scale_a != nullptr) x *= p.scale_a[i];
    if (ad.scaling != nullptr) x *= ad.scaling[which];
    if (lane == 0) u[(int64_t)i * ad.rank + r] = x;
}

template <int T>
__global__ void __launch_bounds__(256)
combine_plain(int64_t tokens, int top_k, int n, const void *Z, int64_t ldz, const float *weights,
              const int32_t *ids, const void *base, int64_t ld_base, void *out, int64_t ldo) {
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < tokens * n;
         e += (int64_t)gridDim.x * 256) {
        const int64_t t = e / n;
        const int c = (int)(e - t * n);
        float x = base != nullptr ? get<T>(base, t * ld_base + c) : 0.0f;
        for (int j = 0; j < top_k; ++j) {
            const int64_t s = t * top_k + j;
            if (ids == nullptr || ids[s] >= 0) x += weights[s] * get<T>(Z, s * ldz + c);
        }
        put<T>(out, t * ldo + c, x);
    }
}

}  // namespace

int64_t product_workspace(int64_t rows, int64_t n, int64_t k, int64_t groups, int64_t adapters,
                          int64_t rank, int num_cu) {
    return adapters > 0 && rank > 0 ? (rows * rank * 4 + 255) / 256 * 256 : 0;
}

int launch_product(const Product &p, const Adapters &ad, int num_cu, void *workspace,
                   void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    float *u = (float *)workspace;
    if (ad.adapters > 0)
        shrink_plain<<<dim3((unsigned)p.rows, (unsigned)ad.rank), 64, 0, stream>>>(p, ad, u);
    // Upper bound of the row tiles: every group may end inside one.
    const int64_t t = (p.rows + kTile - 1) / kTile + (p.offsets != nullptr ? p.groups : 0);
    const int64_t grid = t * ((p.n + kTile - 1) / kTile);
    if (grid > 0x7fffffff) return IGEMM_ENOTSUP;
    product_plain<<<dim3((unsigned)grid), 256, 0, stream>>>(p, ad, u);
    return hipGetLastError() == hipSuccess ? IGEMM_OK : IGEMM_EHIP;
}

int launch_combine(int64_t tokens, int64_t top_k, int64_t n, int type, const void *Z, int64_t ldz,
                   const float *weights, const int32_t *ids, const void *base, int64_t ld_base,
                   void *out, int64_t ldo, void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const int64_t blocks = (tokens * n + 255) / 256;
    const dim3 grid((unsigned)(blocks < 8192 ? blocks : 8192));
    if (type == IGEMM_F32)
        combine_plain<IGEMM_F32><<<grid, 256, 0, stream>>>(tokens, (int)top_k, (int)n, Z, ldz, weights,
                                                           ids, base, ld_base, out, ldo);
    else if (type == IGEMM_BF16)
        combine_plain<IGEMM_BF16><<<grid, 256, 0, stream>>>(tokens, (int)top_k, (int)n, Z, ldz,
                                                            weights, ids, base, ld_base, out, ldo);
    else
        combine_plain<IGEMM_F16><<<grid, 256, 0, stream>>>(tokens, (int)top_k, (int)n, Z, ldz,
                                                           weights, ids, base, ld_base, out, ldo);
    return hipGetLastError() == hipSuccess ? IGEMM_OK : IGEMM_EHIP;
}

}  // namespace rows
}  // namespace igemm
