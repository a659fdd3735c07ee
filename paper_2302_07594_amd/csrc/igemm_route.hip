// Routing of tokens to experts, and the plan of the experts' products.
//
// One wave a token. Scores and keys are formed in 64-bit floating point: with
// 32 bits about one token in a few thousand has an expert within rounding of
// the border of the chosen ones, and which side it falls on would depend on
// the order of the softmax's sum.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_rows_device.h"

namespace igemm {
namespace rows {
namespace {

constexpr double kNone = -__builtin_huge_val();

// The largest key of the wave and its index (the lower one of equals); index -1
// if every key is kNone.
__device__ __forceinline__ void wave_best(double &key, int &idx) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double k = __shfl_xor(key, d);
        const int i = __shfl_xor(idx, d);
        const bool take = k > key || (k == key && (unsigned)i < (unsigned)idx);
        key = take ? k : key;
        idx = take ? i : idx;
    }
}

// Expert e = 64 v + lane in register v.
template <int V, int T>
__global__ void __launch_bounds__(64)
route_tokens(igemm_route_desc d, const void *__restrict__ logits, int64_t ld,
             const float *__restrict__ bias, int32_t *__restrict__ ids,
             float *__restrict__ weights) {
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x;
    __shared__ double key_s[64 * V];
    float l[V];
    double s[V], key[V];
    float top = -__builtin_huge_valf();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = 64 * v + lane;
        l[v] = e < d.experts ? get<T>(logits, t * ld + e) : -__builtin_huge_valf();
        l[v] = l[v] == l[v] ? fminf(l[v], 3.402823466e38f) : -__builtin_huge_valf();
        top = fmaxf(top, l[v]);
    }
    // (exp and the sigmoid lose the order of logits that are far apart or large)
    const bool by_logit = bias == nullptr && (d.groups == 1 || d.group_best == 1);
    double total = 1.0;
    if (d.score == IGEMM_SOFTMAX) {
        for (int x = 32; x > 0; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
        total = 0.0;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool in = l[v] > -__builtin_huge_valf();
        if (d.score == IGEMM_SOFTMAX) {
            s[v] = in ? exp((double)l[v] - (double)top) : 0.0;
            total += s[v];
        } else {
            s[v] = in ? 1.0 / (1.0 + exp(-(double)l[v])) : 0.0;
        }
    }
    if (d.score == IGEMM_SOFTMAX) {
        for (int x = 32; x > 0; x /= 2) total += __shfl_xor(total, x);
        if (total == 0.0) total = 1.0;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = 64 * v + lane;
        const bool in = l[v] > -__builtin_huge_valf();
        s[v] /= total;
        key[v] = !in ? kNone : by_logit ? (double)l[v] : s[v] + (bias != nullptr ? (double)bias[e] : 0.0);
        if (!(key[v] == key[v])) key[v] = kNone;
    }
    if (d.groups > 1) {
        const int size = d.experts / d.groups;
#pragma unroll
        for (int v = 0; v < V; ++v) key_s[64 * v + lane] = key[v];
        __syncthreads();
        // lane g: its group's best one or two
        double a = kNone, b = kNone;
        if (lane < d.groups)
            for (int e = lane * size; e < (lane + 1) * size; ++e) {
                const double x = key_s[e];
                if (x > a) {
                    b = a;
                    a = x;
                } else if (x > b) {
                    b = x;
                }
            }
        double score = d.group_best == 2 && b > kNone ? a + b : a;
        uint64_t kept = 0;
        for (int c = 0; c < d.top_groups; ++c) {
            double k = score;
            int i = k > kNone ? lane : -1;
            wave_best(k, i);
            if (i < 0) break;
            kept |= 1ull << i;
            if (lane == i) score = kNone;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (!((kept >> ((64 * v + lane) / size & 63)) & 1)) key[v] = kNone;
    }
    double mine = 0.0, sum = 0.0;
    int id = -1;
    for (int c = 0; c < d.top_k; ++c) {
        double k = kNone, sc = 0.0;
        int i = -1;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (key[v] > k) {
                k = key[v];
                i = 64 * v + lane;
                sc = s[v];
            }
        const int own = i;
        wave_best(k, i);
        if (i < 0) break;
        sc = __shfl(own == i ? sc : 0.0, i & 63);
        sum += sc;
        if (lane == c) {
            mine = sc;
            id = i;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (64 * v + lane == i) key[v] = kNone;
    }
    if (lane < d.top_k) {
        double w = mine;
        if (d.renormalise) w = sum > 0.0 ? w / sum : 0.0;
        ids[t * d.top_k + lane] = id;
        weights[t * d.top_k + lane] = (float)(w * (double)d.scale);
    }
}

// One workgroup an expert: where it begins, and its slots in order.
__global__ void __launch_bounds__(256)
plan_plain(const int32_t *__restrict__ ids, int slots, int experts, int32_t *__restrict__ offsets,
           int32_t *__restrict__ order) {
    const int e = blockIdx.x, tid = threadIdx.x;   // e == experts: the end
    __shared__ int cnt[256];
    int below = 0;
    for (int s = tid; s < slots; s += 256) below += ids[s] >= 0 && ids[s] < e;
    cnt[tid] = below;
    __syncthreads();
    for (int d = 128; d > 0; d /= 2) {
        if (tid < d) cnt[tid] += cnt[tid + d];
        __syncthreads();
    }
    int at = cnt[0];
    __syncthreads();
    if (tid == 0) offsets[e] = at;
    if (e == experts) {
        for (int s = at + tid; s < slots; s += 256) order[s] = -1;
        return;
    }
    for (int s0 = 0; s0 < slots; s0 += 256) {
        const bool mine = s0 + tid < slots && ids[s0 + tid] == e;
        cnt[tid] = mine;
        __syncthreads();
        for (int d = 1; d < 256; d *= 2) {
            const int x = tid >= d ? cnt[tid - d] : 0;
            __syncthreads();
            cnt[tid] += x;
            __syncthreads();
        }
        if (mine) order[at + cnt[tid] - 1] = s0 + tid;
        at += cnt[255];
        __syncthreads();
    }
}

template <int V>
const void *pick(int type) {
    return type == IGEMM_F32    ? (const void *)route_tokens<V, IGEMM_F32>
           : type == IGEMM_BF16 ? (const void *)route_tokens<V, IGEMM_BF16>
                                : (const void *)route_tokens<V, IGEMM_F16>;
}

}  // namespace

int64_t route_workspace(const igemm_route_desc &d, bool plan) { return 0; }

int launch_route(const igemm_route_desc &d, const void *logits, int64_t ld, const float *bias,
                 int32_t *ids, float *weights, int32_t *offsets, int32_t *order, void *workspace,
                 void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    if (d.tokens > 0) {
        const void *fn = d.experts <= 64    ? pick<1>(d.type)
                         : d.experts <= 128 ? pick<2>(d.type)
                         : d.experts <= 256 ? pick<4>(d.type)
                         : d.experts <= 512 ? pick<8>(d.type)
                                            : pick<16>(d.type);
        igemm_route_desc dd = d;
        void *args[] = {&dd, (void *)&logits, &ld, (void *)&bias, &ids, &weights};
        if (hipLaunchKernel(fn, dim3((unsigned)d.tokens), dim3(64), args, 0, stream) != hipSuccess)
            return IGEMM_EHIP;
    }
    if (offsets != nullptr)
        plan_plain<<<dim3((unsigned)d.experts + 1), 256, 0, stream>>>(
            ids, (int)(d.tokens * d.top_k), d.experts, offsets, order);
    return hipGetLastError() == hipSuccess ? IGEMM_OK : IGEMM_EHIP;
}

}  // namespace rows
}  // namespace igemm
