// Routing of tokens to experts, and the plan of the experts' products.
//
// A wave a token, expert e = 64 v + lane in register v. The top_k largest keys
// are found by their bits: a threshold is built from the highest bit down, a
// ballot and a population count telling how many keys reach it, and the search
// ends as soon as that is top_k (some 20 steps of a compare a register and scalar
// work, where top_k rounds of a maximum over the wave take six exchanges each).
// The chosen then move to the first lanes, where each counts the ones before it.
//
// Keys are compared as 64-bit floating point: with 32 bits about one token in a
// few thousand has an expert within rounding of the border of the chosen ones,
// and which side it falls on would depend on the order of the softmax's sum.
// Where the keys are in the order of the logits (no bias, and one group or groups
// by their best), the logits' 32 bits are compared instead, and exp is taken of
// the chosen ones alone.
//
// Bound by latency: a launch, one round of loads and the search's dependent steps, and
// straight-line code costs the fetch of its instructions (unrolled or two bits a step the
// search is slower); for many tokens by the issue of instructions (two workgroups a
// compute unit are no faster). 8 tokens of 64 experts with their plan 6 us in one launch;
// 4096 of 256 in 8 groups 13 us and 9 for the plan; 16384 of 128 18.5 us and 8.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_rows_device.h"

namespace igemm {
namespace rows {
namespace {

// Unsigned integers in the order of the floating point numbers, all above 0,
// which stands for an excluded expert. (-0 is made +0 by the callers.)
__device__ __forceinline__ u32 ordered(float x) {
    const u32 b = __builtin_bit_cast(u32, x);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double unordered(uint64_t k) {
    return __builtin_bit_cast(double, k >> 63 ? k & 0x7fffffffffffffffull : ~k);
}
__device__ __forceinline__ double read_lane(double x, int l) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const u32 lo = (u32)__builtin_amdgcn_readlane((int)(u32)b, l);
    const u32 hi = (u32)__builtin_amdgcn_readlane((int)(u32)(b >> 32), l);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint64_t read_lane(uint64_t x, int l) {
    return __builtin_bit_cast(uint64_t, read_lane(__builtin_bit_cast(double, x), l));
}
__device__ __forceinline__ u32 read_lane(u32 x, int l) {
    return (u32)__builtin_amdgcn_readlane((int)x, l);
}
__device__ __forceinline__ int below_me(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((u32)(mask >> 32), __builtin_amdgcn_mbcnt_lo((u32)mask, 0));
}

// Wave-wide maximum and sum by data-parallel moves: within pairs, quads, halves of a
// row of 16, rows, then a row's last lane to the next row and the half's to the
// next half; lane 63 has it all. (Exchanges through LDS take an address and a wait
// each.)
template <int CTRL, int ROWS>
__device__ __forceinline__ u32 moved(u32 x) {
    return (u32)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float max_step(float x) {
    return fmaxf(x, __builtin_bit_cast(float, moved<CTRL, ROWS>(__builtin_bit_cast(u32, x))));
}
__device__ __forceinline__ float wave_max(float x) {
    x = max_step<0xb1, 0xf>(x);   // lanes 1 0 3 2 of a quad
    x = max_step<0x4e, 0xf>(x);   // 2 3 0 1
    x = max_step<0x141, 0xf>(x);  // mirror of half a row
    x = max_step<0x140, 0xf>(x);  // mirror of a row
    x = max_step<0x142, 0xa>(x);  // lane 15 of a row to the next (rows 1 and 3)
    x = max_step<0x143, 0xc>(x);  // lane 31 to rows 2 and 3
    return __builtin_bit_cast(
        float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double sum_step(double x) {
    // rows that are not written add 0
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const u32 lo = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)b, CTRL, ROWS, 0xf, false);
    const u32 hi = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)(b >> 32), CTRL, ROWS, 0xf, false);
    return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) {
    x = sum_step<0xb1, 0xf>(x);
    x = sum_step<0x4e, 0xf>(x);
    x = sum_step<0x141, 0xf>(x);
    x = sum_step<0x140, 0xf>(x);
    x = sum_step<0x142, 0xa>(x);
    x = sum_step<0x143, 0xc>(x);
    return read_lane(x, 63);
}

// 1 / x for x from 1e-290 to 1.79e308: the hardware's estimate and two Newton steps, within
// two units of the last place, those of numbers below the normal range from 4.5e307 on (the
// compiler's division, three times the instructions, also covers what x cannot be here).
__device__ __forceinline__ double reciprocal(double x) {
    double r = __builtin_amdgcn_rcp(x);
    r = fma(fma(-x, r, 1.0), r, r);
    return fma(fma(-x, r, 1.0), r, r);
}

template <bool WIDE>
struct KeyOf {
    typedef u32 type;
};
template <>
struct KeyOf<true> {
    typedef uint64_t type;
};

// A wave's LDS: the keys by expert (groups), then the chosen ones.
template <int V, bool WIDE>
struct Scratch {
    typename KeyOf<WIDE>::type key[64 * V];
    typename KeyOf<WIDE>::type best[64];
    float logit[64];
    int index[64];
};

// LDS written by lanes of a wave and read by others of the same wave.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A token's logits: expert 64 v + lane in x[v]. Every lane loads, a clamped place if
// need be: a load under a branch is waited for before the next one is issued.
template <int V, int T>
__device__ __forceinline__ void load_token(const igemm_route_desc &d, int64_t t,
                                           const void *__restrict__ logits, int64_t ld,
                                           float (&x)[V]) {
    const int lane = threadIdx.x & 63;
    const int64_t at = min(t, d.tokens - 1) * ld;
    float y[V];
#pragma unroll
    for (int v = 0; v < V; ++v) y[v] = get<T>(logits, at + min(64 * v + lane, d.experts - 1));
#pragma unroll
    for (int v = 0; v < V; ++v)
        x[v] = 64 * v + lane < d.experts ? y[v] : -__builtin_huge_valf();
}

// Returns the lane's chosen expert, or -1.
template <int V, bool WIDE>
__device__ int route_token(const igemm_route_desc &d, int64_t t, const float (&l_in)[V],
                           const float *__restrict__ bias, int32_t *__restrict__ ids,
                           float *__restrict__ weights, Scratch<V, WIDE> &sc) {
    typedef typename KeyOf<WIDE>::type key_t;
    constexpr int BITS = (int)sizeof(key_t) * 8;
    const float none = -__builtin_huge_valf();
    const int lane = threadIdx.x & 63;
    float l[V];
    key_t key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float x = l_in[v];
        // (x + 0: no -0)
        l[v] = x == x ? fminf(x, 3.402823466e38f) + 0.0f : none;
    }
    const bool all = WIDE || !d.renormalise;  // every expert's score is needed
    float top = 0.0f;
    double total = 1.0;
    if (all && d.score == IGEMM_SOFTMAX) {
        top = none;
#pragma unroll
        for (int v = 0; v < V; ++v) top = fmaxf(top, l[v]);
        top = wave_max(top);
        total = 0.0;
    }
    auto score = [&](float x) -> double {  // before the division by total
        if (d.score == IGEMM_SOFTMAX) return exp((double)x - (double)top);
        // (from -709.7827 on exp overflows and the score is 0)
        return x > -709.7827f ? reciprocal(1.0 + exp(-(double)x)) : 0.0;
    };
    if constexpr (WIDE) {
        // One copy of exp for all registers, through the scratch (rolled: what a wave
        // runs once costs the fetch of its instructions more than their execution).
#pragma unroll
        for (int v = 0; v < V; ++v) sc.key[64 * v + lane] = __builtin_bit_cast(u32, l[v]);
        double sum = 0.0;
#pragma unroll 1
        for (int e = lane; e < 64 * V; e += 64) {
            const float x = __builtin_bit_cast(float, (u32)sc.key[e]);
            const double y = x > none ? score(x) : 0.0;
            sum += y;
            sc.key[e] = __builtin_bit_cast(uint64_t, y);
        }
        if (d.score == IGEMM_SOFTMAX) {
            total = wave_sum(sum);
            if (total == 0.0) total = 1.0;
        }
        const double share = reciprocal(total);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float b = bias != nullptr ? bias[min(64 * v + lane, d.experts - 1)] : 0.0f;
            const double k =
                __builtin_bit_cast(double, sc.key[64 * v + lane]) * share + (double)b;
            key[v] = l[v] > none && k > -__builtin_huge_val() ? ordered(k + 0.0) : 0;
        }
    } else {
        if (all && d.score == IGEMM_SOFTMAX) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const double x = score(l[v] > none ? l[v] : 0.0f);
                total += l[v] > none ? x : 0.0;
            }
            total = wave_sum(total);
            if (total == 0.0) total = 1.0;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = l[v] > none ? ordered(l[v]) : 0;
    }

    // ---- groups -----------------------------------------------------------------
    if (d.groups > 1) {
        const int size = d.experts / d.groups;
        const float per_size = 1.0f / (float)size;
        int per = 1, lg = 0;  // lanes a group: a power of two
        while (2 * per * d.groups <= 64) per *= 2, ++lg;
#pragma unroll
        for (int v = 0; v < V; ++v) sc.key[64 * v + lane] = key[v];
        wave_sync();
        const int g = lane >> lg, sub = lane & (per - 1);
        key_t a = 0, b = 0;  // the best two
        if (g < d.groups)
            for (int e = sub; e < size; e += per) {
                const key_t x = sc.key[g * size + e];
                b = x > a ? a : (x > b ? x : b);
                a = x > a ? x : a;
            }
        for (int x = 1; x < per; x *= 2) {
            const key_t oa = __shfl_xor(a, x), ob = __shfl_xor(b, x);
            const key_t lo = a < oa ? a : oa;
            a = a < oa ? oa : a;
            b = b < ob ? ob : b;
            b = b < lo ? lo : b;
        }
        key_t mine = a;
        if constexpr (WIDE) {
            if (d.group_best == 2 && b != 0) mine = ordered(unordered(a) + unordered(b) + 0.0);
        }
        int rank = 0;
        for (int x = 0; x < d.groups; ++x) {
            const key_t other = read_lane(mine, x << lg);
            rank += other > mine || (other == mine && x < g);
        }
        // bit x << lg: group x stays
        const uint64_t kept = __ballot(g < d.groups && mine != 0 && rank < d.top_groups);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            // (experts and sizes up to 1024: the product is far from any integer)
            const int x = min((int)((64 * v + lane + 0.5f) * per_size), d.groups - 1);
            if (!((kept >> (x << lg)) & 1)) key[v] = 0;
        }
    }

    // ---- the top_k --------------------------------------------------------------
    // The search runs on the keys' high words and goes on to the low ones only if
    // these leave more than top_k of them.
    u32 hi[V];
#pragma unroll
    for (int v = 0; v < V; ++v) hi[v] = (u32)(key[v] >> (BITS - 32));
    auto reach = [&](u32 th) -> int {
        int c = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) c += __popcll(__ballot(hi[v] >= th));
        return c;
    };
    // (every key above 0 has a high word above 0)
    const int k = min(d.top_k, reach(1));
    key_t th = 0;
    if (k > 0) {
        u32 th_hi = 0;
        int c = 0;
#pragma unroll 1
        for (int b = 31; b >= 0 && c != k; --b) {
            const u32 next = th_hi | 1u << b;
            const int n = reach(next);
            c = n >= k ? n : c;
            th_hi = n >= k ? next : th_hi;
        }
        th = (key_t)th_hi << (BITS - 32);
        if constexpr (WIDE) {
            if (c != k) {
                for (int b = 31; b >= 0; --b) {
                    const key_t next = th | (key_t)1 << b;
                    int n = 0;
#pragma unroll
                    for (int v = 0; v < V; ++v) n += __popcll(__ballot(key[v] >= next));
                    if (n >= k) th = next;
                    if (n == k) break;
                }
            }
        }
    }
    // keys above th, and of those equal to it the first ones that still fit
    int room = k;
#pragma unroll
    for (int v = 0; v < V; ++v) room -= __popcll(__ballot(key[v] > th));
    int base = 0;
    if (k > 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint64_t equal = __ballot(key[v] == th);
            const bool in = key[v] > th || (key[v] == th && below_me(equal) < room);
            room -= min(room, __popcll(equal));
            const uint64_t mask = __ballot(in);
            if (in) {
                const int at = base + below_me(mask);
                sc.best[at] = key[v];
                sc.logit[at] = l[v];
                sc.index[at] = 64 * v + lane;
            }
            base += __popcll(mask);
        }
    }
    wave_sync();
    // The chosen are in the order of their index: of equals the first comes first.
    const bool mine = lane < k;
    const key_t best = mine ? sc.best[lane] : 0;
    const float x = mine ? sc.logit[lane] : none;
    const int index = mine ? sc.index[lane] : -1;
    if (!all && d.score == IGEMM_SOFTMAX) {
        top = wave_max(x);  // the largest logit is among the chosen
    }
    const double s = mine ? score(x) * reciprocal(total) : 0.0;
    int rank = 0;
    double sum = 0.0;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        const key_t other = read_lane(best, j);
        rank += other > best || (other == best && j < lane);
        sum += read_lane(s, j);
    }
    double w = s;
    if (d.renormalise) w = sum > 1e-290 ? s * reciprocal(sum) : sum > 0.0 ? s / sum : 0.0;
    if (lane < d.top_k) {
        const int at = mine ? rank : lane;
        ids[t * d.top_k + at] = index;
        weights[t * d.top_k + at] = mine ? (float)(w * (double)d.scale) : 0.0f;
    }
    wave_sync();  // (the scratch is the next token's)
    return index;
}

// ---- the plan -------------------------------------------------------------------
//
// The slots of [s0, s1) into order, a run of consecutive slots a wave: the waves
// count their slots of each expert, the counts become each wave's first place,
// and each wave then takes its slots 64 at a time, in order; lanes of the same
// expert find each other by one ballot for each bit of the index. start[e]: the
// place of this range's first slot of expert e.
template <int WAVES>
__device__ void place_slots(const int32_t *ids, int s0, int s1, int experts, int *start,
                            int *count /* WAVES x experts */, int32_t *order) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int e = tid; e < WAVES * experts; e += WAVES * 64) count[e] = 0;
    __syncthreads();
    const int run = ((s1 - s0 + WAVES - 1) / WAVES + 63) / 64 * 64;
    const int w0 = s0 + wave * run, w1 = min(w0 + run, s1);
    for (int s = w0 + lane; s < w1; s += 64) {
        const int id = ids[s];
        if (id >= 0) atomicAdd(&count[wave * experts + id], 1);
    }
    __syncthreads();
    for (int e = tid; e < experts; e += WAVES * 64) {
        int at = start[e];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int c = count[w * experts + e];
            count[w * experts + e] = at;
            at += c;
        }
    }
    __syncthreads();
    const int bits = 32 - __clz(experts);  // (ids and experts itself, for none)
    for (int s = w0; s < w1; s += 64) {
        const int id = s + lane < w1 ? ids[s + lane] : -1;
        const int x = id >= 0 ? id : experts;
        uint64_t same = ~0ull;
        for (int b = 0; b < bits; ++b) {
            const bool on = (x >> b) & 1;
            const uint64_t m = __ballot(on);
            same &= on ? m : ~m;
        }
        if (id >= 0) {
            const int rank = below_me(same);
            const int at = count[wave * experts + id];
            order[at + rank] = s + lane;
        }
        wave_sync();
        if (id >= 0 && below_me(same) == 0) count[wave * experts + id] += __popcll(same);
        wave_sync();
    }
}

// Exclusive sums of value[0 .. n), n <= 1024, in place; returns their total.
template <int WAVES>
__device__ int scan_experts(int *value, int n, int *waves /* WAVES */) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int carry = 0;
    for (int e0 = 0; e0 < n; e0 += WAVES * 64) {
        const int v = e0 + tid < n ? value[e0 + tid] : 0;
        int sum = v;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int up = __shfl_up(sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 63) waves[wave] = sum;
        __syncthreads();
        int before = carry;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) before += waves[w];
            carry += waves[w];
        }
        if (e0 + tid < n) value[e0 + tid] = before + sum - v;
        __syncthreads();
    }
    return carry;
}

// The whole plan by one workgroup.
template <int WAVES>
__device__ void plan_alone(const int32_t *ids, int slots, int experts, int32_t *offsets,
                           int32_t *order, int *start, int *count, int *waves) {
    const int tid = threadIdx.x;
    for (int e = tid; e < experts; e += WAVES * 64) start[e] = 0;
    __syncthreads();
    for (int s = tid; s < slots; s += WAVES * 64)
        if (ids[s] >= 0) atomicAdd(&start[ids[s]], 1);
    __syncthreads();
    const int total = scan_experts<WAVES>(start, experts, waves);
    for (int e = tid; e < experts; e += WAVES * 64) offsets[e] = start[e];
    if (tid == 0) offsets[experts] = total;
    for (int s = total + tid; s < slots; s += WAVES * 64) order[s] = -1;
    place_slots<WAVES>(ids, 0, slots, experts, start, count, order);
}

// ---- kernels ----------------------------------------------------------------------

// `each` tokens a wave, one after the other. counts (null: none wanted): the
// workgroup's slots of each expert go to counts[block][expert].
// (from 512 experts on, eight waves: their registers)
constexpr int waves_of(int experts) { return experts <= 256 ? 16 : 8; }
template <int V, int T, bool WIDE>
__global__ void __launch_bounds__(waves_of(64 * V) * 64)
route_tokens(igemm_route_desc d, const void *__restrict__ logits, int64_t ld,
             const float *__restrict__ bias, int32_t *ids, float *weights, int each,
             int32_t *__restrict__ counts) {
    constexpr int kWaves = waves_of(64 * V);
    __shared__ Scratch<V, WIDE> sc[kWaves];
    __shared__ int count[64 * V];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (counts != nullptr) {
        for (int e = threadIdx.x; e < d.experts; e += kWaves * 64) count[e] = 0;
        __syncthreads();
    }
    int64_t t = (int64_t)blockIdx.x * kWaves * each + wave;
    float l[V], ahead[V];
    load_token<V, T>(d, t, logits, ld, ahead);
    for (int x = 0; x < each && t < d.tokens; ++x, t += kWaves) {
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = ahead[v];
        if (x + 1 < each) load_token<V, T>(d, t + kWaves, logits, ld, ahead);
        const int id = route_token<V, WIDE>(d, t, l, bias, ids, weights, sc[wave]);
        if (counts != nullptr && id >= 0) atomicAdd(&count[id], 1);
    }
    if (counts != nullptr) {
        __syncthreads();
        const int row = (d.experts + 3) & ~3;  // (rows of whole 16 bytes)
        for (int e = threadIdx.x; e < row; e += kWaves * 64)
            counts[blockIdx.x * row + e] = e < d.experts ? count[e] : 0;
    }
}

// A few tokens: one workgroup routes them, a wave each, and makes the plan.
constexpr int kFewWaves = 16, kFewExperts = 256;
template <int V, int T, bool WIDE>
__global__ void __launch_bounds__(kFewWaves * 64)
route_few(igemm_route_desc d, const void *__restrict__ logits, int64_t ld,
          const float *__restrict__ bias, int32_t *ids, float *weights, int32_t *offsets,
          int32_t *order) {
    __shared__ union {
        Scratch<V, WIDE> sc[kFewWaves];
        int count[kFewWaves * 64 * V];
    } m;
    __shared__ int start[64 * V], waves[kFewWaves];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int t = wave; t < d.tokens; t += kFewWaves) {
        float l[V];
        load_token<V, T>(d, t, logits, ld, l);
        route_token<V, WIDE>(d, t, l, bias, ids, weights, m.sc[wave]);
    }
    __syncthreads();
    plan_alone<kFewWaves>(ids, (int)d.tokens * d.top_k, d.experts, offsets, order, start, m.count,
                          waves);
}

constexpr int kPlanWaves = 16;
__global__ void __launch_bounds__(kPlanWaves * 64)
plan_one(const int32_t *ids, int slots, int experts, int32_t *offsets, int32_t *order) {
    __shared__ int start[1024], waves[kPlanWaves];
    __shared__ int count[kPlanWaves * 1024];
    plan_alone<kPlanWaves>(ids, slots, experts, offsets, order, start, count, waves);
}

// Many slots: `join` of the blocks that route_tokens counted a workgroup, `block` slots
// each, placed after those of the experts, and of the workgroups, before.
__global__ void __launch_bounds__(kPlanWaves * 64)
plan_places(const int32_t *__restrict__ ids, int slots, int experts, int block, int blocks,
            int join, const int32_t *__restrict__ counts, int32_t *__restrict__ offsets,
            int32_t *__restrict__ order) {
    __shared__ int start[1024], before[1024], waves[kPlanWaves];
    __shared__ int count[kPlanWaves * 1024];
    const int tid = threadIdx.x, mine = blockIdx.x * join;
    const int64_t s0 = (int64_t)mine * block;
    const int64_t s1 = min(s0 + (int64_t)join * block, (int64_t)slots);
    for (int e = tid; e < experts; e += kPlanWaves * 64) start[e] = before[e] = 0;
    __syncthreads();
    // The sums over the blocks by `parts` threads for every four experts, so that the
    // loads of all are in flight together.
    const int fours = (experts + 3) / 4;
    int parts = 1;
    while (2 * parts * fours <= kPlanWaves * 64) parts *= 2;
    const int span = (blocks + parts - 1) / parts;
    for (int x = tid; x < parts * fours; x += kPlanWaves * 64) {
        const int part = x / fours, q = x - part * fours;
        const int b0 = part * span, b1 = min(b0 + span, blocks);
        v4i low = {0, 0, 0, 0}, all = {0, 0, 0, 0};
#pragma unroll 8
        for (int b = b0; b < b1; ++b) {
            const v4i c = ((const v4i *)counts)[b * fours + q];
            low += b < mine ? c : v4i{0, 0, 0, 0};
            all += c;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * q + i < experts) {
                atomicAdd(&start[4 * q + i], all[i]);
                atomicAdd(&before[4 * q + i], low[i]);
            }
    }
    __syncthreads();
    const int total = scan_experts<kPlanWaves>(start, experts, waves);
    if (blockIdx.x == 0) {
        for (int e = tid; e < experts; e += kPlanWaves * 64) offsets[e] = start[e];
        if (tid == 0) offsets[experts] = total;
    }
    __syncthreads();
    for (int e = tid; e < experts; e += kPlanWaves * 64) start[e] += before[e];
    for (int64_t s = max((int64_t)total, s0) + tid; s < s1; s += kPlanWaves * 64) order[s] = -1;
    __syncthreads();
    place_slots<kPlanWaves>(ids, (int)s0, (int)s1, experts, start, count, order);
}

template <int V>
const void *pick(int type, bool wide) {
    if (wide)
        return type == IGEMM_F32    ? (const void *)route_tokens<V, IGEMM_F32, true>
               : type == IGEMM_BF16 ? (const void *)route_tokens<V, IGEMM_BF16, true>
                                    : (const void *)route_tokens<V, IGEMM_F16, true>;
    return type == IGEMM_F32    ? (const void *)route_tokens<V, IGEMM_F32, false>
           : type == IGEMM_BF16 ? (const void *)route_tokens<V, IGEMM_BF16, false>
                                : (const void *)route_tokens<V, IGEMM_F16, false>;
}
template <int V>
const void *pick_few(int type, bool wide) {
    if (wide)
        return type == IGEMM_F32    ? (const void *)route_few<V, IGEMM_F32, true>
               : type == IGEMM_BF16 ? (const void *)route_few<V, IGEMM_BF16, true>
                                    : (const void *)route_few<V, IGEMM_F16, true>;
    return type == IGEMM_F32    ? (const void *)route_few<V, IGEMM_F32, false>
           : type == IGEMM_BF16 ? (const void *)route_few<V, IGEMM_BF16, false>
                                : (const void *)route_few<V, IGEMM_F16, false>;
}

// One workgroup places up to this many slots; of more, each workgroup places at
// least kRange.
constexpr int64_t kAlone = 8192, kRange = 2048;
// At most 256 workgroups of route_tokens, one a compute unit.
int64_t tokens_a_block(int64_t tokens, int experts) {
    const int64_t waves = waves_of(experts), each = (tokens + 256 * waves - 1) / (256 * waves);
    return (each > 1 ? each : 1) * waves;
}

}  // namespace

int64_t route_workspace(const igemm_route_desc &d, bool plan) {
    if (!plan || d.tokens * d.top_k <= kAlone) return 0;
    const int64_t per = tokens_a_block(d.tokens, d.experts);
    return ((d.tokens + per - 1) / per * ((d.experts + 3) / 4) * 16 + 255) / 256 * 256;
}

int launch_route(const igemm_route_desc &d, const void *logits, int64_t ld, const float *bias,
                 int32_t *ids, float *weights, int32_t *offsets, int32_t *order, void *workspace,
                 void *stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    const bool wide = bias != nullptr || (d.groups > 1 && d.group_best == 2);
    igemm_route_desc dd = d;
    const int slots = (int)(d.tokens * d.top_k);
    if (offsets != nullptr && d.tokens > 0 && d.tokens <= 2 * kFewWaves &&
        d.experts <= kFewExperts) {
        const void *fn = d.experts <= 64    ? pick_few<1>(d.type, wide)
                         : d.experts <= 128 ? pick_few<2>(d.type, wide)
                                            : pick_few<4>(d.type, wide);
        void *args[] = {&dd,  (void *)&logits, &ld, (void *)&bias, &ids, &weights, &offsets,
                        &order};
        return hipLaunchKernel(fn, dim3(1), dim3(kFewWaves * 64), args, 0, stream) == hipSuccess
                   ? IGEMM_OK
                   : IGEMM_EHIP;
    }
    const int per = (int)tokens_a_block(d.tokens, d.experts), blocks = (int)((d.tokens + per - 1) / per);
    const bool alone = slots <= kAlone;
    int32_t *counts = offsets == nullptr || alone ? nullptr : (int32_t *)workspace;
    if (d.tokens > 0) {
        const void *fn = d.experts <= 64    ? pick<1>(d.type, wide)
                         : d.experts <= 128 ? pick<2>(d.type, wide)
                         : d.experts <= 256 ? pick<4>(d.type, wide)
                         : d.experts <= 512 ? pick<8>(d.type, wide)
                                            : pick<16>(d.type, wide);
        const int waves = waves_of(d.experts);
        int each = per / waves;
        void *args[] = {&dd,  (void *)&logits, &ld,   (void *)&bias,
                        &ids, &weights,        &each, &counts};
        if (hipLaunchKernel(fn, dim3((unsigned)blocks), dim3((unsigned)waves * 64), args, 0, stream) !=
            hipSuccess)
            return IGEMM_EHIP;
    }
    if (offsets == nullptr) return IGEMM_OK;
    if (alone) {
        plan_one<<<dim3(1), kPlanWaves * 64, 0, stream>>>(ids, slots, d.experts, offsets, order);
    } else {
        const int64_t block = (int64_t)per * d.top_k;
        const int join = block < kRange ? (int)((kRange + block - 1) / block) : 1;
        plan_places<<<dim3((unsigned)((blocks + join - 1) / join)), kPlanWaves * 64, 0, stream>>>(
            ids, slots, d.experts, (int)block, blocks, join, counts, offsets, order);
    }
    return hipGetLastError() == hipSuccess ? IGEMM_OK : IGEMM_EHIP;
}

}  // namespace rows
}  // namespace igemm
