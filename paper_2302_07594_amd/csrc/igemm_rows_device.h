// Device helpers of the products whose rows choose their weights: conversions
// between float and the 16-bit types, and the rows that a position names.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "igemm_device.h"
#include "igemm_rows_find.h"
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
