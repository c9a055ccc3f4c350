// Rows of fp32 or bf16 values moved in wide accesses of any alignment, widened to
// 32 bits in registers.
#pragma once

#include <type_traits>

#include "nsd_internal.hpp"

namespace nsd {

using Bf16 = uint16_t;  // a bfloat16 by its bits

__device__ __forceinline__ float widened(float x) { return x; }
__device__ __forceinline__ float widened(Bf16 x) { return __uint_as_float((uint32_t)x << 16); }

template <class T>
__device__ __forceinline__ T narrowed(float x) {
    if constexpr (sizeof(T) == 4) {
        return x;
    } else {
        const __bf16 r = static_cast<__bf16>(x);  // to nearest, ties to even
        return __builtin_bit_cast(Bf16, r);
    }
}

// N consecutive values at p (global memory takes accesses of any size at any
// address of the type).
template <int N, class T>
__device__ __forceinline__ void load_values(const T *p, float (&x)[N]) {
    T t[N];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = widened(t[e]);
}
template <int N, class T>
__device__ __forceinline__ void store_row_values(T *p, const float (&x)[N]) {
    T t[N];
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = narrowed<T>(x[e]);
    __builtin_memcpy(p, t, sizeof t);
}

// The same of a row's end: `left` values (any number, below N the first of them
// alone) exist; the others read 0 and are not written.
template <int N, class T>
__device__ __forceinline__ void load_left(const T *p, int left, float (&x)[N]) {
    if (left >= N) {
        load_values<N, T>(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = e < left ? widened(p[e]) : 0.f;
    }
}
template <int N, class T>
__device__ __forceinline__ void store_left(T *p, int left, const float (&x)[N]) {
    if (left >= N) {
        store_row_values<N, T>(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < left) p[e] = narrowed<T>(x[e]);
    }
}

inline bool known_dtype(int32_t t) { return t == NSD_F32 || t == NSD_BF16; }
inline size_t dtype_bytes(int32_t t) { return t == NSD_F32 ? 4 : 2; }

}  // namespace nsd
