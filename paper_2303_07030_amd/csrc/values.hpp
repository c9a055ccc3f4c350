// Rows of fp32 or bf16 values moved in wide accesses of any alignment, widened to
// 32 bits in registers.
#pragma once

#include <initializer_list>
#include <type_traits>

#include "aliasing.hpp"
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

// N columns from `col` on of a row of `width`, where a lane has some: at the row's end it steps
// back to the last N (the first of which are another lane's: store_cols leaves them), so that
// every lane moves whole pieces.  Rows of fewer than N columns are read and written one by one.
template <int N, class T>
__device__ __forceinline__ void load_cols(const T *row, int col, int width, float (&x)[N]) {
    if (width >= N) load_values<N, T>(row + min(col, width - N), x);
    else load_left<N, T>(row + min(col, width), max(width - col, 0), x);
}
template <int N, class T>
__device__ __forceinline__ void store_cols(T *row, int col, int width, const float (&x)[N]) {
    if (col + N <= width) {
        store_row_values<N, T>(row + col, x);
    } else if (width >= N) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (width - N + e >= col) row[width - N + e] = narrowed<T>(x[e]);
    } else {
        store_left<N, T>(row + min(col, width), max(width - col, 0), x);
    }
}

// The same as they lie in memory, to be widened where they are used: rows on their way take
// half the registers.  WIDE: rows have N columns at least.
template <int N, class T, bool WIDE>
struct Piece {
    uint32_t w[N * sizeof(T) / 4];
    __device__ __forceinline__ void load(const T *row, int col, int width) {
        if constexpr (WIDE) {
            __builtin_memcpy(w, row + min(col, width - N), sizeof w);
        } else {
            T t[N];
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = col + e < width ? row[col + e] : T(0);
            __builtin_memcpy(w, t, sizeof w);
        }
    }
    __device__ __forceinline__ float value(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
};

inline bool known_dtype(int32_t t) { return t == NSD_F32 || t == NSD_BF16; }
inline size_t dtype_bytes(int32_t t) { return t == NSD_F32 ? 4 : 2; }

// Rows of values of a call's type.
inline Area row_area(const void *p, int64_t rows, int64_t width, int64_t ld, int32_t dtype, int same = 0) {
    const int64_t b = (int64_t)dtype_bytes(dtype);
    return Area{p, rows, width * b, ld * b, same};
}

// What a call writes is apart from what it reads and from what else it writes.
inline nsd_status check_apart(std::initializer_list<Area> written, std::initializer_list<Area> read) {
    for (const Area *w = written.begin(); w != written.end(); ++w) {
        for (const Area &r : read)
            NSD_REQUIRE((w->same && w->same == r.same && w->p == r.p && w->ld == r.ld) || !areas_meet(*w, r),
                        "what is written shares memory with what is read");
        for (const Area *o = written.begin(); o != w; ++o)
            NSD_REQUIRE(!areas_meet(*w, *o), "what is written shares memory");
    }
    return NSD_OK;
}

}  // namespace nsd
