// What the two families of differential attention kernels share: the call's
// shapes and arguments, the value types, the joins' view of a plan.
#pragma once

#include <algorithm>
#include <type_traits>

#include "nsd_internal.hpp"

namespace nsd {
namespace attn {

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / kWave;
// Blocks of one launch: a grid's threads are counted in 32 bits.
constexpr int64_t kMaxBlocks = UINT32_MAX / kAttnThreads;
constexpr int kMaxD = 128, kMaxDv = 256;
constexpr float kLog2e = 1.44269504088896340736f;

template <class T, int V>
__device__ __forceinline__ void store_values(T *p, const float (&x)[V]) {
    T t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        if constexpr (sizeof(T) == 4) {
            t[e] = x[e];
        } else {
            const __bf16 r = static_cast<__bf16>(x[e]);
            t[e] = __builtin_bit_cast(uint16_t, r);
        }
    }
    __builtin_memcpy(p, t, sizeof t);
}

template <class T>
__device__ __forceinline__ T narrow(float x) {
    T t[1];
    const float y[1] = {x};
    store_values<T, 1>(t, y);
    return t[0];
}

struct Shape {
    int32_t H, Hk, grp, d, dv;
    int64_t ldq, ldk, ldv, ldo;
    float scale;
    int32_t hps_log2;  // heads per slot (of queries; of keys in the column pass)
    int32_t nhb;       // groups of them
};

__device__ __forceinline__ float exp_diff(float s, float m) {
    return __builtin_amdgcn_exp2f((s - m) * kLog2e);
}
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// The blocks of one XCD take neighbouring work.
__device__ __forceinline__ int64_t near_block(int b, int nb) {
    const int x = b % 8;
    int start = 0;
    for (int y = 0; y < x; ++y) start += (nb - y + 7) / 8;
    return start + b / 8;
}

struct FwdArgs {
    Shape s;
    const void *Q, *K, *V;
    const float *lambda, *bias;
    void *O;
    float *stat;  // [rows][H][4]: maximum and sum of either map, or NULL
    float *part;  // [partial][H][4 + 2 dv]
    const int32_t *rowptr, *rowidx, *colind;
    // plan
    nsd_plan plan;
    int32_t nrows;
    // decode: splits of a row, entries of one
    int32_t nsplit, per;
    int64_t nmain;  // blocks that walk entries
    int32_t all_empty;
};

// Rows without entries: the empty sums.  One wave a row.
template <class T>
__device__ __forceinline__ void empty_row(const FwdArgs &a, int64_t row) {
    const int lane = threadIdx.x % kWave;
    T *o = static_cast<T *>(a.O) + row * a.s.ldo;
    for (int c = lane; c < a.s.H * a.s.dv; c += kWave) o[c] = T(0);
    if (a.stat)
        for (int c = lane; c < a.s.H * 4; c += kWave) a.stat[row * a.s.H * 4 + c] = 0.f;
}

// Calls f(segment) for the segments without entries that this wave takes: the
// blocks past the first nmain walk them all, four at a time each.
template <class F>
__device__ __forceinline__ void for_empty(const nsd_plan &plan, int nseg, int all, int64_t nmain,
                                          F f) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t end = all ? nseg : plan.nempty;
    const int64_t step = ((int64_t)gridDim.x - nmain) * kAttnWaves;
    for (int64_t n = ((int64_t)blockIdx.x - nmain) * kAttnWaves + wave; n < end; n += step)
        f(all ? n : (int64_t)plan.empty_seg[n]);
}

struct BwdArgs {
    Shape s;
    const void *Q, *K, *V, *dO;
    const float *lambda, *bias, *stat;
    void *dQ, *dK, *dV;
    float *coef;    // [nnz][H][3]: a^1, a^2, t; on the matrix cores [nnz][H][4]
    float *D;       // [rows][H][2]
    float *part;    // rows: [partial][H][2 + 4 d] (matrix cores: 2 d, and D apart);
                    // columns: [partial][Hk][2 d + dv]
    float *part_D;  // [partial][H][2]
    const int32_t *ptr, *idx, *other, *perm;
    nsd_plan plan;
    int32_t nseg;
    int64_t nmain;
    int32_t all_empty;
};

// Rows and columns without entries have no gradient.  One wave each.
template <class T>
__device__ __forceinline__ void empty_row(const BwdArgs &a, int64_t row) {
    const int lane = threadIdx.x % kWave;
    T *o = static_cast<T *>(a.dQ) + row * a.s.ldq;
    for (int c = lane; c < a.s.H * 2 * a.s.d; c += kWave) o[c] = T(0);
    for (int c = lane; c < a.s.H * 2; c += kWave) a.D[row * a.s.H * 2 + c] = 0.f;
}
template <class T>
__device__ __forceinline__ void empty_column(const BwdArgs &a, int64_t col) {
    const int lane = threadIdx.x % kWave;
    T *k = static_cast<T *>(a.dK) + col * a.s.ldk, *v = static_cast<T *>(a.dV) + col * a.s.ldv;
    for (int c = lane; c < a.s.Hk * 2 * a.s.d; c += kWave) k[c] = T(0);
    for (int c = lane; c < a.s.Hk * a.s.dv; c += kWave) v[c] = T(0);
}

// (row, first partial, partials) of the i-th long segment or decode row.
__device__ __forceinline__ void long_segment(const nsd_plan &plan, const int32_t *ptr, int nsplit,
                                             int64_t i, int64_t &row, int64_t &first,
                                             int64_t &n) {
    if (nsplit > 0) {
        row = i;
        first = i * nsplit;
        n = nsplit;
    } else {
        row = plan.long_seg[i];
        first = plan.chunk_ord[plan.long_first[i]];
        n = ((int64_t)ptr[row + 1] - ptr[row] + plan.item_len - 1) / plan.item_len;
    }
}

}  // namespace attn
}  // namespace nsd
