// The router of a sparse mixture: softmax over the experts, the top-k gates as
// the rows of a CSR, the use of every expert and the balance loss; and the
// gradient of gates and loss with respect to the logits.
//
//   p = softmax(x_t),  S = the k largest of x_t,  gate = p or p / sum_S p
//   n_e = tokens that chose e,  N = tokens routed
//   L = w E sum_e (n_e / sum n) (sum_t p_te / N)
//   dx_te = p_te (u_te - sum_e' p_te' u_te'),  u_te = seed w E n_e / (sum n N)
//           + [e in S] dgate_te; normalised gates: the same form over S alone
//
// HBM-bound in the large: the logits are read once in either direction.  A row
// of E logits lies on a slot of G lanes, NE consecutive ones a lane, so that a
// wave takes 64 / G rows at once: the k rounds of the selection cost every lane
// NE - 1 maxima and log2 G exchanges each, whatever the rows a wave takes, and
// few lanes with eight logits each make the fewest instructions a row.  The
// rounds compare unique keys: the logit's bits in an order of whole numbers,
// and below them the expert's number from the top, so that ties fall to the
// lowest expert and a round has one winner.
//
// Measured at 131,072 tokens of 128 experts, 8 chosen, bf16: gates and statistics 35
// us, totals 10, gradient 27 (2.8 TB/s); the first is bound by the instructions of the
// selection.
#include <algorithm>
#include <type_traits>

#include "nsd_internal.hpp"

namespace nsd {

namespace {

// Threads of a block that gathers statistics, by the experts of a lane:
// sixteen and their sums do not fit the registers of 1024 threads.
constexpr int kRouteThreads = 1024;
constexpr int stat_threads(int ne) { return ne > 8 ? kRouteThreads / 2 : kRouteThreads; }
constexpr int kPlainThreads = 256;
constexpr int kMaxExperts = 1024;
constexpr int kMaxRouteBlocks = 256;  // one a CU; each leaves a partial sum

template <class T>
using Key = std::conditional_t<sizeof(T) == 2, uint32_t, uint64_t>;

// The value of the partner in a butterfly step of span M.  Written so that the
// exchange becomes an operand of the instruction that uses it (every lane has a
// partner, so what the bounds rule gives the others does not matter).
template <int M>
__device__ __forceinline__ uint32_t partner(uint32_t v) {
    constexpr int kControl = M == 1 ? 0xB1 : M == 2 ? 0x4E : M == 4 ? 0x141 : 0x140;
    if constexpr (M <= 8) return __builtin_amdgcn_update_dpp(0, (int)v, kControl, 0xF, 0xF, true);
    else return __float_as_uint(lane_xor<M>(__uint_as_float(v)));
}
template <int M>
__device__ __forceinline__ uint64_t partner(uint64_t v) {
    return (uint64_t)partner<M>((uint32_t)(v >> 32)) << 32 | partner<M>((uint32_t)v);
}
// Reductions over a slot of G lanes, the result in every lane.
template <int G, int M = 1, class V, class Op>
__device__ __forceinline__ V slot_reduce(V v, Op op) {
    if constexpr (M < G) {
        V o;
        if constexpr (std::is_same_v<V, float>)
            o = __uint_as_float(partner<M>(__float_as_uint(v)));
        else o = partner<M>(v);
        return slot_reduce<G, 2 * M>(op(v, o), op);
    } else {
        return v;
    }
}
template <int G, class V>
__device__ __forceinline__ V slot_max(V v) {
    return slot_reduce<G>(v, [](V a, V b) { return a > b ? a : b; });
}
template <int G>
__device__ __forceinline__ float slot_fmax(float v) {
    return slot_reduce<G>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int G, class V>
__device__ __forceinline__ V slot_sum(V v) {
    return slot_reduce<G>(v, [](V a, V b) { return a + b; });
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void narrow(float x, float *y) { *y = x; }
__device__ __forceinline__ void narrow(float x, uint16_t *y) {
    const __bf16 r = static_cast<__bf16>(x);
    *y = __builtin_bit_cast(uint16_t, r);
}

// This lane's experts [e0, e0 + NE) of a row; those past E read -infinity.
template <class T, int NE>
__device__ __forceinline__ void load_row(const T *row, int e0, int E, float (&x)[NE]) {
    if (e0 + NE <= E) {
        T t[NE];
        __builtin_memcpy(t, row + e0, sizeof t);
#pragma unroll
        for (int n = 0; n < NE; ++n) x[n] = widen(t[n]);
    } else {
#pragma unroll
        for (int n = 0; n < NE; ++n) x[n] = e0 + n < E ? widen(row[e0 + n]) : -INFINITY;
    }
}
template <class T, int NE>
__device__ __forceinline__ void store_row(T *row, int e0, int E, const float (&x)[NE]) {
    T t[NE];
#pragma unroll
    for (int n = 0; n < NE; ++n) narrow(x[n], &t[n]);
    if (e0 + NE <= E) {
        __builtin_memcpy(row + e0, t, sizeof t);
    } else {
#pragma unroll
        for (int n = 0; n < NE; ++n)
            if (e0 + n < E) row[e0 + n] = t[n];
    }
}

// 1 / a sum of e^(x - max): at least 1 where it is not 0, so that the hardware's
// reciprocal serves (within 1 ulp).
__device__ __forceinline__ float inverse(float s) {
    return s == 0.f ? 0.f : __builtin_amdgcn_rcpf(s);
}

// e^(x - max) of a row and 1 / its sum over the row.  A row without a finite
// logit has no probabilities (all 0); one with NaN or +infinity only NaN.
template <int G, int NE>
__device__ __forceinline__ float softmax_row(const float (&x)[NE], float (&e)[NE]) {
    float m = x[0];
#pragma unroll
    for (int n = 1; n < NE; ++n) m = fmaxf(m, x[n]);
    m = slot_fmax<G>(m);
    m = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int n = 0; n < NE; ++n) {
        e[n] = __builtin_amdgcn_exp2f((x[n] - m) * 1.44269504088896340736f);
        s += e[n];
    }
    return inverse(slot_sum<G>(s));
}

// Unique keys in the order of (logit, -expert); NaN above all, -0 with +0.
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0xFFFFFFFFu : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
template <class T>
__device__ __forceinline__ Key<T> make_key(float x, int e) {
    if constexpr (sizeof(T) == 2) return (order_bits(x) & 0xFFFF0000u) | (uint32_t)(0xFFFF - e);
    else return (uint64_t)order_bits(x) << 32 | (uint32_t)(0x7FFFFFFF - e);
}

struct RouteArgs {
    int32_t T, E, k, norm;
    int64_t ld;
    const void *x;
    const uint8_t *skip;
    int32_t *col;
    float *gate;
    // statistics
    float weight;
    double *part_p;
    int32_t *part_n;  // [blocks][E + 1]
    int32_t *counts;
    double *loss;
};

// Descending order of 8 or 16 keys by merging sorted halves (odd and even
// places apart).
template <int LO, int N, int STEP, int NE, class K>
__device__ __forceinline__ void merge_keys(K (&key)[NE]) {
    auto order = [&](int i, int j) {
        const K a = key[i], b = key[j];
        key[i] = a > b ? a : b;
        key[j] = a > b ? b : a;
    };
    if constexpr (2 * STEP < N) {
        merge_keys<LO, N, 2 * STEP>(key);
        merge_keys<LO + STEP, N, 2 * STEP>(key);
#pragma unroll
        for (int i = LO + STEP; i + STEP < LO + N; i += 2 * STEP) order(i, i + STEP);
    } else {
        order(LO, LO + STEP);
    }
}
template <int LO, int N, int NE, class K>
__device__ __forceinline__ void sort_keys(K (&key)[NE]) {
    if constexpr (N > 1) {
        sort_keys<LO, N / 2>(key);
        sort_keys<LO + N / 2, N / 2>(key);
        merge_keys<LO, N, 1>(key);
    }
}

// Keys of this lane's experts (0 past the last) and the smallest of the k chosen
// ones.  Each lane sorts its keys once; a round is then a maximum over the lanes'
// first keys and a step of the winner's list (without the sort, where a round
// looks through all of a lane's keys, the kernel took 50 us in place of 43 at
// 131K tokens of 128 experts).
template <class T, int G, int NE>
__device__ __forceinline__ Key<T> choose(int E, int k, const float (&x)[NE], int e0,
                                         Key<T> (&key)[NE]) {
    Key<T> list[NE];
#pragma unroll
    for (int n = 0; n < NE; ++n) {
        const Key<T> held = make_key<T>(x[n], e0 + n);
        list[n] = key[n] = e0 + n < E ? held : Key<T>(0);
    }
    sort_keys<0, NE>(list);
    Key<T> m = 0;
    for (int j = 0; j < k; ++j) {
        m = slot_max<G>(list[0]);
        const bool won = list[0] == m;
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            const Key<T> keep = list[n], next = n + 1 < NE ? list[n + 1] : Key<T>(0);
            list[n] = won ? next : keep;
        }
    }
    return m;
}
// The smallest key of an expert that is available (a logit above -infinity).
template <class T>
constexpr Key<T> kOpenKey = Key<T>(0x00800000u) << (sizeof(T) == 2 ? 0 : 32);

// Totals of all blocks (part[b] for b < nb) by one block: counts and the loss.
__device__ __forceinline__ void route_total(const RouteArgs &a, int nb) {
    __shared__ double sh_p[kRouteThreads];
    __shared__ int32_t sh_n[kRouteThreads];
    const int t = threadIdx.x, per = kRouteThreads / a.E;  // threads that share an expert
    const int e = t % a.E, q = t / a.E;
    double p = 0.0;
    int32_t n = 0;
    if (q < per) {
        // eight blocks' partials in flight
        constexpr int F = 8;
        for (int b0 = q; b0 < nb; b0 += F * per) {
            double x[F];
            int32_t y[F];
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int b = min(b0 + i * per, nb - 1);
                x[i] = a.part_p[(int64_t)b * a.E + e];
                y[i] = a.part_n[(int64_t)b * (a.E + 1) + e];
            }
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const bool in = b0 + i * per < nb;
                p += in ? x[i] : 0.0;
                n += in ? y[i] : 0;
            }
        }
    }
    sh_p[t] = p;
    sh_n[t] = n;
    __syncthreads();
    if (q == 0) {
        for (int o = 1; o < per; ++o) {
            p += sh_p[t + o * a.E];
            n += sh_n[t + o * a.E];
        }
        a.counts[e] = n;
    }
    __syncthreads();
    // sum_e n_e P_e and sum_e n_e in a fixed order
    sh_p[t] = q == 0 ? p * n : 0.0;
    sh_n[t] = q == 0 ? n : 0;
    __syncthreads();
    for (int w = kRouteThreads / 2; w >= 1; w >>= 1) {
        if (t < w) {
            sh_p[t] += sh_p[t + w];
            sh_n[t] += sh_n[t + w];
        }
        __syncthreads();
    }
    const double np = sh_p[0];
    const int32_t total = sh_n[0];
    __syncthreads();
    int32_t rows = 0;
    for (int b = t; b < nb; b += kRouteThreads) rows += a.part_n[(int64_t)b * (a.E + 1) + a.E];
    sh_n[t] = rows;
    __syncthreads();
    for (int w = kRouteThreads / 2; w >= 1; w >>= 1) {
        if (t < w) sh_n[t] += sh_n[t + w];
        __syncthreads();
    }
    if (t == 0) {
        rows = sh_n[0];
        a.counts[a.E] = rows;
        *a.loss = total > 0 && rows > 0 ? (double)a.weight * a.E * np / ((double)total * rows) : 0.0;
    }
}

// STATS: a block adds up its tokens' probabilities and choices, lane by lane,
// then in wave order, into one partial row (no atomics).
template <class T, int G, int NE, bool STATS>
__global__ __launch_bounds__(STATS ? stat_threads(NE) : kPlainThreads) void route_kernel(
    RouteArgs a) {
    constexpr int THREADS = STATS ? stat_threads(NE) : kPlainThreads;
    constexpr int WAVES = THREADS / kWave, RW = kWave / G;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int slot = lane / G, g = lane % G, e0 = g * NE;
    // Up to kFold tokens are added up in 32 bits (probabilities) and in bytes
    // (choices), those sums in 64 and 32.
    constexpr int kFold = 16, PK = NE / 4;
    double ps[NE];
    float near_p[NE];
    uint32_t near_n[PK];
    int32_t cnt[NE], rows = 0, held = 0;
    if constexpr (STATS) {
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            ps[n] = 0.0;
            near_p[n] = 0.f;
            near_n[n / 4] = 0;
            cnt[n] = 0;
        }
    }
    auto fold = [&]() {
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            ps[n] += near_p[n];
            cnt[n] += near_n[n / 4] >> 8 * (n % 4) & 0xFF;
            near_p[n] = 0.f;
        }
#pragma unroll
        for (int n = 0; n < PK; ++n) near_n[n] = 0;
        held = 0;
    };
    const int64_t step = (int64_t)gridDim.x * WAVES * RW;
    for (int64_t base = ((int64_t)blockIdx.x * WAVES + wave) * RW; base < a.T; base += step) {
        const int64_t t = min(base + slot, (int64_t)a.T - 1);
        const bool mine = base + slot < a.T;
        float x[NE], e[NE];
        load_row<T, NE>(static_cast<const T *>(a.x) + t * a.ld, e0, a.E, x);
        const bool on = !(a.skip && a.skip[t]);
        const float inv = softmax_row<G, NE>(x, e);
        Key<T> key[NE];
        const Key<T> m = choose<T, G, NE>(a.E, a.k, x, e0, key);
        uint32_t sel = 0;
        float scale = 0.f;
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            sel |= key[n] >= m ? 1u << n : 0u;
            scale += key[n] >= m ? e[n] : 0.f;
        }
        scale = a.norm ? inverse(slot_sum<G>(scale)) : inv;
        if constexpr (STATS) {
            uint32_t counted = sel;
            if (__any(m < kOpenKey<T>)) {  // fewer than k available
                counted = 0;
#pragma unroll
                for (int n = 0; n < NE; ++n)
                    counted |= key[n] >= max(m, kOpenKey<T>) ? 1u << n : 0u;
            }
            if (mine && on) {
#pragma unroll
                for (int n = 0; n < NE; ++n) near_p[n] += e[n] * inv;
#pragma unroll
                for (int n = 0; n < PK; ++n)
                    near_n[n] += __umul24(counted >> 4 * n & 0xF, 0x204081) & 0x01010101;
                rows += inv != 0.f;
            }
            if (++held == kFold) fold();
        }
        // a token that is not routed stores zeros at the first k experts
        if (!on) {
            sel = 0;
#pragma unroll
            for (int n = 0; n < NE; ++n) sel |= e0 + n < a.k ? 1u << n : 0u;
        }
        // places before this lane's in the row
        int rank = __popc(sel);
        const int own = rank;
#pragma unroll
        for (int m = 1; m < G; m <<= 1) {
            const int o = __shfl_up(rank, m, G);
            rank += g >= m ? o : 0;
        }
        rank -= own;
        // the wave's rows lie together: one address, and 32-bit places from it
        const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane((int)base) * a.k;
        int32_t *const col = a.col + first;
        float *const gate = a.gate + first;
        uint32_t to = slot * a.k + rank;
        sel = mine ? sel : 0u;
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            if (sel >> n & 1) {
                col[to] = e0 + n;
                gate[to] = on ? e[n] * scale : 0.f;
                ++to;
            }
        }
    }
    if constexpr (STATS) {
        __shared__ double sh_p[G * NE];
        __shared__ int32_t sh_n[G * NE + 1];
        fold();
        // slots of the wave
#pragma unroll
        for (int n = 0; n < NE; ++n) {
#pragma unroll
            for (int m = G; m < kWave; m <<= 1) ps[n] += __shfl_xor(ps[n], m, kWave);
#pragma unroll
            for (int m = G; m < kWave; m <<= 1) cnt[n] += __shfl_xor(cnt[n], m, kWave);
        }
#pragma unroll
        for (int m = G; m < kWave; m <<= 1) rows += __shfl_xor(rows, m, kWave);
        for (int w = 0; w < WAVES; ++w) {
            if (wave == w && slot == 0) {
#pragma unroll
                for (int n = 0; n < NE; ++n) {
                    sh_p[e0 + n] = (w ? sh_p[e0 + n] : 0.0) + ps[n];
                    sh_n[e0 + n] = (w ? sh_n[e0 + n] : 0) + cnt[n];
                }
                if (g == 0) sh_n[G * NE] = (w ? sh_n[G * NE] : 0) + rows;
            }
            __syncthreads();
        }
        for (int e = threadIdx.x; e < a.E; e += THREADS) {
            a.part_p[(int64_t)blockIdx.x * a.E + e] = sh_p[e];
            a.part_n[(int64_t)blockIdx.x * (a.E + 1) + e] = sh_n[e];
        }
        if (threadIdx.x == 0) a.part_n[(int64_t)blockIdx.x * (a.E + 1) + a.E] = sh_n[G * NE];
        if constexpr (THREADS == kRouteThreads) {
            if (gridDim.x == 1) {  // the only block reads its own row back
                __syncthreads();
                route_total(a, 1);
            }
        }
    }
}

__global__ __launch_bounds__(kRouteThreads) void route_total_kernel(RouteArgs a, int nb) {
    route_total(a, nb);
}

// Orders a wave's LDS accesses (the hardware takes them in order: this is for the
// compiler).
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct VjpArgs {
    int32_t T, E, k, norm;
    int64_t ld;
    const void *x;
    const uint8_t *skip;
    const int32_t *col;
    const float *gate;
    const int32_t *counts;
    float scale;  // seed w E
    const float *dgate;
    void *dx;
};

template <class T, int G, int NE>
__global__ __launch_bounds__(kPlainThreads) void route_vjp_kernel(VjpArgs a) {
    constexpr int WAVES = kPlainThreads / kWave, RW = kWave / G;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int slot = lane / G, g = lane % G, e0 = g * NE;
    // one row's contributions of the gates, by expert
    __shared__ float sh[WAVES][RW][G * NE];
    float *mine = sh[wave][slot];
    float u[NE];  // the balance loss's part, the same for every token
    {
        float n_all = 0.f, n[NE];
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            n[i] = a.counts && e0 + i < a.E ? (float)a.counts[e0 + i] : 0.f;
            n_all += n[i];
        }
        n_all = slot_sum<G>(n_all);
        const float rows = a.counts ? (float)a.counts[a.E] : 0.f;
        const float c = n_all > 0.f && rows > 0.f ? a.scale / n_all / rows : 0.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) u[i] = c * n[i];
    }
    const int64_t step = (int64_t)gridDim.x * WAVES * RW;
    for (int64_t base = ((int64_t)blockIdx.x * WAVES + wave) * RW; base < a.T; base += step) {
        const int64_t t = min(base + slot, (int64_t)a.T - 1);
        const bool in = base + slot < a.T;
        float x[NE], e[NE], d[NE], b[NE];
        load_row<T, NE>(static_cast<const T *>(a.x) + t * a.ld, e0, a.E, x);
        const bool on = !(a.skip && a.skip[t]);
#pragma unroll
        for (int n = 0; n < NE; ++n) b[n] = 0.f;
        if (a.dgate) {
            // the row's entries, one a lane (all of them where k <= G)
            const int64_t o = t * a.k;
            const int j0 = min(g, a.k - 1);
            const int c0 = a.col[o + j0];
            const float dg0 = a.dgate[o + j0], ga0 = a.norm ? a.gate[o + j0] : 0.f;
            // a closed expert's gate is 0, and its gradient may be anything
            auto part = [](float ga, float dg) { return ga != 0.f ? ga * dg : 0.f; };
            float dot = 0.f;
            if (a.norm) {
                dot = g < a.k ? part(ga0, dg0) : 0.f;
                for (int j = g + G; j < a.k; j += G) dot += part(a.gate[o + j], a.dgate[o + j]);
                dot = slot_sum<G>(dot);
            }
#pragma unroll
            for (int n = 0; n < NE; ++n) mine[e0 + n] = 0.f;
            wave_fence();
            auto put = [&](int c, float ga, float dg) {
                if ((unsigned)c < (unsigned)a.E) mine[c] = a.norm ? part(ga, dg - dot) : dg;
            };
            if (g < a.k) put(c0, ga0, dg0);
            for (int j = g + G; j < a.k; j += G)
                put(a.col[o + j], a.norm ? a.gate[o + j] : 0.f, a.dgate[o + j]);
            wave_fence();
#pragma unroll
            for (int n = 0; n < NE; ++n) b[n] = x[n] == -INFINITY ? 0.f : mine[e0 + n];
            wave_fence();
        }
        const float inv = softmax_row<G, NE>(x, e);
        float dot = 0.f;
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            e[n] *= inv;
            d[n] = a.norm ? u[n] : u[n] + b[n];
            dot += e[n] * d[n];
        }
        dot = slot_sum<G>(dot);
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            d[n] = e[n] * (d[n] - dot);
            if (a.norm) d[n] += b[n];
            if (!on) d[n] = 0.f;
        }
        if (in) store_row<T, NE>(static_cast<T *>(a.dx) + t * a.E, e0, a.E, d);
    }
}

// Slot of a row: eight experts a lane on as few lanes as hold them, sixteen
// above 512 experts.
template <class T, class F>
void with_slot(int E, F f) {
    using std::integral_constant;
    if (E <= 8) f(T(), integral_constant<int, 1>(), integral_constant<int, 8>());
    else if (E <= 16) f(T(), integral_constant<int, 2>(), integral_constant<int, 8>());
    else if (E <= 32) f(T(), integral_constant<int, 4>(), integral_constant<int, 8>());
    else if (E <= 64) f(T(), integral_constant<int, 8>(), integral_constant<int, 8>());
    else if (E <= 128) f(T(), integral_constant<int, 16>(), integral_constant<int, 8>());
    else if (E <= 256) f(T(), integral_constant<int, 32>(), integral_constant<int, 8>());
    else if (E <= 512) f(T(), integral_constant<int, 64>(), integral_constant<int, 8>());
    else f(T(), integral_constant<int, 64>(), integral_constant<int, 16>());
}
template <class F>
void with_types(const nsd_router *s, F f) {
    if (s->dtype == NSD_BF16) with_slot<uint16_t>(s->experts, f);
    else with_slot<float>(s->experts, f);
}

int slot_lanes(int E) {
    int g = 1;
    while (g < 64 && g * 8 < E) g <<= 1;
    return g;
}

// Blocks that gather statistics: each wave takes a group of rows at least.  One
// block makes the totals itself, so a second launch is spared where two would
// do (above 512 experts a block has too few threads for that).
int stat_blocks(int32_t T, int E) {
    const bool small = E <= 512;
    const int64_t per = (int64_t)stat_threads(small ? 8 : 16) / slot_lanes(E);
    const int64_t nb = std::min<int64_t>(ceil_div(std::max(T, 1), per), kMaxRouteBlocks);
    return nb > 2 ? (int)nb : small ? 1 : 2;
}

nsd_status check_router(int32_t ntok, const nsd_router *s) {
    NSD_REQUIRE(s != nullptr, "router descriptor is NULL");
    NSD_REQUIRE(ntok >= 0, "negative number of tokens");
    NSD_REQUIRE(s->experts >= 1 && s->topk >= 1 && s->topk <= s->experts,
                "%d of %d experts", s->topk, s->experts);
    NSD_REQUIRE(s->dtype == NSD_F32 || s->dtype == NSD_BF16, "unknown type %d", s->dtype);
    NSD_REQUIRE(s->ld >= s->experts, "rows of %lld values hold %d experts", (long long)s->ld,
                s->experts);
    if (s->experts > kMaxExperts)
        return fail(NSD_ERR_UNSUPPORTED, "%d experts (at most %d)", s->experts, kMaxExperts);
    if ((int64_t)ntok * s->topk > INT32_MAX)
        return fail(NSD_ERR_TOO_LARGE, "%d tokens of %d entries", ntok, s->topk);
    return NSD_OK;
}

struct RouteWs {
    double *p;
    int32_t *n;
};
size_t carve_route(void *ws, int32_t ntok, int E, RouteWs *out) {
    const int nb = stat_blocks(ntok, E);
    Carver c(ws);
    out->p = c.take<double>((size_t)nb * E);
    out->n = c.take<int32_t>((size_t)nb * (E + 1));
    return c.bytes();
}

}  // namespace

}  // namespace nsd

using namespace nsd;

extern "C" {

nsd_status nsd_route_workspace_size(int32_t ntok, const nsd_router *s, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_TRY(check_router(ntok, s));
    RouteWs w;
    *bytes = carve_route(nullptr, ntok, s->experts, &w);
    return NSD_OK;
}

nsd_status nsd_route(int32_t ntok, const nsd_router *s, const void *logits, const uint8_t *skip,
                     float weight, int32_t *colind, float *gate, int32_t *counts, double *loss,
                     void *ws, size_t ws_bytes, void *stream) {
    NSD_TRY(check_router(ntok, s));
    NSD_REQUIRE(ntok == 0 || (logits && colind && gate), "a NULL array");
    NSD_REQUIRE((counts == nullptr) == (loss == nullptr), "counts and loss go together");
    RouteArgs a = {};
    a.T = ntok;
    a.E = s->experts;
    a.k = s->topk;
    a.norm = s->normalize;
    a.ld = s->ld;
    a.x = logits;
    a.skip = skip;
    a.col = colind;
    a.gate = gate;
    a.weight = weight;
    a.counts = counts;
    a.loss = loss;
    const hipStream_t st = as_stream(stream);
    if (counts == nullptr) {
        if (ntok == 0) return NSD_OK;
        const int64_t per = kPlainThreads / slot_lanes(a.E);
        const unsigned nb = (unsigned)std::min<int64_t>(ceil_div(ntok, per), 1 << 16);
        with_types(s, [&](auto T, auto G, auto NE) {
            route_kernel<decltype(T), G(), NE(), false><<<nb, kPlainThreads, 0, st>>>(a);
        });
        return check_launch("route_kernel");
    }
    RouteWs w;
    const size_t need = carve_route(ws, ntok, a.E, &w);
    if (ws == nullptr || ws_bytes < need)
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, need);
    a.part_p = w.p;
    a.part_n = w.n;
    const int nb = stat_blocks(ntok, a.E);
    with_types(s, [&](auto T, auto G, auto NE) {
        route_kernel<decltype(T), G(), NE(), true><<<nb, stat_threads(NE()), 0, st>>>(a);
    });
    NSD_TRY(check_launch("route_kernel"));
    if (nb > 1) {
        route_total_kernel<<<1, kRouteThreads, 0, st>>>(a, nb);
        return check_launch("route_total_kernel");
    }
    return NSD_OK;
}

nsd_status nsd_route_vjp(int32_t ntok, const nsd_router *s, const void *logits,
                         const uint8_t *skip, const int32_t *colind, const float *gate,
                         const int32_t *counts, float weight, float seed, const float *dgate,
                         void *dlogits, void *stream) {
    NSD_TRY(check_router(ntok, s));
    if (ntok == 0) return NSD_OK;
    NSD_REQUIRE(logits && dlogits, "a NULL array");
    NSD_REQUIRE(dgate == nullptr || (colind && gate), "dgate without the chosen experts");
    VjpArgs a = {};
    a.T = ntok;
    a.E = s->experts;
    a.k = s->topk;
    a.norm = s->normalize;
    a.ld = s->ld;
    a.x = logits;
    a.skip = skip;
    a.col = colind;
    a.gate = gate;
    a.counts = counts;
    a.scale = seed * weight * (float)s->experts;
    a.dgate = dgate;
    a.dx = dlogits;
    const int64_t per = kPlainThreads / slot_lanes(a.E);
    const unsigned nb = (unsigned)std::min<int64_t>(ceil_div(ntok, per), 2048);
    with_types(s, [&](auto T, auto G, auto NE) {
        route_vjp_kernel<decltype(T), G(), NE()><<<nb, kPlainThreads, 0, as_stream(stream)>>>(a);
    });
    return check_launch("route_vjp_kernel");
}

}  // extern "C"
