// Norm and rotation of every head's query and key in one pass, its gradient, and the
// serving form that appends keys and values to a cache.
//
//   n = x r w,  r = 1 / sqrt(mean(x^2) + eps);   y = n turned pair by pair by pos_t freq_p
//   g = dy turned back,  dw = sum g x r,  dx = r (g w - x r mean(g w x r))
//
// HBM-bound: every value is read and written once (the gradient reads x and dy; r is
// found again instead of stored).  A head lies on a slot of G lanes of four pairs each,
// so that a lane's pairs, and their angles, are the same for every head of a token: a
// wave takes one token, its lanes find the token's sines and cosines once, pass them
// through LDS to the lanes of those pairs, and walk the token's heads, 64 / G at a
// time.  Angles are products in 64 bits less whole turns: in 32 bits position 10^6
// would be off by a thirtieth of a turn.
//
// The gradient's blocks walk tokens with a stride, hold their share of dw in registers
// and leave one partial each; a second launch adds those up in their order.
//
// 16,384 tokens of 32 and 8 heads of 128 in bf16: 65 us (5.1 TB/s), the gradient 113 (4.5
// TB/s) and 7 for the weights'.  8 tokens of 16 and 4 heads of 64 appended: 4.0 us, a launch.
// 10,007 tokens of 6 and 3 heads of 40, pairs side by side, in fp32: 10.2, 14.8 and 6.0 us.
#include <algorithm>

#include "values.hpp"

namespace nsd {

namespace {

constexpr int kQkThreads = 256;
constexpr int kQkWaves = kQkThreads / kWave;
constexpr int64_t kMaxQkBlocks = UINT32_MAX / kQkThreads;
constexpr int kMaxHead = 512;
constexpr int kPairs = 4;           // of a lane
constexpr int kHeadsAhead = 2;      // heads of a slot in flight
// Blocks of the gradient: four a CU (16,384 tokens of 40 heads of 128: 512 blocks 162 us, 1,024
// 107, 2,048 115).
constexpr int kMaxGradBlocks = 1024;

struct QkArgs {
    int32_t ntok, H, Hk, d, rot, pairs;  // pairs: those of a head, rotated or not
    int32_t parts;                       // waves that share a token's heads
    bool interleaved, norm;
    float eps;
    int64_t ldq, ldk, ldqo, ldko;
    const void *Q, *K;
    const float *wq, *wk;
    const int32_t *pos;
    const double *freq;
    void *Qo, *Ko;  // forward: written; gradient: the upstream, read
    // appending
    const int32_t *slot;
    int32_t nslots, vwidth;
    const void *V;
    void *Vo;
    int64_t ldv, ldvo;
    // gradient
    void *dQ, *dK;
    float *part;  // [block][2][d]
};

// How a lane's values lie: anyhow; its a and b four consecutive ones each; a and b in turn,
// eight consecutive ones.
enum Lie { kAnyhow, kHalves, kNext };

// The pairs p0 to p0 + 3 of a head, as a lane holds them: values a and b of pair e.  Values
// that are not rotated pair up as they come.
template <class T, Lie LIE>
struct Head {
    float a[kPairs], b[kPairs];
    static __device__ __forceinline__ int place_a(const QkArgs &s, int p) {
        return s.interleaved ? 2 * p : p < s.rot / 2 ? p : s.rot + 2 * (p - s.rot / 2);
    }
    static __device__ __forceinline__ int place_b(const QkArgs &s, int p) {
        return s.interleaved ? 2 * p + 1 : p < s.rot / 2 ? p + s.rot / 2 : place_a(s, p) + 1;
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) a[e] = b[e] = 0.f;
    }
    __device__ __forceinline__ void load(const QkArgs &s, const T *x, int p0) {
        if constexpr (LIE == kNext) {
            float t[2 * kPairs];
            load_values<2 * kPairs, T>(x + 2 * p0, t);
#pragma unroll
            for (int e = 0; e < kPairs; ++e) a[e] = t[2 * e], b[e] = t[2 * e + 1];
        } else if constexpr (LIE == kHalves) {
            const int at = place_a(s, p0);
            load_values<kPairs, T>(x + at, a);
            load_values<kPairs, T>(x + (p0 < s.rot / 2 ? at + s.rot / 2 : at + kPairs), b);
        } else {
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
                const int p = p0 + e, ia = place_a(s, p), ib = place_b(s, p);
                a[e] = p < s.pairs && ia < s.d ? widened(x[ia]) : 0.f;
                b[e] = p < s.pairs && ib < s.d ? widened(x[ib]) : 0.f;
            }
        }
    }
    __device__ __forceinline__ void store(const QkArgs &s, T *x, int p0) const {
        if constexpr (LIE == kNext) {
            float t[2 * kPairs];
#pragma unroll
            for (int e = 0; e < kPairs; ++e) t[2 * e] = a[e], t[2 * e + 1] = b[e];
            store_row_values<2 * kPairs, T>(x + 2 * p0, t);
        } else if constexpr (LIE == kHalves) {
            const int at = place_a(s, p0);
            store_row_values<kPairs, T>(x + at, a);
            store_row_values<kPairs, T>(x + (p0 < s.rot / 2 ? at + s.rot / 2 : at + kPairs), b);
        } else {
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
                const int p = p0 + e, ia = place_a(s, p), ib = place_b(s, p);
                if (p < s.pairs && ia < s.d) x[ia] = narrowed<T>(a[e]);
                if (p < s.pairs && ib < s.d) x[ib] = narrowed<T>(b[e]);
            }
        }
    }
    __device__ __forceinline__ float dot(const Head &o) const {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            t = __builtin_fmaf(a[e], o.a[e], t);
            t = __builtin_fmaf(b[e], o.b[e], t);
        }
        return t;
    }
    // The first n pairs turned by the lane's angles, or back.  (The others are no pairs: an
    // infinite one times a sine of 0 would take the number beside it away.)
    __device__ __forceinline__ void turn(const float (&c)[kPairs], const float (&s)[kPairs], int n,
                                         bool back) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const float sn = back ? -s[e] : s[e], x = a[e], y = b[e];
            a[e] = e < n ? x * c[e] - y * sn : x;
            b[e] = e < n ? x * sn + y * c[e] : y;
        }
    }
};

// A lane's view of the weights of a head.
template <Lie LIE>
__device__ __forceinline__ void load_weights(const QkArgs &s, const float *w, int p0, bool on,
                                             Head<float, LIE> &h) {
#pragma unroll
    for (int e = 0; e < kPairs; ++e) h.a[e] = h.b[e] = 1.f;
    if (w != nullptr && s.norm && on) h.load(s, w, p0);
}

// Sum over the aligned group of G lanes.
template <int G>
__device__ __forceinline__ float over_slot(float v) {
    if constexpr (G > 1) v += lane_xor<1>(v);
    if constexpr (G > 2) v += lane_xor<2>(v);
    if constexpr (G > 4) v += lane_xor<4>(v);
    if constexpr (G > 8) v += lane_xor<8>(v);
    if constexpr (G > 16) v += lane_xor<16>(v);
    if constexpr (G > 32) v += lane_xor<32>(v);
    return v;
}

// Cosines and sines of a token's angles for this lane's pairs, found once a wave.
template <int G>
struct Angles {
    float c[kPairs], s[kPairs];
    __device__ __forceinline__ void find(const QkArgs &q, float2 (&lds)[G * kPairs], int pos, int lane,
                                         int p0) {
        const int half = q.rot / 2;
        // what the last token's lanes still read is read before it is overwritten
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int p = lane; p < G * kPairs; p += kWave) {
            float2 v = make_float2(1.f, 0.f);
            if (p < half) {
                const double angle = (double)pos * q.freq[p];
                constexpr double kTurn = 6.283185307179586476925;
                const double rest = __builtin_fma(-rint(angle * (1.0 / kTurn)), kTurn, angle);
                sincosf((float)rest, &v.y, &v.x);
            }
            lds[p] = v;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const float2 v = lds[p0 + e];
            c[e] = v.x;
            s[e] = v.y;
        }
    }
};

template <class T>
__device__ __forceinline__ void copy_row(const T *__restrict__ from, T *__restrict__ to, int n, int lane) {
    constexpr int N = 16 / sizeof(T);
    for (int c = lane * N; c < n; c += kWave * N) {
        if (n - c >= N) {
            T t[N];
            __builtin_memcpy(t, from + c, sizeof t);
            __builtin_memcpy(to + c, t, sizeof t);
        } else {
            for (int e = 0; e < n - c; ++e) to[c + e] = from[c + e];
        }
    }
}

// Unit u: part u % parts of token u / parts.  Heads 0 to H - 1 are queries, the others keys.
template <class T, int G, Lie LIE>
__global__ __launch_bounds__(kQkThreads) void qk_rotate_kernel(QkArgs s, int64_t units) {
    __shared__ float2 lds[kQkWaves][G * kPairs];
    constexpr int SLOTS = kWave / G;
    const int lane = threadIdx.x % kWave, slot = lane / G, p0 = lane % G * kPairs;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const bool on = p0 < s.pairs;
    Head<float, LIE> wq, wk;
    load_weights<LIE>(s, s.wq, p0, on, wq);
    load_weights<LIE>(s, s.wk, p0, on, wk);
    const float mean = 1.f / (float)s.d;
    for (int64_t u = (int64_t)blockIdx.x * kQkWaves + wave; u < units;
         u += (int64_t)gridDim.x * kQkWaves) {
        const int64_t t = u / s.parts;
        const int part = (int)(u % s.parts);
        int64_t krow = t;
        if (s.slot != nullptr) {
            krow = s.slot[t];
            if (krow < 0 || krow >= s.nslots) krow = -1;
            if (part == 0 && krow >= 0 && s.vwidth > 0)
                copy_row(static_cast<const T *>(s.V) + t * s.ldv,
                         static_cast<T *>(s.Vo) + krow * s.ldvo, s.vwidth, lane);
        }
        Angles<G> angle;
        angle.find(s, lds[wave], s.pos ? s.pos[t] : 0, lane, p0);
        const int heads = s.H + s.Hk;
        for (int h0 = part * SLOTS * kHeadsAhead; h0 < heads; h0 += s.parts * SLOTS * kHeadsAhead) {
            Head<T, LIE> x[kHeadsAhead];
#pragma unroll
            for (int i = 0; i < kHeadsAhead; ++i) {
                const int h = h0 + i * SLOTS + slot;
                x[i].zero();
                if (on && h < heads)
                    x[i].load(s, h < s.H ? static_cast<const T *>(s.Q) + t * s.ldq + (int64_t)h * s.d
                                         : static_cast<const T *>(s.K) + t * s.ldk +
                                               (int64_t)(h - s.H) * s.d, p0);
            }
#pragma unroll
            for (int i = 0; i < kHeadsAhead; ++i) {
                const int h = h0 + i * SLOTS + slot;
                if (s.norm) {
                    const float ss = over_slot<G>(x[i].dot(x[i]));
                    const float r = 1.f / sqrtf(__builtin_fmaf(ss, mean, s.eps));
#pragma unroll
                    for (int e = 0; e < kPairs; ++e) {
                        x[i].a[e] = x[i].a[e] * r * (h < s.H ? wq.a[e] : wk.a[e]);
                        x[i].b[e] = x[i].b[e] * r * (h < s.H ? wq.b[e] : wk.b[e]);
                    }
                }
                x[i].turn(angle.c, angle.s, s.rot / 2 - p0, false);
                if (on && h < s.H)
                    x[i].store(s, static_cast<T *>(s.Qo) + t * s.ldqo + (int64_t)h * s.d, p0);
                else if (on && h < heads && krow >= 0)
                    x[i].store(s, static_cast<T *>(s.Ko) + krow * s.ldko + (int64_t)(h - s.H) * s.d, p0);
            }
        }
    }
}

// Tokens by a wave, in order with a stride: dQ, dK, and the block's share of dw.
template <class T, int G, Lie LIE>
__global__ __launch_bounds__(kQkThreads) void qk_rotate_vjp_kernel(QkArgs s, int64_t units) {
    __shared__ float2 lds[kQkWaves][G * kPairs];
    __shared__ float sum[kQkWaves][2][2 * G * kPairs];
    constexpr int SLOTS = kWave / G;
    const int lane = threadIdx.x % kWave, slot = lane / G, p0 = lane % G * kPairs;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const bool on = p0 < s.pairs;
    Head<float, LIE> wq, wk, gw[2];
    load_weights<LIE>(s, s.wq, p0, on, wq);
    load_weights<LIE>(s, s.wk, p0, on, wk);
    gw[0].zero();
    gw[1].zero();
    const float mean = 1.f / (float)s.d;
    for (int64_t u = (int64_t)blockIdx.x * kQkWaves + wave; u < units;
         u += (int64_t)gridDim.x * kQkWaves) {
        const int64_t t = u / s.parts;
        const int part = (int)(u % s.parts);
        Angles<G> angle;
        angle.find(s, lds[wave], s.pos ? s.pos[t] : 0, lane, p0);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const int heads = side ? s.Hk : s.H;
            const T *x0 = side ? static_cast<const T *>(s.K) + t * s.ldk
                               : static_cast<const T *>(s.Q) + t * s.ldq;
            const T *y0 = side ? static_cast<const T *>(s.Ko) + t * s.ldko
                               : static_cast<const T *>(s.Qo) + t * s.ldqo;
            T *g0 = side ? static_cast<T *>(s.dK) + t * s.ldk : static_cast<T *>(s.dQ) + t * s.ldq;
            const Head<float, LIE> &w = side ? wk : wq;
            for (int h0 = part * SLOTS * kHeadsAhead; h0 < heads;
                 h0 += s.parts * SLOTS * kHeadsAhead) {
                Head<T, LIE> x[kHeadsAhead], y[kHeadsAhead];
#pragma unroll
                for (int i = 0; i < kHeadsAhead; ++i) {
                    const int h = h0 + i * SLOTS + slot;
                    x[i].zero();
                    y[i].zero();
                    if (on && h < heads) {
                        if (s.norm) x[i].load(s, x0 + (int64_t)h * s.d, p0);
                        y[i].load(s, y0 + (int64_t)h * s.d, p0);
                    }
                }
#pragma unroll
                for (int i = 0; i < kHeadsAhead; ++i) {
                    const int h = h0 + i * SLOTS + slot;
                    y[i].turn(angle.c, angle.s, s.rot / 2 - p0, true);
                    if (s.norm) {
                        const float ss = over_slot<G>(x[i].dot(x[i]));
                        // (a slot without a head: nothing of it, also where eps is 0)
                        const float r = h < heads ? 1.f / sqrtf(__builtin_fmaf(ss, mean, s.eps)) : 0.f;
#pragma unroll
                        for (int e = 0; e < kPairs; ++e) {
                            x[i].a[e] *= r;
                            x[i].b[e] *= r;
                            gw[side].a[e] = __builtin_fmaf(y[i].a[e], x[i].a[e], gw[side].a[e]);
                            gw[side].b[e] = __builtin_fmaf(y[i].b[e], x[i].b[e], gw[side].b[e]);
                            y[i].a[e] *= w.a[e];
                            y[i].b[e] *= w.b[e];
                        }
                        const float along = over_slot<G>(x[i].dot(y[i])) * mean;
#pragma unroll
                        for (int e = 0; e < kPairs; ++e) {
                            y[i].a[e] = r * __builtin_fmaf(-along, x[i].a[e], y[i].a[e]);
                            y[i].b[e] = r * __builtin_fmaf(-along, x[i].b[e], y[i].b[e]);
                        }
                    }
                    if (on && h < heads) y[i].store(s, g0 + (int64_t)h * s.d, p0);
                }
            }
        }
    }
    if (s.part == nullptr) return;
    // the wave's slots, then the block's waves, in their order
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int e = 0; e < kPairs; ++e)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                float v = z ? gw[side].b[e] : gw[side].a[e];
#pragma unroll
                for (int m = G; m < kWave; m <<= 1) v += __shfl_xor(v, m, kWave);
                if (slot == 0) sum[wave][side][(p0 + e) * 2 + z] = v;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * 2 * G * kPairs; i += kQkThreads) {
        const int side = i / (2 * G * kPairs), j = i % (2 * G * kPairs), p = j / 2;
        if (p >= s.pairs) continue;
        int at;
        if (LIE == kHalves && p >= s.rot / 2) {  // as Head::load pairs them
            const int q = p / kPairs * kPairs;
            at = Head<T, LIE>::place_a(s, q) + p % kPairs + (j % 2) * kPairs;
        } else {
            at = j % 2 ? Head<T, LIE>::place_b(s, p) : Head<T, LIE>::place_a(s, p);
        }
        if (at >= s.d) continue;
        float v = 0.f;
        for (int w = 0; w < kQkWaves; ++w) v += sum[w][side][j];
        s.part[((int64_t)blockIdx.x * 2 + side) * s.d + at] = v;
    }
}

// dw from the blocks' partials: 16 columns a block, 64 threads for each.
constexpr int kWeightThreads = 1024, kWeightCols = 16;
__global__ __launch_bounds__(kWeightThreads) void qk_weights_kernel(const float *__restrict__ part,
                                                                    int blocks, int d, float *dwq,
                                                                    float *dwk) {
    constexpr int ROWS = kWeightThreads / kWeightCols;
    __shared__ float sum[ROWS][kWeightCols];
    const int row = threadIdx.x / kWeightCols, c = threadIdx.x % kWeightCols;
    const int col = blockIdx.x * kWeightCols + c;  // of [2][d]
    float v = 0.f;
    if (col < 2 * d)
        for (int b = row; b < blocks; b += ROWS) v += part[(int64_t)b * 2 * d + col];
    sum[row][c] = v;
    __syncthreads();
    for (int m = ROWS / 2; m > 0; m /= 2) {
        if (row < m) sum[row][c] += sum[row + m][c];
        __syncthreads();
    }
    if (row > 0 || col >= 2 * d) return;
    float *to = col < d ? dwq : dwk;
    if (to != nullptr) to[col < d ? col : col - d] = sum[0][c];
}

// ------------------------------------------------------------------- host

nsd_status check_qk(int32_t ntok, const nsd_qk *s) {
    NSD_REQUIRE(s != nullptr, "descriptor is NULL");
    NSD_REQUIRE(ntok >= 0, "negative number of tokens");
    NSD_REQUIRE(s->heads >= 0 && s->kv_heads >= 0 && s->d >= 1, "%d and %d heads of %d", s->heads,
                s->kv_heads, s->d);
    NSD_REQUIRE(s->rot >= 0 && s->rot <= s->d && s->rot % 2 == 0, "%d of %d values rotated", s->rot,
                s->d);
    NSD_REQUIRE(known_dtype(s->dtype), "unknown type %d", s->dtype);
    NSD_REQUIRE(s->eps >= 0.f, "eps %g below 0", s->eps);
    if (s->d > kMaxHead) return fail(NSD_ERR_UNSUPPORTED, "heads of %d values (up to %d)", s->d, kMaxHead);
    if (s->heads > 65536 || s->kv_heads > 65536)
        return fail(NSD_ERR_TOO_LARGE, "%d and %d heads", s->heads, s->kv_heads);
    NSD_REQUIRE(s->ldq >= (int64_t)s->heads * s->d && s->ldqo >= (int64_t)s->heads * s->d &&
                    s->ldk >= (int64_t)s->kv_heads * s->d && s->ldko >= (int64_t)s->kv_heads * s->d,
                "row distances below the heads' widths");
    return NSD_OK;
}

QkArgs qk_args(int32_t ntok, const nsd_qk *s, const void *Q, const void *K, const float *wq,
               const float *wk, const int32_t *pos, const double *freq) {
    QkArgs a{};
    a.ntok = ntok;
    a.H = s->heads;
    a.Hk = s->kv_heads;
    a.d = s->d;
    a.rot = s->rot;
    a.pairs = (s->d + 1) / 2;
    a.interleaved = s->interleaved != 0;
    a.norm = s->norm != 0;
    a.eps = s->eps;
    a.ldq = s->ldq;
    a.ldk = s->ldk;
    a.ldqo = s->ldqo;
    a.ldko = s->ldko;
    a.Q = Q;
    a.K = K;
    a.wq = wq;
    a.wk = wk;
    a.pos = pos;
    a.freq = freq;
    return a;
}

// Lanes of a head, and whether every lane's values are consecutive ones.
int slot_lanes(int d) {
    int g = 1;
    while (g * kPairs * 2 < d) g <<= 1;
    return g;
}
Lie lie_of(const nsd_qk *s) {
    if (s->d % (2 * kPairs) != 0 || (!s->interleaved && s->rot / 2 % kPairs != 0)) return kAnyhow;
    return s->interleaved ? kNext : kHalves;
}

// Waves for a token: one, but where that leaves the card without work the heads are shared
// by as many as there are rounds of heads (8 tokens of 20 heads of 64: 4.2 us, by one wave 4.9;
// 4,096 of 40 heads of 128: by one 17.2, by two 18.3).
int head_parts(int32_t ntok, const nsd_qk *s, int heads) {
    const int round = kWave / slot_lanes(s->d) * kHeadsAhead;
    const int rounds = (int)ceil_div(std::max(heads, 1), round);
    constexpr int64_t kEnough = 4096;
    return (int)std::max<int64_t>(1, std::min<int64_t>(rounds, kEnough / std::max(ntok, 1)));
}

template <class F>
nsd_status by_head(const nsd_qk *s, F f) {
    auto shape = [&](auto t) -> nsd_status {
        auto lanes = [&](auto g) -> nsd_status {
            switch (lie_of(s)) {
                case kHalves: return f(t, g, std::integral_constant<Lie, kHalves>());
                case kNext: return f(t, g, std::integral_constant<Lie, kNext>());
                default: return f(t, g, std::integral_constant<Lie, kAnyhow>());
            }
        };
        switch (slot_lanes(s->d)) {
            case 1: return lanes(std::integral_constant<int, 1>());
            case 2: return lanes(std::integral_constant<int, 2>());
            case 4: return lanes(std::integral_constant<int, 4>());
            case 8: return lanes(std::integral_constant<int, 8>());
            case 16: return lanes(std::integral_constant<int, 16>());
            case 32: return lanes(std::integral_constant<int, 32>());
            default: return lanes(std::integral_constant<int, 64>());
        }
    };
    return s->dtype == NSD_F32 ? shape(float()) : shape(Bf16());
}

nsd_status launch_rotate(const nsd_qk *s, QkArgs a, hipStream_t st) {
    a.parts = head_parts(a.ntok, s, a.H + a.Hk);
    const int64_t units = (int64_t)a.ntok * a.parts;
    const int64_t blocks = std::min(ceil_div(units, kQkWaves), kMaxQkBlocks);
    return by_head(s, [&](auto t, auto g, auto lie) -> nsd_status {
        qk_rotate_kernel<decltype(t), decltype(g)::value, decltype(lie)::value>
            <<<blocks, kQkThreads, 0, st>>>(a, units);
        return check_launch("qk_rotate_kernel");
    });
}

int64_t grad_units(int32_t ntok, const nsd_qk *s) {
    return (int64_t)ntok * head_parts(ntok, s, std::max(s->heads, s->kv_heads));
}
int64_t grad_blocks(int32_t ntok, const nsd_qk *s) {
    return std::min<int64_t>(ceil_div(grad_units(ntok, s), kQkWaves), kMaxGradBlocks);
}

nsd_status check_heads(const nsd_qk *s, const void *Q, const void *K, const int32_t *pos,
                       const double *freq) {
    NSD_REQUIRE((Q || s->heads == 0) && (K || s->kv_heads == 0), "Q or K is NULL");
    NSD_REQUIRE(s->rot == 0 || (pos && freq), "positions or frequencies are NULL");
    return NSD_OK;
}

// A call's arrays; of queries (1) and keys (2) those that a call may take in place have one number.
struct Areas {
    int64_t n;  // tokens
    const nsd_qk *s;
    Area q(const void *p, int64_t ld) const { return row_area(p, n, (int64_t)s->heads * s->d, ld, s->dtype, 1); }
    Area k(const void *p, int64_t ld) const { return row_area(p, n, (int64_t)s->kv_heads * s->d, ld, s->dtype, 2); }
    Area weights(const float *p) const { return flat_area(s->norm ? p : nullptr, 4 * (int64_t)s->d); }
    Area pos(const int32_t *p) const { return flat_area(s->rot ? p : nullptr, 4 * n); }
    Area freq(const double *p) const { return flat_area(p, 4 * (int64_t)s->rot); }
};

}  // namespace

}  // namespace nsd

using namespace nsd;

extern "C" {

nsd_status nsd_qk_rotate(int32_t ntok, const nsd_qk *s, const void *Q, const void *K,
                         const float *wq, const float *wk, const int32_t *pos,
                         const double *freq, void *Qo, void *Ko, void *stream) {
    NSD_TRY(check_qk(ntok, s));
    if (ntok == 0 || s->heads + s->kv_heads == 0) return NSD_OK;
    NSD_TRY(check_heads(s, Q, K, pos, freq));
    NSD_REQUIRE((Qo || s->heads == 0) && (Ko || s->kv_heads == 0), "Qo or Ko is NULL");
    NSD_REQUIRE((Qo != Q || s->ldqo == s->ldq) && (Ko != K || s->ldko == s->ldk || s->kv_heads == 0),
                "in place with another row distance");
    const Areas of{ntok, s};
    NSD_TRY(check_apart({of.q(Qo, s->ldqo), of.k(Ko, s->ldko)},
                        {of.q(Q, s->ldq), of.k(K, s->ldk), of.weights(wq), of.weights(wk), of.pos(pos),
                         of.freq(freq)}));
    QkArgs a = qk_args(ntok, s, Q, K, wq, wk, pos, freq);
    a.Qo = Qo;
    a.Ko = Ko;
    return launch_rotate(s, a, as_stream(stream));
}

nsd_status nsd_qk_rotate_vjp_workspace_size(int32_t ntok, const nsd_qk *s, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_TRY(check_qk(ntok, s));
    Carver c(nullptr);
    // (as many as any smaller batch takes: fewer tokens have their heads shared by more waves)
    c.take<float>((size_t)kMaxGradBlocks * 2 * s->d);
    *bytes = std::max<size_t>(c.bytes(), 256);
    return NSD_OK;
}

nsd_status nsd_qk_rotate_vjp(int32_t ntok, const nsd_qk *s, const void *Q, const void *K,
                             const float *wq, const float *wk, const int32_t *pos,
                             const double *freq, const void *dQo, const void *dKo, void *dQ,
                             void *dK, float *dwq, float *dwk, void *ws, size_t ws_bytes,
                             void *stream) {
    NSD_TRY(check_qk(ntok, s));
    const bool weights = dwq != nullptr || dwk != nullptr;
    const bool any = ntok > 0 && s->heads + s->kv_heads > 0;
    if (!any && !weights) return NSD_OK;
    NSD_REQUIRE(!weights || s->norm, "gradients of weights without a norm");
    if (any) {
        NSD_TRY(check_heads(s, Q, K, pos, freq));
        NSD_REQUIRE((dQo || s->heads == 0) && (dKo || s->kv_heads == 0), "dQo or dKo is NULL");
        NSD_REQUIRE((dQ || s->heads == 0) && (dK || s->kv_heads == 0), "dQ or dK is NULL");
        NSD_REQUIRE((dQ != dQo || s->ldqo == s->ldq || s->heads == 0) &&
                        (dK != dKo || s->ldko == s->ldk || s->kv_heads == 0),
                    "in place with another row distance");
    }
    const hipStream_t st = as_stream(stream);
    QkArgs a = qk_args(ntok, s, Q, K, wq, wk, pos, freq);
    a.Qo = const_cast<void *>(dQo);
    a.Ko = const_cast<void *>(dKo);
    a.dQ = dQ;
    a.dK = dK;
    size_t need = 0;
    if (weights) {
        NSD_TRY(nsd_qk_rotate_vjp_workspace_size(ntok, s, &need));
        if (ws == nullptr || ws_bytes < need)
            return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, need);
        NSD_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255) == 0,
                    "workspace is not 256-byte aligned");
        a.part = static_cast<float *>(ws);
    }
    const Areas of{any ? ntok : 0, s};
    NSD_TRY(check_apart({of.q(dQ, s->ldq), of.k(dK, s->ldk), of.weights(dwq), of.weights(dwk),
                         flat_area(a.part, (int64_t)need)},
                        {of.q(Q, s->ldq), of.k(K, s->ldk), of.q(dQo, s->ldqo), of.k(dKo, s->ldko),
                         of.weights(any ? wq : nullptr), of.weights(any ? wk : nullptr), of.pos(pos),
                         of.freq(any ? freq : nullptr)}));
    int64_t blocks = 0;
    if (any) {
        a.parts = head_parts(ntok, s, std::max(s->heads, s->kv_heads));
        blocks = grad_blocks(ntok, s);
        NSD_TRY(by_head(s, [&](auto t, auto g, auto lie) -> nsd_status {
            qk_rotate_vjp_kernel<decltype(t), decltype(g)::value, decltype(lie)::value>
                <<<blocks, kQkThreads, 0, st>>>(a, grad_units(ntok, s));
            return check_launch("qk_rotate_vjp_kernel");
        }));
    }
    if (!weights) return NSD_OK;
    qk_weights_kernel<<<ceil_div(2 * s->d, kWeightCols), kWeightThreads, 0, st>>>(
        a.part, (int)blocks, s->d, dwq, dwk);
    return check_launch("qk_weights_kernel");
}

nsd_status nsd_qk_append(int32_t ntok, const nsd_qk *s, const void *Q, const void *K,
                         const void *V, int32_t vwidth, int64_t ldv, int64_t ldvo,
                         const float *wq, const float *wk, const int32_t *pos,
                         const double *freq, const int32_t *slot, int32_t nslots, void *Qo,
                         void *Kc, void *Vc, void *stream) {
    NSD_TRY(check_qk(ntok, s));
    NSD_REQUIRE(nslots >= 0 && vwidth >= 0, "%d slots, values of %d", nslots, vwidth);
    NSD_REQUIRE(vwidth == 0 || (ldv >= vwidth && ldvo >= vwidth), "row distances below %d", vwidth);
    if (ntok == 0) return NSD_OK;
    NSD_TRY(check_heads(s, Q, K, pos, freq));
    NSD_REQUIRE(slot, "slots are NULL");
    NSD_REQUIRE((Qo || s->heads == 0) && (Kc || s->kv_heads == 0 || nslots == 0), "Qo or Kc is NULL");
    NSD_REQUIRE(vwidth == 0 || (V && (Vc || nslots == 0)), "V or Vc is NULL");
    NSD_REQUIRE((Kc != K || s->kv_heads == 0) && (Vc != V || vwidth == 0), "a cache is what is appended");
    NSD_REQUIRE(Qo != Q || s->ldqo == s->ldq || s->heads == 0, "in place with another row distance");
    const Areas of{ntok, s};
    // (a key that lies in the cache would be overwritten by another token's before it is read)
    Area kc = of.k(Kc, s->ldko);
    kc.rows = nslots;
    kc.same = 0;
    NSD_TRY(check_apart({of.q(Qo, s->ldqo), kc, row_area(Vc, nslots, vwidth, ldvo, s->dtype)},
                        {of.q(Q, s->ldq), of.k(K, s->ldk), row_area(V, ntok, vwidth, ldv, s->dtype),
                         of.weights(wq), of.weights(wk), of.pos(pos), of.freq(freq),
                         flat_area(slot, 4 * (int64_t)ntok)}));
    QkArgs a = qk_args(ntok, s, Q, K, wq, wk, pos, freq);
    a.Qo = Qo;
    a.Ko = Kc;
    a.slot = slot;
    a.nslots = nslots;
    a.V = V;
    a.Vo = Vc;
    a.vwidth = vwidth;
    a.ldv = ldv;
    a.ldvo = ldvo;
    return launch_rotate(s, a, as_stream(stream));
}

}  // extern "C"
