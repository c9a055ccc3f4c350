// Differential attention over the stored keys of a CSR mask: the difference of
// two softmax maps, the second weighted by a learned number per head; its
// gradients; and its form for single tokens.
//
//   s^m_p = scale <q^m_i, k^m_j> + bias_p,   a^m = softmax of s^m over row i
//   O_i   = sum_p (a^1_p - lambda a^2_p) v_j
//   t_p   = <dO_i, v_j>,  D^m_i = sum_p a^m_p t_p
//   ds^1  = a^1 (t - D^1),  ds^2 = -lambda a^2 (t - D^2)
//   dq^m_i = scale sum ds^m k^m_j,  dk^m_j = scale sum ds^m q^m_i,
//   dv_j  = sum (a^1 - lambda a^2) dO_i,  dlambda = -sum_i D^2_i
//
// Bound by the gathers: an entry brings a key and a value of every key head,
// and little is computed with them, on a pattern that promises no tile.  One
// wave walks one work item of the pattern's plan (rows, or a chunk of a long
// row) for a group of heads.  Its lanes are split three ways: G lanes hold a
// key's two halves (one half of the lanes each, 16 bytes a lane) and, all of
// them, its value; `hps` heads lie side by side, as they do in memory; the
// lanes left take different entries.  The lanes of half m reduce and hold map
// m's score, so both maps' softmaxes advance in one instruction.
//
// One pass: the running maximum and sum of both maps and the two weighted sums
// of values are kept per entry slot, rescaled when a maximum grows, and joined
// at the row's end; a chunk of a long row leaves them to a second kernel.  The
// backward pass over rows recomputes the scores, writes a^1, a^2, t of every
// entry and head and forms dq from two sums, of a t k and a k (dq = scale (sum
// a t k - D sum a k)), so that it needs no D beforehand; the pass over columns
// (the CSC) is then a plain weighted gather of q and dO, without a dot product
// or an atomic.
//
// Measured: forward over 4M entries, 8 heads of d = 16, dv = 32 in bf16 750 us (5.5
// TB/s of gathered rows; rows of 512 bytes alone gather at 7.2); a training step of
// 1M entries in 100K rows, 4 heads of d = 8 in fp32 482 us, most of it latency: 10
// entries a row.
#include "attn.hpp"
#include "attn_mfma.hpp"

namespace nsd {

using namespace attn;

namespace {

constexpr int kDeep = 4;       // entries in flight per lane
constexpr int kMinSplit = 64;  // entries of a decode split

// ------------------------------------------------------------ values

// V consecutive values of type T as they lie in memory.
template <class T, int V>
struct Raw {
    static constexpr int W = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[W];
    __device__ __forceinline__ void load(const T *p) {
        w[W - 1] = 0;
        __builtin_memcpy(w, p, V * sizeof(T));
    }
    __device__ __forceinline__ void keep(uint32_t mask) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] &= mask;
    }
    __device__ __forceinline__ void keep(const Raw &mask) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] &= mask.w[i];
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
};

// ------------------------------------------------------------ shapes

// How a wave's lanes are split: g within a head's G lanes, the head, the entry.
template <int G>
struct Lane {
    int g, head, slot, slots;
    __device__ __forceinline__ Lane(int hps_log2) {
        const int lane = threadIdx.x % kWave;
        g = lane % G;
        head = (lane / G) & ((1 << hps_log2) - 1);
        slot = (lane / G) >> hps_log2;
        slots = (kWave / G) >> hps_log2;
    }
};

// The V columns of n that lane g holds: a lane whose columns would cross the
// end steps back to the last V (its first `dup` are the lane before's too).
struct Cols {
    int col, dup;
    bool on;
};
template <int V>
__device__ __forceinline__ Cols columns(int g, int n) {
    Cols c;
    c.col = g * V;
    c.on = c.col < n;
    c.dup = c.on ? max(c.col + V - n, 0) : 0;
    c.col = c.on ? c.col - c.dup : 0;
    return c;
}

// Bits of the columns that are this lane's own.
template <class T, int V>
__device__ __forceinline__ Raw<T, V> own_mask(const Cols &c) {
    Raw<T, V> r;
#pragma unroll
    for (int i = 0; i < Raw<T, V>::W; ++i) {
        if constexpr (sizeof(T) == 4) {
            r.w[i] = c.on && i >= c.dup ? ~0u : 0u;
        } else {
            const uint32_t lo = c.on && 2 * i >= c.dup ? 0xFFFFu : 0u;
            const uint32_t hi = c.on && 2 * i + 1 >= c.dup ? 0xFFFF0000u : 0u;
            r.w[i] = lo | hi;
        }
    }
    return r;
}

template <int N, int M = 1>
__device__ __forceinline__ float sum_lanes(float v) {  // over aligned groups of N
    if constexpr (M < N) return sum_lanes<N, 2 * M>(v + lane_xor<M>(v));
    else return v;
}

// x where it is not the other half's, of lanes that all hold their half's value.
template <int G>
__device__ __forceinline__ float other_half(float x) {
    return lane_xor<G / 2>(x);
}

// ------------------------------------------------------------ forward

// The entries that this lane takes of a batch, and the number of a key it may
// read instead of one that is not there.
struct Batch {
    int c[kDeep];
    float b[kDeep];
};

__device__ __forceinline__ void load_batch(const FwdArgs &a, int64_t p, int64_t last, int slot,
                                           int slots, Batch &x) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
        const int64_t e = min(p + u * slots + slot, last);
        x.c[u] = a.colind[e];
        x.b[u] = a.bias ? a.bias[e] : 0.f;
    }
}

template <class T, int VK, int VV, int G, bool EXACT>
struct FwdLane {
    static constexpr int GH = G / 2;
    const FwdArgs &a;
    Lane<G> L;
    int h, kvh;
    bool hon;
    Cols kc, vc;
    Raw<T, VK> kmask;
    float q[VK], acc1[VV], acc2[VV], m, l;

    __device__ __forceinline__ FwdLane(const FwdArgs &a_, int hb) : a(a_), L(a_.s.hps_log2) {
        h = (hb << a.s.hps_log2) + L.head;
        hon = h < a.s.H;
        h = hon ? h : a.s.H - 1;
        kvh = h / a.s.grp;
        kc = columns<VK>(L.g % GH, a.s.d);
        vc = columns<VV>(L.g, a.s.dv);
        if (!EXACT) kmask = own_mask<T, VK>(kc);
    }
    __device__ __forceinline__ int64_t key_offset() const {
        return (int64_t)kvh * 2 * a.s.d + (L.g / GH) * a.s.d + kc.col;
    }
    __device__ __forceinline__ int64_t value_offset() const {
        return (int64_t)kvh * a.s.dv + vc.col;
    }

    __device__ __forceinline__ void begin(int64_t row) {
        Raw<T, VK> r;
        r.load(static_cast<const T *>(a.Q) + row * a.s.ldq + (int64_t)h * 2 * a.s.d +
               (L.g / GH) * a.s.d + kc.col);
        if (!EXACT) r.keep(kmask);
#pragma unroll
        for (int e = 0; e < VK; ++e) q[e] = r.at(e) * a.s.scale;
#pragma unroll
        for (int e = 0; e < VV; ++e) acc1[e] = acc2[e] = 0.f;
        m = -INFINITY;
        l = 0.f;
    }

    // The entries p + u slots + slot < end.
    __device__ __forceinline__ void batch(int64_t p, int64_t end, const Batch &x) {
        const T *K = static_cast<const T *>(a.K) + key_offset();
        const T *V = static_cast<const T *>(a.V) + value_offset();
        const int64_t first = a.colind[p];
        Raw<T, VK> k[kDeep];
        Raw<T, VV> v[kDeep];
        bool in[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            in[u] = p + u * L.slots + L.slot < end && x.b[u] != -INFINITY;
            const int64_t c = in[u] ? (int64_t)x.c[u] : first;
            k[u].load(K + c * a.s.ldk);
            v[u].load(V + c * a.s.ldv);
        }
        float s[kDeep], top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (!EXACT) k[u].keep(kmask);
            float t = q[0] * k[u].at(0);
#pragma unroll
            for (int e = 1; e < VK; ++e) t = __builtin_fmaf(q[e], k[u].at(e), t);
            t = sum_lanes<GH>(t) + x.b[u];
            s[u] = in[u] ? t : -INFINITY;
            top = fmaxf(top, s[u]);
        }
        if (__any(top > m)) {
            const float mn = fmaxf(m, top);
            const float f = exp_diff(m, finite_max(mn));
            const float o = other_half<G>(f);
            const float f1 = L.g < GH ? f : o, f2 = L.g < GH ? o : f;
            l *= f;
#pragma unroll
            for (int e = 0; e < VV; ++e) {
                acc1[e] *= f1;
                acc2[e] *= f2;
            }
            m = mn;
        }
        const float ms = finite_max(m);
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const float w = exp_diff(s[u], ms);
            const float o = other_half<G>(w);
            const float w1 = L.g < GH ? w : o, w2 = L.g < GH ? o : w;
            l += w;
            v[u].keep(in[u] ? ~0u : 0u);
#pragma unroll
            for (int e = 0; e < VV; ++e) {
                acc1[e] = __builtin_fmaf(w1, v[u].at(e), acc1[e]);
                acc2[e] = __builtin_fmaf(w2, v[u].at(e), acc2[e]);
            }
        }
    }

    // Joins the slots: every lane ends with its columns' whole sums.
    __device__ __forceinline__ void join() {
        const int width = kWave / L.slots;
        float mt = m;
        for (int b = width; b < kWave; b <<= 1) mt = fmaxf(mt, __shfl_xor(mt, b));
        const float f = exp_diff(m, finite_max(mt));
        const float o = other_half<G>(f);
        const float f1 = L.g < GH ? f : o, f2 = L.g < GH ? o : f;
        l *= f;
#pragma unroll
        for (int e = 0; e < VV; ++e) {
            acc1[e] *= f1;
            acc2[e] *= f2;
        }
        m = mt;
        for (int b = width; b < kWave; b <<= 1) {
            l += __shfl_xor(l, b);
#pragma unroll
            for (int e = 0; e < VV; ++e) {
                acc1[e] += __shfl_xor(acc1[e], b);
                acc2[e] += __shfl_xor(acc2[e], b);
            }
        }
    }

    __device__ __forceinline__ void finish(int64_t row) {
        join();
        const float lo = other_half<G>(l);
        const float l1 = L.g < GH ? l : lo, l2 = L.g < GH ? lo : l;
        const float i1 = l1 == 0.f ? 0.f : 1.f / l1;
        const float i2 = l2 == 0.f ? 0.f : a.lambda[h] / l2;
        if (L.slot != 0 || !hon) return;
        if (vc.on) {
            float o[VV];
#pragma unroll
            for (int e = 0; e < VV; ++e) o[e] = acc1[e] * i1 - acc2[e] * i2;
            store_values<T, VV>(static_cast<T *>(a.O) + row * a.s.ldo + (int64_t)h * a.s.dv +
                                    vc.col, o);
        }
        if (a.stat && L.g % GH == 0) {
            float *st = a.stat + (row * a.s.H + h) * 4 + (L.g / GH) * 2;
            st[0] = m;
            st[1] = l;
        }
    }

    __device__ __forceinline__ void partial(int64_t at) {
        join();
        if (L.slot != 0 || !hon) return;
        float *o = a.part + (at * a.s.H + h) * (4 + 2 * a.s.dv);
        if (L.g % GH == 0) {
            o[(L.g / GH) * 2] = m;
            o[(L.g / GH) * 2 + 1] = l;
        }
        if (vc.on) {
            store_values<float, VV>(o + 4 + vc.col, acc1);
            store_values<float, VV>(o + 4 + a.s.dv + vc.col, acc2);
        }
    }
};

template <class T, int VK, int VV, int G, bool EXACT, bool DECODE>
__global__ __launch_bounds__(kAttnThreads) void attn_fwd_kernel(FwdArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (!DECODE && (int64_t)blockIdx.x >= a.nmain) {
        for_empty(a.plan, a.nrows, a.all_empty, a.nmain,
                  [&](int64_t row) { empty_row<T>(a, row); });
        return;
    }
    const int64_t unit = near_block(blockIdx.x, (int)a.nmain) * kAttnWaves + wave;
    const int64_t item = unit / a.s.nhb;
    const int hb = (int)(unit - item * a.s.nhb);
    FwdLane<T, VK, VV, G, EXACT> f(a, hb);
    const int step = f.L.slots * kDeep;
    if constexpr (DECODE) {
        if (item >= (int64_t)a.nrows * a.nsplit) return;
        const int64_t row = item / a.nsplit, j = item - row * a.nsplit;
        const int64_t r0 = a.rowptr[row], r1 = a.colind ? a.rowptr[row + 1] : r0;
        int64_t p = min(r0 + j * a.per, r1);
        const int64_t end = j + 1 == a.nsplit ? r1 : min(p + a.per, r1);
        f.begin(row);
        Batch x, y;
        if (p < end) load_batch(a, p, end - 1, f.L.slot, f.L.slots, x);
        for (; p < end; p += step) {
            if (p + step < end) load_batch(a, p + step, end - 1, f.L.slot, f.L.slots, y);
            f.batch(p, end, x);
            x = y;
        }
        if (a.nsplit == 1) f.finish(row);
        else f.partial(item);
    } else {
        if (item >= a.plan.nitems) return;
        int64_t p = a.plan.item_ptr[item];
        const int64_t b0 = a.plan.item_ptr[item + 1];
        const int chunk = a.plan.nchunks > 0 ? a.plan.chunk_ord[item] : -1;
        Batch x, y;
        load_batch(a, p, b0 - 1, f.L.slot, f.L.slots, x);
        while (p < b0) {
            const int64_t row = a.rowidx[p];
            const int64_t end = min((int64_t)a.rowptr[row + 1], b0);
            f.begin(row);
            while (p < end) {
                const int64_t next = min(p + step, end);
                if (next < b0) load_batch(a, next, b0 - 1, f.L.slot, f.L.slots, y);
                f.batch(p, end, x);
                x = y;
                p = next;
            }
            if (chunk >= 0) f.partial(chunk);
            else f.finish(row);
        }
    }
}

// Joins the partials of a long row (or of a decode row's splits): one block for
// a row and head.
struct JoinArgs {
    Shape s;
    const float *part;
    const float *lambda;
    void *O;
    float *stat;
    const int32_t *rowptr;
    nsd_plan plan;
    int32_t nsplit;  // decode (> 0)
};

__device__ __forceinline__ float block_max(float v, float *sh) {
    for (int b = 1; b < kWave; b <<= 1) v = fmaxf(v, __shfl_xor(v, b));
    if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = v;
    __syncthreads();
    v = sh[0];
    for (int w = 1; w < kAttnWaves; ++w) v = fmaxf(v, sh[w]);
    __syncthreads();
    return v;
}
__device__ __forceinline__ float block_sum(float v, float *sh) {
    for (int b = 1; b < kWave; b <<= 1) v += __shfl_xor(v, b);
    if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = v;
    __syncthreads();
    v = sh[0];
    for (int w = 1; w < kAttnWaves; ++w) v += sh[w];
    __syncthreads();
    return v;
}

template <class T>
__global__ __launch_bounds__(kAttnThreads) void attn_join_kernel(JoinArgs a) {
    __shared__ float sh[kAttnWaves], wt[2][kAttnThreads], acc[2 * kMaxDv];
    const int t = threadIdx.x, dv = a.s.dv, W = 2 * dv;
    const int h = blockIdx.x % a.s.H;
    int64_t row, first, n;
    long_segment(a.plan, a.rowptr, a.nsplit, blockIdx.x / a.s.H, row, first, n);
    const int64_t ld = (int64_t)a.s.H * (4 + W);
    const float *base = a.part + first * ld + (int64_t)h * (4 + W);
    float m1 = -INFINITY, m2 = -INFINITY;
    for (int64_t j = t; j < n; j += kAttnThreads) {
        m1 = fmaxf(m1, base[j * ld]);
        m2 = fmaxf(m2, base[j * ld + 2]);
    }
    m1 = block_max(m1, sh);
    m2 = block_max(m2, sh);
    const float s1 = finite_max(m1), s2 = finite_max(m2);
    float l1 = 0.f, l2 = 0.f, x0 = 0.f, x1 = 0.f;  // columns t and t + 256
    for (int64_t j0 = 0; j0 < n; j0 += kAttnThreads) {
        const int64_t j = j0 + t;
        float w1 = 0.f, w2 = 0.f;
        if (j < n) {
            w1 = exp_diff(base[j * ld], s1);
            w2 = exp_diff(base[j * ld + 2], s2);
            l1 += w1 * base[j * ld + 1];
            l2 += w2 * base[j * ld + 3];
        }
        __syncthreads();
        wt[0][t] = w1;
        wt[1][t] = w2;
        __syncthreads();
        const int c = (int)min(n - j0, (int64_t)kAttnThreads);
        const float *p = base + j0 * ld + 4;
        if (t < W) {
            const float *w = wt[t >= dv];
#pragma unroll 8
            for (int i = 0; i < c; ++i) x0 = __builtin_fmaf(w[i], p[i * ld + t], x0);
        }
        if (t + kAttnThreads < W) {
            const float *w = wt[t + kAttnThreads >= dv];
#pragma unroll 8
            for (int i = 0; i < c; ++i) x1 = __builtin_fmaf(w[i], p[i * ld + t + kAttnThreads], x1);
        }
    }
    l1 = block_sum(l1, sh);
    l2 = block_sum(l2, sh);
    if (t < W) acc[t] = x0;
    if (t + kAttnThreads < W) acc[t + kAttnThreads] = x1;
    __syncthreads();
    const float i1 = l1 == 0.f ? 0.f : 1.f / l1;
    const float i2 = l2 == 0.f ? 0.f : a.lambda[h] / l2;
    if (t < dv)
        static_cast<T *>(a.O)[row * a.s.ldo + (int64_t)h * dv + t] =
            narrow<T>(acc[t] * i1 - acc[dv + t] * i2);
    if (a.stat && t < 4)
        a.stat[(row * a.s.H + h) * 4 + t] = t == 0 ? m1 : t == 1 ? l1 : t == 2 ? m2 : l2;
}

// ------------------------------------------------------------ backward, rows

template <class T, int VK, int VV, int G>
struct RowLane {
    static constexpr int GH = G / 2;
    const BwdArgs &a;
    Lane<G> L;
    int h, kvh;
    bool hon;
    Cols kc, vc;
    float q[VK], go[VV], A[VK], B[VK], D, m, inv;

    __device__ __forceinline__ RowLane(const BwdArgs &a_, int hb) : a(a_), L(a_.s.hps_log2) {
        h = (hb << a.s.hps_log2) + L.head;
        hon = h < a.s.H;
        h = hon ? h : a.s.H - 1;
        kvh = h / a.s.grp;
        kc = columns<VK>(L.g % GH, a.s.d);
        vc = columns<VV>(L.g, a.s.dv);
    }
    __device__ __forceinline__ int64_t query_offset(int64_t row) const {
        return row * a.s.ldq + (int64_t)h * 2 * a.s.d + (L.g / GH) * a.s.d + kc.col;
    }

    __device__ __forceinline__ void begin(int64_t row) {
        Raw<T, VK> r;
        r.load(static_cast<const T *>(a.Q) + query_offset(row));
        Raw<T, VV> o;
        o.load(static_cast<const T *>(a.dO) + row * a.s.ldo + (int64_t)h * a.s.dv + vc.col);
        r.keep(own_mask<T, VK>(kc));  // each column once in the dot products
        o.keep(own_mask<T, VV>(vc));
#pragma unroll
        for (int e = 0; e < VK; ++e) {
            q[e] = r.at(e) * a.s.scale;
            A[e] = B[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < VV; ++e) go[e] = o.at(e);
        D = 0.f;
        const float *st = a.stat + (row * a.s.H + h) * 4 + (L.g / GH) * 2;
        m = finite_max(st[0]);
        inv = st[1] == 0.f ? 0.f : 1.f / st[1];
    }

    __device__ __forceinline__ void batch(int64_t p, int64_t end, const Batch &x) {
        const T *K = static_cast<const T *>(a.K) + (int64_t)kvh * 2 * a.s.d +
                     (L.g / GH) * a.s.d + kc.col;
        const T *V = static_cast<const T *>(a.V) + (int64_t)kvh * a.s.dv + vc.col;
        const int64_t first = a.other[p];
        Raw<T, VK> k[kDeep];
        Raw<T, VV> v[kDeep];
        bool in[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            in[u] = p + u * L.slots + L.slot < end && x.b[u] != -INFINITY;
            const int64_t c = in[u] ? (int64_t)x.c[u] : first;
            k[u].load(K + c * a.s.ldk);
            v[u].load(V + c * a.s.ldv);
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            k[u].keep(in[u] ? ~0u : 0u);
            v[u].keep(in[u] ? ~0u : 0u);
            float s = q[0] * k[u].at(0);
#pragma unroll
            for (int e = 1; e < VK; ++e) s = __builtin_fmaf(q[e], k[u].at(e), s);
            s = sum_lanes<GH>(s) + x.b[u];
            float t = go[0] * v[u].at(0);
#pragma unroll
            for (int e = 1; e < VV; ++e) t = __builtin_fmaf(go[e], v[u].at(e), t);
            t = sum_lanes<G>(t);
            t = in[u] ? t : 0.f;
            const float w = in[u] ? exp_diff(s, m) * inv : 0.f;
            const float o = other_half<G>(w);
            const int64_t e0 = p + u * L.slots + L.slot;
            if (L.g == 0 && hon && e0 < end) {
                float *co = a.coef + (e0 * a.s.H + h) * 3;
                co[0] = w;
                co[1] = o;
                co[2] = t;
            }
            const float wt = w * t;
            D += wt;
#pragma unroll
            for (int e = 0; e < VK; ++e) {
                A[e] = __builtin_fmaf(wt, k[u].at(e), A[e]);
                B[e] = __builtin_fmaf(w, k[u].at(e), B[e]);
            }
        }
    }

    __device__ __forceinline__ void join() {
        for (int b = kWave / L.slots; b < kWave; b <<= 1) {
            D += __shfl_xor(D, b);
#pragma unroll
            for (int e = 0; e < VK; ++e) {
                A[e] += __shfl_xor(A[e], b);
                B[e] += __shfl_xor(B[e], b);
            }
        }
    }
    // The gradient of half m from its sums.
    __device__ __forceinline__ void finish(int64_t row) {
        join();
        const float f = L.g < GH ? a.s.scale : -a.lambda[h] * a.s.scale;
        if (L.slot != 0 || !hon) return;
        if (L.g % GH == 0) a.D[(row * a.s.H + h) * 2 + L.g / GH] = D;
        if (kc.on) {
            float o[VK];
#pragma unroll
            for (int e = 0; e < VK; ++e) o[e] = f * (A[e] - D * B[e]);
            store_values<T, VK>(static_cast<T *>(a.dQ) + query_offset(row), o);
        }
    }
    __device__ __forceinline__ void partial(int64_t at) {
        join();
        if (L.slot != 0 || !hon) return;
        float *o = a.part + (at * a.s.H + h) * (2 + 4 * a.s.d);
        const int c = (L.g / GH) * a.s.d + kc.col;
        if (L.g % GH == 0) o[L.g / GH] = D;
        if (kc.on) {
            store_values<float, VK>(o + 2 + c, A);
            store_values<float, VK>(o + 2 + 2 * a.s.d + c, B);
        }
    }
};

__device__ __forceinline__ void load_batch(const BwdArgs &a, int64_t p, int64_t last, int slot,
                                           int slots, Batch &x) {
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
        const int64_t e = min(p + u * slots + slot, last);
        x.c[u] = a.other[e];
        x.b[u] = a.bias ? a.bias[e] : 0.f;
    }
}

template <class T, int VK, int VV, int G>
__global__ __launch_bounds__(kAttnThreads) void attn_row_kernel(BwdArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if ((int64_t)blockIdx.x >= a.nmain) {
        for_empty(a.plan, a.nseg, a.all_empty, a.nmain, [&](int64_t row) { empty_row<T>(a, row); });
        return;
    }
    const int64_t unit = near_block(blockIdx.x, (int)a.nmain) * kAttnWaves + wave;
    const int64_t item = unit / a.s.nhb;
    if (item >= a.plan.nitems) return;
    RowLane<T, VK, VV, G> f(a, (int)(unit - item * a.s.nhb));
    const int step = f.L.slots * kDeep;
    int64_t p = a.plan.item_ptr[item];
    const int64_t b0 = a.plan.item_ptr[item + 1];
    const int chunk = a.plan.nchunks > 0 ? a.plan.chunk_ord[item] : -1;
    Batch x, y;
    load_batch(a, p, b0 - 1, f.L.slot, f.L.slots, x);
    while (p < b0) {
        const int64_t row = a.idx[p];
        const int64_t end = min((int64_t)a.ptr[row + 1], b0);
        f.begin(row);
        while (p < end) {
            const int64_t next = min(p + step, end);
            if (next < b0) load_batch(a, next, b0 - 1, f.L.slot, f.L.slots, y);
            f.batch(p, end, x);
            x = y;
            p = next;
        }
        if (chunk >= 0) f.partial(chunk);
        else f.finish(row);
    }
}

// dq and D of a long row from its chunks' sums: one block for a row and head.
template <class T>
__global__ __launch_bounds__(kAttnThreads) void attn_row_join_kernel(BwdArgs a) {
    __shared__ float sum[2 + 4 * kMaxD];
    const int h = blockIdx.x % a.s.H, W = 2 + 4 * a.s.d;
    int64_t row, first, n;
    long_segment(a.plan, a.ptr, 0, blockIdx.x / a.s.H, row, first, n);
    const int64_t ld = (int64_t)a.s.H * W;
    const float *base = a.part + first * ld + (int64_t)h * W;
    for (int c = threadIdx.x; c < W; c += kAttnThreads) {
        float s = 0.f;
#pragma unroll 8
        for (int64_t j = 0; j < n; ++j) s += base[j * ld + c];
        sum[c] = s;
    }
    __syncthreads();
    if (threadIdx.x < 2) a.D[(row * a.s.H + h) * 2 + threadIdx.x] = sum[threadIdx.x];
    for (int c = threadIdx.x; c < 2 * a.s.d; c += kAttnThreads) {
        const int half = c >= a.s.d;
        const float f = half ? -a.lambda[h] * a.s.scale : a.s.scale;
        static_cast<T *>(a.dQ)[row * a.s.ldq + (int64_t)h * 2 * a.s.d + c] =
            narrow<T>(f * (sum[2 + c] - sum[half] * sum[2 + 2 * a.s.d + c]));
    }
}

// ------------------------------------------------------------ backward, columns

// dk and dv of a key head: no dot products, the entries' coefficients are there.
template <class T, int VK, int VV, int G>
struct ColLane {
    static constexpr int GH = G / 2;
    const BwdArgs &a;
    Lane<G> L;
    int kvh;
    bool hon;
    Cols kc, vc;
    float dk[VK], dv[VV];

    __device__ __forceinline__ ColLane(const BwdArgs &a_, int hb) : a(a_), L(a_.s.hps_log2) {
        kvh = (hb << a.s.hps_log2) + L.head;
        hon = kvh < a.s.Hk;
        kvh = hon ? kvh : a.s.Hk - 1;
        kc = columns<VK>(L.g % GH, a.s.d);
        vc = columns<VV>(L.g, a.s.dv);
    }
    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int e = 0; e < VK; ++e) dk[e] = 0.f;
#pragma unroll
        for (int e = 0; e < VV; ++e) dv[e] = 0.f;
    }

    __device__ __forceinline__ void segment(int64_t p0, int64_t end) {
        const int step = L.slots * kDeep;
        for (int gi = 0; gi < a.s.grp; ++gi) {
            const int h = kvh * a.s.grp + gi;
            const float lambda = a.lambda[h];
            const T *Q = static_cast<const T *>(a.Q) + (int64_t)h * 2 * a.s.d +
                         (L.g / GH) * a.s.d + kc.col;
            const T *O = static_cast<const T *>(a.dO) + (int64_t)h * a.s.dv + vc.col;
            for (int64_t p = p0; p < end; p += step) {
                Raw<T, VK> q[kDeep];
                Raw<T, VV> o[kDeep];
                float co[kDeep][3], Dm[kDeep];
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const int64_t e = min(p + u * L.slots + L.slot, end - 1);
                    const int64_t row = a.other[e], at = a.perm[e];
                    __builtin_memcpy(co[u], a.coef + (at * a.s.H + h) * 3, 12);
                    Dm[u] = a.D[(row * a.s.H + h) * 2 + L.g / GH];
                    q[u].load(Q + row * a.s.ldq);
                    o[u].load(O + row * a.s.ldo);
                }
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    // an entry of no weight brings nothing, whatever its row holds
                    const bool in = p + u * L.slots + L.slot < end &&
                                    (co[u][0] != 0.f || co[u][1] != 0.f);
                    q[u].keep(in ? ~0u : 0u);
                    o[u].keep(in ? ~0u : 0u);
                    float c = co[u][0] - lambda * co[u][1];
                    float ds = (L.g < GH ? co[u][0] : -lambda * co[u][1]) * (co[u][2] - Dm[u]);
                    c = in ? c : 0.f;
                    ds = in ? ds * a.s.scale : 0.f;
#pragma unroll
                    for (int e = 0; e < VK; ++e) dk[e] = __builtin_fmaf(ds, q[u].at(e), dk[e]);
#pragma unroll
                    for (int e = 0; e < VV; ++e) dv[e] = __builtin_fmaf(c, o[u].at(e), dv[e]);
                }
            }
        }
        for (int b = kWave / L.slots; b < kWave; b <<= 1) {
#pragma unroll
            for (int e = 0; e < VK; ++e) dk[e] += __shfl_xor(dk[e], b);
#pragma unroll
            for (int e = 0; e < VV; ++e) dv[e] += __shfl_xor(dv[e], b);
        }
    }

    template <class O>
    __device__ __forceinline__ void store(O *k, O *v) const {
        if (L.slot != 0 || !hon) return;
        if (kc.on) store_values<O, VK>(k + (L.g / GH) * a.s.d + kc.col, dk);
        if (vc.on) store_values<O, VV>(v + vc.col, dv);
    }
};

template <class T, int VK, int VV, int G>
__global__ __launch_bounds__(kAttnThreads) void attn_col_kernel(BwdArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    T *dK = static_cast<T *>(a.dK), *dV = static_cast<T *>(a.dV);
    if ((int64_t)blockIdx.x >= a.nmain) {
        for_empty(a.plan, a.nseg, a.all_empty, a.nmain,
                  [&](int64_t col) { empty_column<T>(a, col); });
        return;
    }
    const int64_t unit = near_block(blockIdx.x, (int)a.nmain) * kAttnWaves + wave;
    const int64_t item = unit / a.s.nhb;
    if (item >= a.plan.nitems) return;
    ColLane<T, VK, VV, G> f(a, (int)(unit - item * a.s.nhb));
    int64_t p = a.plan.item_ptr[item];
    const int64_t b0 = a.plan.item_ptr[item + 1];
    const int chunk = a.plan.nchunks > 0 ? a.plan.chunk_ord[item] : -1;
    while (p < b0) {
        const int64_t col = a.idx[p];
        const int64_t end = min((int64_t)a.ptr[col + 1], b0);
        f.begin();
        f.segment(p, end);
        if (chunk >= 0) {
            float *o = a.part + ((int64_t)chunk * a.s.Hk + f.kvh) * (2 * a.s.d + a.s.dv);
            f.template store<float>(o, o + 2 * a.s.d);
        } else {
            f.template store<T>(dK + col * a.s.ldk + (int64_t)f.kvh * 2 * a.s.d,
                                dV + col * a.s.ldv + (int64_t)f.kvh * a.s.dv);
        }
        p = end;
    }
}

template <class T>
__global__ __launch_bounds__(kAttnThreads) void attn_col_join_kernel(BwdArgs a) {
    const int g = blockIdx.x % a.s.Hk, W = 2 * a.s.d + a.s.dv;
    int64_t col, first, n;
    long_segment(a.plan, a.ptr, 0, blockIdx.x / a.s.Hk, col, first, n);
    const int64_t ld = (int64_t)a.s.Hk * W;
    const float *base = a.part + first * ld + (int64_t)g * W;
    for (int c = threadIdx.x; c < W; c += kAttnThreads) {
        float s = 0.f;
#pragma unroll 8
        for (int64_t j = 0; j < n; ++j) s += base[j * ld + c];
        if (c < 2 * a.s.d)
            static_cast<T *>(a.dK)[col * a.s.ldk + (int64_t)g * 2 * a.s.d + c] = narrow<T>(s);
        else
            static_cast<T *>(a.dV)[col * a.s.ldv + (int64_t)g * a.s.dv + c - 2 * a.s.d] =
                narrow<T>(s);
    }
}

// ------------------------------------------------------------ bias, lambda

__global__ __launch_bounds__(kAttnThreads) void attn_bias_kernel(int64_t nnz, int H,
                                                                 const int32_t *rowidx,
                                                                 const float *coef, const float *D,
                                                                 const float *lambda,
                                                                 float *dbias) {
    const int64_t step = (int64_t)gridDim.x * kAttnThreads;
    for (int64_t e = (int64_t)blockIdx.x * kAttnThreads + threadIdx.x; e < nnz; e += step) {
        const int64_t row = rowidx[e];
        float s = 0.f;
        for (int h = 0; h < H; ++h) {
            const float *c = coef + (e * H + h) * 3, *d = D + (row * H + h) * 2;
            const float a1 = c[0], a2 = c[1];
            // a masked entry has no gradient, whatever its row holds
            if (a1 != 0.f || a2 != 0.f) s += a1 * (c[2] - d[0]) - lambda[h] * a2 * (c[2] - d[1]);
        }
        dbias[e] = s;
    }
}

// The same from the matrix cores' coefficients, (ds^1, -, ds^2, -) by head.
__global__ __launch_bounds__(kAttnThreads) void attn_bias_sum_kernel(int64_t nnz, int H,
                                                                     const float *coef,
                                                                     float *dbias) {
    const int64_t step = (int64_t)gridDim.x * kAttnThreads;
    for (int64_t e = (int64_t)blockIdx.x * kAttnThreads + threadIdx.x; e < nnz; e += step) {
        float s = 0.f;
        for (int h = 0; h < H; ++h) s += coef[(e * H + h) * 4] + coef[(e * H + h) * 4 + 2];
        dbias[e] = s;
    }
}

// dlambda = -sum over rows of D^2: each block adds a range of rows head by head
// (fp64), the last launch adds the blocks.
constexpr int kLambdaBlocks = 256;

__global__ __launch_bounds__(kAttnThreads) void attn_lambda_part_kernel(int64_t nrows, int H,
                                                                        const float *D,
                                                                        double *part) {
    __shared__ double sh[kAttnThreads];
    const int64_t per = (nrows + gridDim.x - 1) / gridDim.x;
    const int64_t r0 = blockIdx.x * per, r1 = min(r0 + per, nrows);
    for (int h0 = 0; h0 < H; h0 += kAttnThreads) {
        const int heads = min(H - h0, kAttnThreads), rows = kAttnThreads / heads;
        const int h = threadIdx.x % heads, r = threadIdx.x / heads;
        double s = 0.0;
        if (r < rows)
            for (int64_t i = r0 + r; i < r1; i += rows) s += D[(i * H + h0 + h) * 2 + 1];
        sh[threadIdx.x] = s;
        __syncthreads();
        if (r == 0) {
            for (int o = 1; o < rows; ++o) s += sh[threadIdx.x + o * heads];
            part[(int64_t)blockIdx.x * H + h0 + h] = s;
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(kAttnThreads) void attn_lambda_kernel(int H, int nb,
                                                                   const double *part,
                                                                   float *dlambda) {
    const int h = blockIdx.x;
    __shared__ double sh[kAttnThreads];
    double s = 0.0;
    for (int b = threadIdx.x; b < nb; b += kAttnThreads) s += part[(int64_t)b * H + h];
    sh[threadIdx.x] = s;
    __syncthreads();
    for (int w = kAttnThreads / 2; w >= 1; w >>= 1) {
        if ((int)threadIdx.x < w) sh[threadIdx.x] += sh[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) dlambda[h] = (float)-sh[0];
}

// ------------------------------------------------------------ host

template <int N>
using Int = std::integral_constant<int, N>;

int pow2_at_least(int n) {
    int p = 1;
    while (p < n) p <<= 1;
    return p;
}

// Lanes of a head: whole 16-byte pieces of a half and of a value.  A width
// below one piece goes one value a lane; those shapes take all the lanes that
// any width needs (one kernel each).
int head_lanes(const nsd_attn *s) {
    const int vec = s->dtype == NSD_BF16 ? 8 : 4;
    if (s->d < vec || s->dv < vec) return s->dtype == NSD_BF16 ? 32 : 64;
    return pow2_at_least(std::max<int>(2 * (int)ceil_div(s->d, vec),
                                       (int)ceil_div(s->dv, vec)));
}

template <class T, int G, class F>
void with_widths(const nsd_attn *s, F f) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool exact = s->d == G / 2 * V;
    if (exact) f(T(), Int<V>(), Int<V>(), Int<G>(), std::true_type());
    else f(T(), Int<V>(), Int<V>(), Int<G>(), std::false_type());
}

template <class T, class F>
void with_lanes(const nsd_attn *s, F f) {
    constexpr int V = 16 / (int)sizeof(T), most = sizeof(T) == 2 ? 32 : 64;
    if (s->d < V && s->dv < V)
        return f(T(), Int<1>(), Int<1>(), Int<most>(), std::false_type());
    if (s->d < V) return f(T(), Int<1>(), Int<V>(), Int<most>(), std::false_type());
    if (s->dv < V) return f(T(), Int<V>(), Int<1>(), Int<most>(), std::false_type());
    switch (head_lanes(s)) {
        case 2: return with_widths<T, 2>(s, f);
        case 4: return with_widths<T, 4>(s, f);
        case 8: return with_widths<T, 8>(s, f);
        case 16: return with_widths<T, 16>(s, f);
        case 32: return with_widths<T, 32>(s, f);
        default:
            if constexpr (sizeof(T) == 4) with_widths<T, 64>(s, f);
    }
}

template <class F>
void with_shape(const nsd_attn *s, F f) {
    if (s->dtype == NSD_BF16) with_lanes<uint16_t>(s, f);
    else with_lanes<float>(s, f);
}

// Heads side by side in a wave.
int heads_per_slot_log2(int heads, int lanes) {
    int n = 0;
    while ((2 << n) <= heads && lanes * (2 << n) <= 32) ++n;
    return n;
}

Shape make_shape(const nsd_attn *s, int heads) {
    Shape r;
    r.H = s->heads;
    r.Hk = s->kv_heads;
    r.grp = s->heads / s->kv_heads;
    r.d = s->d;
    r.dv = s->dv;
    r.ldq = s->ldq;
    r.ldk = s->ldk;
    r.ldv = s->ldv;
    r.ldo = s->ldo;
    r.scale = s->scale;
    r.hps_log2 = heads_per_slot_log2(heads, head_lanes(s));
    r.nhb = (int32_t)ceil_div(heads, 1 << r.hps_log2);
    return r;
}

nsd_status check_attn(const nsd_attn *s) {
    NSD_REQUIRE(s != nullptr, "attention descriptor is NULL");
    NSD_REQUIRE(s->heads >= 1 && s->kv_heads >= 1 && s->heads % s->kv_heads == 0,
                "%d heads over %d key heads", s->heads, s->kv_heads);
    NSD_REQUIRE(s->d >= 1 && s->dv >= 1, "widths %d and %d", s->d, s->dv);
    NSD_REQUIRE(s->dtype == NSD_F32 || s->dtype == NSD_BF16, "unknown type %d", s->dtype);
    if (s->d > kMaxD || s->dv > kMaxDv || s->heads > 4096)
        return fail(NSD_ERR_UNSUPPORTED, "%d heads of widths %d and %d (at most 4096, %d and %d)",
                    s->heads, s->d, s->dv, kMaxD, kMaxDv);
    NSD_REQUIRE(s->ldq >= (int64_t)s->heads * 2 * s->d && s->ldk >= (int64_t)s->kv_heads * 2 * s->d &&
                    s->ldv >= (int64_t)s->kv_heads * s->dv && s->ldo >= (int64_t)s->heads * s->dv,
                "rows overlap: ldq %lld, ldk %lld, ldv %lld, ldo %lld", (long long)s->ldq,
                (long long)s->ldk, (long long)s->ldv, (long long)s->ldo);
    return NSD_OK;
}

struct AttnWs {
    float *part_row, *part_col, *part_D, *coef, *D;
    double *lambda;
};
size_t carve_attn(void *ws, const nsd_csr *A, const nsd_csc *At, const nsd_attn *s, AttnWs *w) {
    Carver c(ws);
    const bool cores = cores_pay(s);
    const size_t chunk_heads = (size_t)A->plan.nchunks * s->heads;
    const size_t row = std::max(4 + 2 * s->dv, !At ? 0 : cores ? 2 * s->d : 2 + 4 * s->d);
    w->part_row = c.take<float>(chunk_heads * row);
    if (At) {
        w->part_col = c.take<float>((size_t)At->plan.nchunks * s->kv_heads * (2 * s->d + s->dv));
        w->part_D = c.take<float>(cores ? chunk_heads * 2 : 0);
        w->coef = c.take<float>((size_t)A->nnz * s->heads * (cores ? 4 : 3));
        w->D = c.take<float>((size_t)A->nrows * s->heads * 2);
        w->lambda = c.take<double>((size_t)kLambdaBlocks * s->heads);
    }
    return c.bytes();
}

// Blocks of a pass: `units` (one item for four waves each), then those that walk
// the empty segments, four at a time.
constexpr int64_t kEmptyBlocks = 1 << 20;
nsd_status pass_blocks(const nsd_plan &plan, int32_t nnz, int32_t nseg, int heads, int64_t units,
                       int64_t *nmain, int64_t *nblocks) {
    *nmain = nnz == 0 ? 0 : units;
    *nblocks = *nmain + std::min(ceil_div(nnz == 0 ? nseg : plan.nempty, kAttnWaves),
                                 kEmptyBlocks);
    const int64_t joins = nnz == 0 ? 0 : (int64_t)plan.nlong * heads;
    if (std::max(*nblocks, joins) > kMaxBlocks)
        return fail(NSD_ERR_TOO_LARGE, "%lld blocks", (long long)std::max(*nblocks, joins));
    return NSD_OK;
}
int64_t pass_units(bool cores, int64_t items, const Shape &shape, const Slab &slab) {
    return cores ? mfma_blocks(items, slab) : ceil_div(items * shape.nhb, kAttnWaves);
}

template <bool DECODE>
void launch_forward(bool cores, const nsd_attn *s, const FwdArgs &a, const Slab &slab, int64_t nb,
                    hipStream_t st) {
    if (cores)
        return mfma_forward(a, DECODE ? one_row(slab) : slab, nb, DECODE, st);
    with_shape(s, [&](auto T, auto VK, auto VV, auto G, auto EX) {
        attn_fwd_kernel<decltype(T), VK(), VV(), G(), EX(), DECODE>
            <<<(unsigned)nb, kAttnThreads, 0, st>>>(a);
    });
}

nsd_status check_chunks(const nsd_plan &pl, int32_t nnz) {
    NSD_REQUIRE(nnz == 0 || pl.nchunks == 0 || (pl.chunk_ord && pl.long_seg), "plan is not built");
    return NSD_OK;
}

}  // namespace

}  // namespace nsd

using namespace nsd;

extern "C" {

nsd_status nsd_attn_item_len(int32_t nnz, const nsd_attn *s, int32_t *item_len) {
    NSD_REQUIRE(item_len != nullptr, "item_len is NULL");
    NSD_REQUIRE(nnz >= 0, "negative nnz");
    NSD_TRY(check_attn(s));
    // The vector form: 16 waves a SIMD of every head group's items, as long as the
    // other passes' at most (1M entries, 4 heads of 8: 472 us a training step at up
    // to 256, 509 at up to 2048).  On the matrix cores: eight, whose rows can share
    // tiles only within an item (a window of 256: 2.19 ms at 256, 1.31 at 1070, 1.48
    // at 2048).
    const bool cores = cores_pay(s);
    const int64_t units = (int64_t)nnz * (cores ? make_slab(s).nslab : make_shape(s, s->heads).nhb);
    *item_len = (int32_t)(cores ? std::min<int64_t>(2048, std::max<int64_t>(32, units / 8192))
                                : std::min<int64_t>(256, std::max<int64_t>(32, units / 16384)));
    return NSD_OK;
}

nsd_status nsd_attn_diff_workspace_size(const nsd_csr *A, const nsd_csc *At, const nsd_attn *s,
                                        size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_TRY(check_csr(A, false, true));
    if (At) NSD_TRY(check_csc(At, A));
    NSD_TRY(check_attn(s));
    AttnWs w;
    *bytes = carve_attn(nullptr, A, At, s, &w);
    return NSD_OK;
}

nsd_status nsd_attn_diff(const nsd_csr *A, const nsd_attn *s, const void *Q, const void *K,
                         const void *V, const float *lambda, const float *bias, void *O,
                         float *stat, void *ws, size_t ws_bytes, void *stream) {
    NSD_TRY(check_csr(A, false, true));
    NSD_TRY(check_chunks(A->plan, A->nnz));
    NSD_TRY(check_attn(s));
    if (A->nrows == 0) return NSD_OK;
    NSD_REQUIRE(Q && lambda && O, "a NULL array");
    NSD_REQUIRE(A->nnz == 0 || (K && V), "a NULL array");
    AttnWs w = {};
    const size_t need = carve_attn(ws, A, nullptr, s, &w);
    if (need > 0 && (ws == nullptr || ws_bytes < need))
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, need);
    FwdArgs a = {};
    a.s = make_shape(s, s->heads);
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.lambda = lambda;
    a.bias = bias;
    a.O = O;
    a.stat = stat;
    a.part = w.part_row;
    a.rowptr = A->rowptr;
    a.rowidx = A->rowidx;
    a.colind = A->colind;
    a.plan = A->plan;
    a.nrows = A->nrows;
    a.all_empty = A->nnz == 0;
    int64_t nb;
    const Slab slab = make_slab(s);
    const bool cores = cores_pay(s);
    NSD_TRY(pass_blocks(A->plan, A->nnz, A->nrows, s->heads,
                        pass_units(cores, A->plan.nitems, a.s, slab), &a.nmain, &nb));
    const hipStream_t st = as_stream(stream);
    launch_forward<false>(cores, s, a, slab, nb, st);
    NSD_TRY(check_launch("attn_fwd_kernel"));
    if (A->nnz > 0 && A->plan.nlong > 0) {
        JoinArgs j = {a.s, a.part, lambda, O, stat, A->rowptr, A->plan, 0};
        const unsigned n = (unsigned)A->plan.nlong * s->heads;
        if (s->dtype == NSD_BF16) attn_join_kernel<uint16_t><<<n, kAttnThreads, 0, st>>>(j);
        else attn_join_kernel<float><<<n, kAttnThreads, 0, st>>>(j);
        return check_launch("attn_join_kernel");
    }
    return NSD_OK;
}

nsd_status nsd_attn_diff_vjp(const nsd_csr *A, const nsd_csc *At, const nsd_attn *s, const void *Q,
                             const void *K, const void *V, const float *lambda, const float *bias,
                             const float *stat, const void *dO, void *dQ, void *dK, void *dV,
                             float *dlambda, float *dbias, void *ws, size_t ws_bytes,
                             void *stream) {
    NSD_TRY(check_csr(A, false, true));
    NSD_TRY(check_csc(At, A));
    NSD_TRY(check_chunks(A->plan, A->nnz));
    NSD_TRY(check_chunks(At->plan, At->nnz));
    NSD_TRY(check_attn(s));
    NSD_REQUIRE(lambda && dlambda, "a NULL array");
    NSD_REQUIRE(A->nrows == 0 || (Q && dO && dQ && stat), "a NULL array");
    NSD_REQUIRE(A->ncols == 0 || (K && V && dK && dV), "a NULL array");
    AttnWs w = {};
    const size_t need = carve_attn(ws, A, At, s, &w);
    if (ws == nullptr || ws_bytes < need)
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, need);
    const hipStream_t st = as_stream(stream);
    BwdArgs a = {};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.dO = dO;
    a.lambda = lambda;
    a.bias = bias;
    a.stat = stat;
    a.dQ = dQ;
    a.dK = dK;
    a.dV = dV;
    a.coef = w.coef;
    a.D = w.D;
    BwdArgs r = a, c = a;
    r.s = make_shape(s, s->heads);
    r.part = w.part_row;
    r.ptr = A->rowptr;
    r.idx = A->rowidx;
    r.other = A->colind;
    r.plan = A->plan;
    r.nseg = A->nrows;
    c.s = make_shape(s, s->kv_heads);
    c.part = w.part_col;
    c.ptr = At->colptr;
    c.idx = At->colidx;
    c.other = At->rowind;
    c.perm = At->perm;
    c.plan = At->plan;
    c.nseg = A->ncols;
    r.all_empty = c.all_empty = A->nnz == 0;
    int64_t nr, nc;
    const Slab slab = make_slab(s), cslab = column_slab(slab);
    const bool cores = cores_pay(s);
    NSD_TRY(pass_blocks(A->plan, A->nnz, A->nrows, s->heads,
                        pass_units(cores, A->plan.nitems, r.s, slab), &r.nmain, &nr));
    NSD_TRY(pass_blocks(At->plan, A->nnz, A->ncols, s->kv_heads,
                        pass_units(cores, At->plan.nitems, c.s, cslab), &c.nmain, &nc));
    const bool bf16 = s->dtype == NSD_BF16;
    const bool long_rows = A->nnz > 0 && A->plan.nlong > 0;
    if (cores) {
        r.part_D = w.part_D;
        if (nr > 0) mfma_rows(r, slab, nr, st);
        if (nc > 0) mfma_columns(c, cslab, nc, st);
        NSD_TRY(check_launch("mfma_row_kernel"));
    } else {
        if (nr > 0) {
            with_shape(s, [&](auto T, auto VK, auto VV, auto G, auto) {
                attn_row_kernel<decltype(T), VK(), VV(), G()>
                    <<<(unsigned)nr, kAttnThreads, 0, st>>>(r);
            });
            NSD_TRY(check_launch("attn_row_kernel"));
        }
        if (long_rows) {
            const unsigned n = (unsigned)A->plan.nlong * s->heads;
            if (bf16) attn_row_join_kernel<uint16_t><<<n, kAttnThreads, 0, st>>>(r);
            else attn_row_join_kernel<float><<<n, kAttnThreads, 0, st>>>(r);
            NSD_TRY(check_launch("attn_row_join_kernel"));
        }
        if (nc > 0) {
            with_shape(s, [&](auto T, auto VK, auto VV, auto G, auto) {
                attn_col_kernel<decltype(T), VK(), VV(), G()>
                    <<<(unsigned)nc, kAttnThreads, 0, st>>>(c);
            });
            NSD_TRY(check_launch("attn_col_kernel"));
        }
    }
    if (A->nnz > 0 && At->plan.nlong > 0) {
        const unsigned n = (unsigned)At->plan.nlong * s->kv_heads;
        if (bf16) attn_col_join_kernel<uint16_t><<<n, kAttnThreads, 0, st>>>(c);
        else attn_col_join_kernel<float><<<n, kAttnThreads, 0, st>>>(c);
        NSD_TRY(check_launch("attn_col_join_kernel"));
    }
    if (dbias && A->nnz > 0) {
        const int64_t nb = std::min<int64_t>(ceil_div(A->nnz, kAttnThreads), 8192);
        if (cores)
            attn_bias_sum_kernel<<<(unsigned)nb, kAttnThreads, 0, st>>>(A->nnz, s->heads, w.coef,
                                                                        dbias);
        else
            attn_bias_kernel<<<(unsigned)nb, kAttnThreads, 0, st>>>(
                A->nnz, s->heads, A->rowidx, w.coef, w.D, lambda, dbias);
        NSD_TRY(check_launch("attn_bias_kernel"));
    }
    const int nl = (int)std::min<int64_t>(std::max<int64_t>(ceil_div(A->nrows, 16), 1),
                                          kLambdaBlocks);
    attn_lambda_part_kernel<<<nl, kAttnThreads, 0, st>>>(A->nrows, s->heads, w.D, w.lambda);
    attn_lambda_kernel<<<s->heads, kAttnThreads, 0, st>>>(s->heads, nl, w.lambda, dlambda);
    return check_launch("attn_lambda_kernel");
}

// Splits of a decode call's rows: enough for four waves a SIMD, of at least
// kMinSplit entries.
static void decode_splits(int32_t nrows, int32_t max_len, const nsd_attn *s, int32_t *nsplit,
                          int32_t *per) {
    const int64_t heads = cores_pay(s) ? make_slab(s).nslab : make_shape(s, s->heads).nhb;
    const int64_t units = std::max<int64_t>(nrows * heads, 1);
    int64_t n = std::min<int64_t>(ceil_div(4096, units), ceil_div(max_len, kMinSplit));
    n = std::max<int64_t>(n, 1);
    *per = (int32_t)std::max<int64_t>(ceil_div(ceil_div(max_len, n), 32) * 32, 32);
    *nsplit = (int32_t)std::max<int64_t>(ceil_div(max_len, *per), 1);
}

nsd_status nsd_attn_diff_decode_workspace_size(int32_t nrows, int32_t max_len, const nsd_attn *s,
                                               size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_REQUIRE(nrows >= 0 && max_len >= 0, "negative size");
    NSD_TRY(check_attn(s));
    int32_t nsplit, per;
    decode_splits(nrows, max_len, s, &nsplit, &per);
    *bytes = nsplit == 1 ? 0
                         : (size_t)nrows * nsplit * s->heads * (4 + 2 * s->dv) * sizeof(float);
    return NSD_OK;
}

nsd_status nsd_attn_diff_decode(int32_t nrows, const int32_t *rowptr, const int32_t *colind,
                                int32_t max_len, const nsd_attn *s, const void *Q, const void *K,
                                const void *V, const float *lambda, const float *bias, void *O,
                                void *ws, size_t ws_bytes, void *stream) {
    size_t need;
    NSD_TRY(nsd_attn_diff_decode_workspace_size(nrows, max_len, s, &need));
    if (nrows == 0) return NSD_OK;
    NSD_REQUIRE(rowptr && Q && lambda && O, "a NULL array");
    NSD_REQUIRE(colind == nullptr || (K && V), "keys without K or V");
    if (need > 0 && (ws == nullptr || ws_bytes < need))
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, need);
    FwdArgs a = {};
    a.s = make_shape(s, s->heads);
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.lambda = lambda;
    a.bias = bias;
    a.O = O;
    a.part = static_cast<float *>(ws);
    a.rowptr = rowptr;
    a.colind = colind;
    a.nrows = nrows;
    decode_splits(nrows, max_len, s, &a.nsplit, &a.per);
    const Slab slab = make_slab(s);
    const bool cores = cores_pay(s);
    a.nmain = pass_units(cores, (int64_t)nrows * a.nsplit, a.s, slab);
    const int64_t joins = a.nsplit > 1 ? (int64_t)nrows * s->heads : 0;
    if (std::max(a.nmain, joins) > kMaxBlocks)
        return fail(NSD_ERR_TOO_LARGE, "%lld blocks", (long long)std::max(a.nmain, joins));
    const hipStream_t st = as_stream(stream);
    launch_forward<true>(cores, s, a, slab, a.nmain, st);
    NSD_TRY(check_launch("attn_fwd_kernel"));
    if (a.nsplit > 1) {
        JoinArgs j = {a.s, a.part, lambda, O, nullptr, rowptr, nsd_plan{}, a.nsplit};
        const unsigned n = (unsigned)joins;
        if (s->dtype == NSD_BF16) attn_join_kernel<uint16_t><<<n, kAttnThreads, 0, st>>>(j);
        else attn_join_kernel<float><<<n, kAttnThreads, 0, st>>>(j);
        return check_launch("attn_join_kernel");
    }
    return NSD_OK;
}

}  // extern "C"
