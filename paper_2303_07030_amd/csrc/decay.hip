// Linear attention with a decay for each head: the calls, the join of segments' states, and
// the step of single tokens.  The scans themselves are in decay.hpp.
//
// A sequence is cut into segments where sequences, heads and columns alone do not fill the
// card: the states of every segment by itself (a scan without outputs), a join that
// carries each sequence's state through its segments,
//   start_{c+1} = w^n start_c + state_c
// (HBM-bound: a prompt of 128 segments of 8 heads of 128 by 128 24 us, 5.5 TB/s),
// and the scan of every segment from its start.  The join leaves at a segment's place in the
// workspace the state that the segment starts from (backwards: the one that comes back to its
// end).
#include <algorithm>
#include <climits>

#include "decay.hpp"

namespace nsd {
namespace decay {

namespace {

constexpr int kJoinThreads = 256, kMaxScanThreads = 512;

// One element of a head's state of a sequence through the sequence's segments.
template <int VEC>
__global__ __launch_bounds__(kJoinThreads) void decay_join_kernel(
    int32_t ntok, int32_t H, const int32_t *__restrict__ seqptr, int32_t seg_len, bool rev,
    const float *__restrict__ decay, float *__restrict__ states, int64_t per, const float *start,
    float *end) {
    const int nb = (int)((per + kJoinThreads * VEC - 1) / (kJoinThreads * VEC));
    const int s = blockIdx.x / nb / H, h = blockIdx.x / nb % H;
    const int64_t e = ((int64_t)(blockIdx.x % nb) * kJoinThreads + threadIdx.x) * VEC;
    if (e >= per) return;
    const int begin = max(seqptr[s], 0), stop = min(seqptr[s + 1], ntok);
    const int n = max(stop - begin, 0), id0 = begin / seg_len + s;
    const int nc = n / seg_len + (n % seg_len != 0);
    const int64_t own = ((int64_t)s * H + h) * per + e, step = (int64_t)H * per;
    float *const at = states + ((int64_t)id0 * H + h) * per + e;
    const double g = (double)decay[h];
    const double whole = exp(g * (double)seg_len);
    const int rest = n - (nc - 1) * seg_len;
    const double part = nc ? exp(g * (double)rest) : 1.0;
    double cur[VEC];  // in 64 bits: each segment's product is one more rounding else
#pragma unroll
    for (int i = 0; i < VEC; ++i) cur[i] = start ? (double)start[own + i] : 0.0;
    constexpr int kAhead = 8;
    for (int c0 = 0; c0 < nc; c0 += kAhead) {
        float x[kAhead][VEC];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int c = min(c0 + u, nc - 1);
            __builtin_memcpy(x[u], at + (int64_t)(rev ? nc - 1 - c : c) * step, sizeof x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (c0 + u >= nc) break;
            const int c = rev ? nc - 1 - c0 - u : c0 + u;
            const double w = c == nc - 1 ? part : whole;
            float y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                y[i] = (float)cur[i];
                cur[i] = __builtin_fma(cur[i], w, (double)x[u][i]);
            }
            __builtin_memcpy(at + (int64_t)c * step, y, sizeof y);
        }
    }
    if (end)
#pragma unroll
        for (int i = 0; i < VEC; ++i) end[own + i] = (float)cur[i];
}

int64_t join_blocks(int32_t nseq, int32_t H, int64_t per) {
    return (int64_t)nseq * H * ceil_div(per, kJoinThreads * (per % 4 == 0 ? 4 : 1));
}

nsd_status join(const Scan &a, bool rev, float *states, const float *start, float *end,
                hipStream_t st) {
    const bool four = a.per % 4 == 0;
    const unsigned grid = (unsigned)join_blocks(a.nseq, a.H, a.per);
    if (four)
        decay_join_kernel<4><<<grid, kJoinThreads, 0, st>>>(a.ntok, a.H, a.seqptr, a.seg_len, rev,
                                                            a.decay, states, a.per, start, end);
    else
        decay_join_kernel<1><<<grid, kJoinThreads, 0, st>>>(a.ntok, a.H, a.seqptr, a.seg_len, rev,
                                                            a.decay, states, a.per, start, end);
    return check_launch("decay_join_kernel");
}

// The gradients of key heads: the sums of their query heads', rows of sequences alone.
constexpr int kSumThreads = 256;
template <class T>
__global__ __launch_bounds__(kSumThreads) void decay_heads_kernel(
    int32_t ntok, int32_t nseq, const int32_t *__restrict__ seqptr, int32_t Hk, int32_t grp,
    int32_t width, const float *__restrict__ part, T *__restrict__ out, int64_t ld) {
    const int64_t n = (int64_t)Hk * width;
    const int first = max(seqptr[0], 0), last = min(seqptr[nseq], ntok);
    for (int64_t t = (int64_t)first + blockIdx.x; t < last; t += gridDim.x)
        for (int64_t c = threadIdx.x; c < n; c += kSumThreads) {
            const float *p = part + (t * Hk * grp + c / width * grp) * width + c % width;
            float v = 0.f;
            for (int i = 0; i < grp; ++i) v += p[(int64_t)i * width];
            out[t * ld + c] = narrowed<T>(v);
        }
}

// Sums of the blocks' shares of a head's decay gradient, in their order.
__global__ __launch_bounds__(kSumThreads) void decay_sums_kernel(int64_t nseg, int32_t H, int32_t nvb,
                                                                 const float *__restrict__ sums,
                                                                 float *__restrict__ out) {
    __shared__ double of[kSumThreads];
    const int h = blockIdx.x;
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < nseg * nvb; i += kSumThreads)
        v += (double)sums[(i / nvb * H + h) * nvb + i % nvb];
    of[threadIdx.x] = v;
    __syncthreads();
    for (int m = kSumThreads / 2; m > 0; m /= 2) {
        if ((int)threadIdx.x < m) of[threadIdx.x] += of[threadIdx.x + m];
        __syncthreads();
    }
    if (threadIdx.x == 0) out[h] = (float)of[0];
}

// ------------------------------------------------------------ single tokens

constexpr int kStepThreads = 256;

struct Step {
    int32_t nrows, nslots, H, grp, d, dv;
    int32_t lanes;  // of VEC columns each, that a block takes of a state's row
    float scale;
    const int32_t *slot;
    const void *Q, *K, *V;
    int64_t ldq, ldk, ldv, ldo;
    const float *decay;
    float *state;
    void *O;
};

// A row's head and some columns of its state: read, decayed, added to, written, multiplied.  HBM-
// bound: the state is 8 bytes a value, the row nothing beside it.  64 rows of 16 heads of 64 by
// 128: 13.4 us (5.0 TB/s).
template <class T, int VEC>
__global__ __launch_bounds__(kStepThreads) void decay_step_kernel(Step a) {
    __shared__ float qs[kMaxWidth], ks[kMaxWidth];
    __shared__ float sum[kStepThreads * VEC];
    __shared__ int before, after;
    const int ncb = (a.dv + a.lanes * VEC - 1) / (a.lanes * VEC);
    const int cb = blockIdx.x % ncb, h = blockIdx.x / ncb % a.H;
    int r = blockIdx.x / ncb / a.H;
    const int slot = a.slot ? a.slot[r] : r;
    const int lane = threadIdx.x % a.lanes, rows = kStepThreads / a.lanes;
    const int row0 = threadIdx.x / a.lanes;
    const int c = (cb * a.lanes + lane) * VEC;
    const bool in = c < a.dv;  // (VEC 4: dv is a multiple of it)
    T *const out = static_cast<T *>(a.O) + (int64_t)h * a.dv + c;
    if (slot < 0 || slot >= a.nslots) {
        const float none[VEC] = {};
        if (in && row0 == 0) store_row_values<VEC, T>(out + (int64_t)r * a.ldo, none);
        return;
    }
    float *const S = a.state + ((int64_t)slot * a.H + h) * a.d * a.dv + c;
    // A slow decay by what it takes away: e^g rounded near 1 would be another decay, the same way
    // off at every token (g = -1e-6: by 1.3%).
    const double g = (double)a.decay[h];
    const bool slow = g != 0.0 && g > -0.6931;  // e^g above 1/2
    const float w = g == 0.0 ? 1.f : (float)(slow ? expm1(g) : exp(g));
    const bool several = a.slot && a.nrows > 1;
    for (;;) {
        if (threadIdx.x == 0) before = after = INT_MAX;
        if (threadIdx.x < a.d) {
            const T *q = static_cast<const T *>(a.Q) + (int64_t)r * a.ldq + (int64_t)h * a.d;
            const T *k = static_cast<const T *>(a.K) + (int64_t)r * a.ldk + (int64_t)(h / a.grp) * a.d;
            qs[threadIdx.x] = widened(q[threadIdx.x]);
            ks[threadIdx.x] = widened(k[threadIdx.x]);
        }
        float v[VEC] = {}, o[VEC] = {};
        if (in)
            load_values<VEC, T>(static_cast<const T *>(a.V) + (int64_t)r * a.ldv +
                                    (int64_t)(h / a.grp) * a.dv + c, v);
        __syncthreads();
        if (several) {  // the slot's first row takes them all, one after the other
            int first = INT_MAX, next = INT_MAX;
            for (int i = threadIdx.x; i < a.nrows; i += kStepThreads)
                if (a.slot[i] == slot) {
                    first = min(first, i);
                    if (i > r) next = min(next, i);
                }
            if (first < r) atomicMin(&before, first);
            if (next != INT_MAX) atomicMin(&after, next);
            __syncthreads();
            if (before < r && r == blockIdx.x / ncb / a.H) return;
        }
        constexpr int kAhead = 8;
        for (int k0 = row0; in && k0 < a.d; k0 += rows * kAhead) {
            float x[kAhead][VEC];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (k0 + u * rows < a.d)
                    __builtin_memcpy(x[u], S + (int64_t)(k0 + u * rows) * a.dv, sizeof x[u]);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int k = k0 + u * rows;
                if (k >= a.d) break;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    x[u][e] = __builtin_fmaf(ks[k], v[e], __builtin_fmaf(x[u][e], w, slow ? x[u][e] : 0.f));
                    o[e] = __builtin_fmaf(qs[k], x[u][e], o[e]);
                }
                __builtin_memcpy(S + (int64_t)k * a.dv, x[u], sizeof x[u]);
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[threadIdx.x * VEC + e] = o[e];
        __syncthreads();
        if (in && row0 == 0) {
            for (int i = 1; i < rows; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] += sum[(i * a.lanes + lane) * VEC + e];
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] *= a.scale;
            store_row_values<VEC, T>(out + (int64_t)r * a.ldo, o);
        }
        const int next = several ? after : INT_MAX;
        if (next == INT_MAX) return;
        r = next;
        __syncthreads();
    }
}

// ------------------------------------------------------------------- host

constexpr int kMaxDistance = 1 << 22;

nsd_status check_decay(const nsd_decay *s) {
    NSD_REQUIRE(s != nullptr, "descriptor is NULL");
    NSD_REQUIRE(s->heads >= 1 && s->kv_heads >= 1 && s->heads % s->kv_heads == 0,
                "%d heads over %d", s->heads, s->kv_heads);
    NSD_REQUIRE(s->d >= 1 && s->dv >= 1, "heads of %d and %d values", s->d, s->dv);
    NSD_REQUIRE(known_dtype(s->dtype), "unknown type %d", s->dtype);
    if (s->d > kMaxWidth || s->dv > kMaxWidth)
        return fail(NSD_ERR_UNSUPPORTED, "heads of %d and %d values (up to %d)", s->d, s->dv, kMaxWidth);
    if (s->heads > 4096) return fail(NSD_ERR_UNSUPPORTED, "%d heads (up to 4096)", s->heads);
    NSD_REQUIRE(s->ldq >= (int64_t)s->heads * s->d && s->ldk >= (int64_t)s->kv_heads * s->d &&
                    s->ldv >= (int64_t)s->kv_heads * s->dv && s->ldo >= (int64_t)s->heads * s->dv,
                "row distances below the heads' widths");
    // a chunk's places in its rows are counted in 32 bits
    if (std::max({s->ldq, s->ldk, s->ldv, s->ldo}) > kMaxDistance)
        return fail(NSD_ERR_UNSUPPORTED, "rows more than %d values apart", kMaxDistance);
    return NSD_OK;
}

// Tokens of a segment: as many as leave the card kEnough blocks, INT_MAX where whole sequences
// do, or are short.  (A training step of 5,003 tokens of 6 heads in fp32: segments of at least
// 256 tokens 315 us, 128 275, 64 182; 4,096 tokens of 8 heads of 64 in bf16, forwards, where 64
// tokens are one chunk: 34, 30 and 35; of 16 heads over 4 of 128: 74, 75 and 85.  A prompt of
// 65,536 tokens of 8 heads of 128, and a training step of 32,768 tokens of 16 heads of 64 by 128:
// 512 blocks 393 and 1,154 us, 1,024 334 and 1,019, 2,048 361 and 1,041.)
constexpr int kShortest = 64, kLongest = 8192, kEnough = 1024;

int segment_tokens(int32_t ntok, int32_t max_len, const nsd_decay *s) {
    const int64_t cols = ceil_div(std::max(s->d, s->dv), 128) * s->heads;
    int len = kLongest;
    while (len > kShortest && ntok / len * cols < kEnough) len /= 2;
    return max_len <= len ? INT_MAX : len;
}

// The most segments that a batch of up to `ntok` tokens is cut into, less one for each sequence; -1
// if none is cut.  (Fewer tokens may have more segments, as theirs are shorter.)
int64_t most_segments(int32_t ntok, int32_t max_len, const nsd_decay *s) {
    const int64_t enough = ceil_div(kEnough, ceil_div(std::max(s->d, s->dv), 128) * s->heads);
    int64_t most = -1;
    for (int64_t len = kShortest; len <= kLongest && len < max_len; len *= 2) {
        // the most tokens whose segments are of this length
        const int64_t n = len == kLongest ? ntok : std::min<int64_t>(ntok, 2 * len * enough - 1);
        if (len == kShortest || n / len >= enough) most = std::max(most, n / len);
    }
    return most;
}

nsd_status check_sizes(int32_t ntok, int32_t nseq, int32_t max_len, const nsd_decay *s) {
    NSD_TRY(check_decay(s));
    NSD_REQUIRE(ntok >= 0 && nseq >= 0 && max_len >= 0, "a negative size");
    // a launch's threads are counted in 32 bits
    const int64_t scans = ((int64_t)ntok / segment_tokens(ntok, max_len, s) + nseq) * s->heads *
                          ceil_div(std::max(s->d, s->dv), 64);
    const int64_t joins = join_blocks(nseq, s->heads, (int64_t)s->d * s->dv);
    if (ntok > INT32_MAX / 2 || std::max(scans, joins) > UINT32_MAX / kMaxScanThreads)
        return fail(NSD_ERR_TOO_LARGE, "%d tokens, %d sequences of %d heads", ntok, nseq, s->heads);
    return NSD_OK;
}

// The workspace of a call; `room`: of any that is no larger (of the same heads).
struct DecayWs {
    float *forth, *back, *dk, *dv, *sums;
    int32_t seg_len, nseg, nvb;
    size_t bytes;
    DecayWs(void *ws, int32_t ntok, int32_t nseq, int32_t max_len, const nsd_decay *s, bool gradient,
            bool room = false) {
        Carver c(ws);
        seg_len = segment_tokens(ntok, max_len, s);
        nseg = ntok / seg_len + nseq;
        const int64_t cuts = room ? most_segments(ntok, max_len, s) : cut() ? ntok / seg_len : -1;
        const int64_t segments = std::max<int64_t>(cuts, 0) + nseq;
        const size_t states = cuts >= 0 ? (size_t)segments * s->heads * s->d * s->dv : 0;
        const bool grouped = s->heads != s->kv_heads;
        forth = c.take<float>(states);
        back = dk = dv = sums = nullptr;
        const int wide = std::max(s->d, s->dv);
        nvb = (int)ceil_div(wide, block_columns(kDerivative, s->dtype == NSD_BF16, wide));
        if (gradient) {
            back = c.take<float>(states);
            dk = c.take<float>(grouped ? (size_t)ntok * s->heads * s->d : 0);
            dv = c.take<float>(grouped ? (size_t)ntok * s->heads * s->dv : 0);
            sums = c.take<float>((size_t)segments * s->heads * nvb);
        }
        bytes = std::max<size_t>(c.bytes(), 256);
    }
    bool cut() const { return seg_len != INT_MAX; }
};

// A call's arrays.  (Other blocks read what one has written: outputs are apart from them all, but
// for the states behind the sequences, of which every block writes what it alone has read.)
struct Areas {
    int64_t n;  // tokens
    const nsd_decay *s;
    int64_t state = 4 * (int64_t)s->heads * s->d * s->dv;
    Area q(const void *p) const { return row_area(p, n, (int64_t)s->heads * s->d, s->ldq, s->dtype); }
    Area k(const void *p) const { return row_area(p, n, (int64_t)s->kv_heads * s->d, s->ldk, s->dtype); }
    Area v(const void *p) const { return row_area(p, n, (int64_t)s->kv_heads * s->dv, s->ldv, s->dtype); }
    Area o(const void *p) const { return row_area(p, n, (int64_t)s->heads * s->dv, s->ldo, s->dtype); }
    Area decay(const void *p) const { return flat_area(p, 4 * (int64_t)s->heads); }
    Area states(const void *p, int64_t count, int same = 0) const {
        return Area{p, 1, count * state, count * state, same};
    }
};

nsd_status launch(Kind kind, const nsd_decay *s, const Scan &a, hipStream_t st) {
    return s->dtype == NSD_F32 ? launch_scan_f32(kind, a, st) : launch_scan_bf16(kind, a, st);
}

// What every scan of a call has in common.
Scan base_scan(int32_t ntok, int32_t nseq, const int32_t *seqptr, const nsd_decay *s,
               const float *decay, const DecayWs &w) {
    Scan a{};
    a.ntok = ntok;
    a.nseq = nseq;
    a.H = s->heads;
    a.seqptr = seqptr;
    a.seg_len = w.seg_len;
    a.nseg = w.nseg;
    a.decay = decay;
    a.per = (int64_t)s->d * s->dv;
    return a;
}

// The states that segments start from: at `states` after the scan of every segment by itself and
// the join, or (whole sequences) the sequences' own.  `end`: the states behind the sequences.
nsd_status segment_states(const nsd_decay *s, const DecayWs &w, Scan a, const Rows &k, const Rows &v,
                          bool rev, float s_update, float *states, const float *start, float *end,
                          hipStream_t st) {
    if (!w.cut()) return NSD_OK;
    a.k = k;
    a.v = v;
    a.rev = rev;
    a.s_update = s_update;
    a.sk = s->dv;
    a.sv = 1;
    a.end = states;
    NSD_TRY(launch(kState, s, a, st));
    return join(a, rev, states, start, end, st);
}

// A scan's start from the segments' states or the sequences' own.
void starts(Scan &a, const DecayWs &w, const float *states, const float *start) {
    a.start = w.cut() ? states : start;
    a.start_by_seq = !w.cut();
}

}  // namespace

}  // namespace decay
}  // namespace nsd

using namespace nsd;
using namespace nsd::decay;

extern "C" {

nsd_status nsd_attn_decay_workspace_size(int32_t ntok, int32_t nseq, int32_t max_len,
                                         const nsd_decay *s, int32_t gradient, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_TRY(check_sizes(ntok, nseq, max_len, s));
    *bytes = DecayWs(nullptr, ntok, nseq, max_len, s, gradient != 0, true).bytes;
    return NSD_OK;
}

nsd_status nsd_attn_decay(int32_t ntok, int32_t nseq, const int32_t *seqptr, int32_t max_len,
                          const nsd_decay *s, const void *Q, const void *K, const void *V,
                          const float *decay, const float *S0, void *O, float *S1, void *ws,
                          size_t ws_bytes, void *stream) {
    NSD_TRY(check_sizes(ntok, nseq, max_len, s));
    if (nseq == 0) return NSD_OK;
    NSD_REQUIRE(seqptr && decay && (ntok == 0 || (Q && K && V && O)), "a NULL array");
    const DecayWs w(ws, ntok, nseq, max_len, s, false);
    if (ws == nullptr || ws_bytes < w.bytes)
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, w.bytes);
    NSD_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    const Areas of{ntok, s};
    NSD_TRY(check_apart({of.o(O), of.states(S1, nseq, 1), flat_area(ws, w.bytes)},
                        {of.q(Q), of.k(K), of.v(V), of.decay(decay), of.states(S0, nseq, 1),
                         flat_area(seqptr, 4 * ((int64_t)nseq + 1))}));
    const hipStream_t st = as_stream(stream);
    const int grp = s->heads / s->kv_heads;
    const Rows q{Q, s->ldq, s->d, 1}, k{K, s->ldk, s->d, grp}, v{V, s->ldv, s->dv, grp};
    Scan a = base_scan(ntok, nseq, seqptr, s, decay, w);
    NSD_TRY(segment_states(s, w, a, k, v, false, 1.f, w.forth, S0, S1, st));
    a.q = q;
    a.k = k;
    a.v = v;
    a.out = O;
    a.ldo = s->ldo;
    a.s_score = a.s_inter = s->scale;
    a.s_update = 1.f;
    a.sk = s->dv;
    a.sv = 1;
    starts(a, w, w.forth, S0);
    a.end = w.cut() ? nullptr : S1;
    a.end_by_seq = true;
    return launch(kOutput, s, a, st);
}

nsd_status nsd_attn_decay_vjp(int32_t ntok, int32_t nseq, const int32_t *seqptr, int32_t max_len,
                              const nsd_decay *s, const void *Q, const void *K, const void *V,
                              const float *decay, const float *S0, const void *dO,
                              const float *dS1, void *dQ, void *dK, void *dV, float *ddecay,
                              float *dS0, void *ws, size_t ws_bytes, void *stream) {
    NSD_TRY(check_sizes(ntok, nseq, max_len, s));
    NSD_REQUIRE(nseq == 0 || (seqptr && decay && (ntok == 0 || (Q && K && V && dO && dQ && dK && dV))),
                "a NULL array");
    const DecayWs w(ws, ntok, nseq, max_len, s, true);
    if (ws == nullptr || ws_bytes < w.bytes)
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, w.bytes);
    NSD_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    const Areas of{nseq > 0 ? ntok : 0, s};
    NSD_TRY(check_apart({of.q(dQ), of.k(dK), of.v(dV), of.decay(ddecay), of.states(dS0, nseq),
                         flat_area(ws, w.bytes)},
                        {of.q(Q), of.k(K), of.v(V), of.o(dO), of.decay(nseq > 0 ? decay : nullptr),
                         of.states(S0, nseq), of.states(dS1, nseq),
                         flat_area(nseq > 0 ? seqptr : nullptr, 4 * ((int64_t)nseq + 1))}));
    const hipStream_t st = as_stream(stream);
    const int grp = s->heads / s->kv_heads;
    if (nseq > 0) {
        const Rows q{Q, s->ldq, s->d, 1}, k{K, s->ldk, s->d, grp}, v{V, s->ldv, s->dv, grp},
            up{dO, s->ldo, s->dv, 1};
        const Scan common = base_scan(ntok, nseq, seqptr, s, decay, w);
        // S forwards from S0, and R backwards from dS1, to S0's gradient
        NSD_TRY(segment_states(s, w, common, k, v, false, 1.f, w.forth, S0, nullptr, st));
        NSD_TRY(segment_states(s, w, common, q, up, true, s->scale, w.back, dS1, dS0, st));
        // The gradient of the decay goes with the scan whose states' columns are the wider side:
        // its state's derivative is held by fewer rows for each wave.
        auto with_decay = [&](Scan &a, bool here, const Rows &rows, const float *meets,
                              const float *ends) {
            if (!ddecay || !here) return kOutput;
            a.up = rows;
            a.back = w.cut() ? meets : ends;
            a.back_by_seq = !w.cut();
            a.sums = w.sums;
            return kDerivative;
        };
        Scan a = common;  // dq: the states transposed
        a.q = up;
        a.k = v;
        a.v = k;
        a.out = dQ;
        a.ldo = s->ldq;
        a.s_score = a.s_inter = s->scale;
        a.s_update = 1.f;
        a.sk = 1;
        a.sv = s->dv;
        starts(a, w, w.forth, S0);
        NSD_TRY(launch(with_decay(a, s->dv < s->d, q, w.back, dS1), s, a, st));
        a = common;  // dk
        a.rev = true;
        a.q = Rows{V, s->ldv, s->dv, grp};
        a.k = up;
        a.v = q;
        a.out = grp > 1 ? (void *)w.dk : dK;
        a.out32 = grp > 1;
        a.ldo = grp > 1 ? (int64_t)s->heads * s->d : s->ldk;
        a.s_score = a.s_update = s->scale;
        a.s_inter = 1.f;
        a.sk = 1;
        a.sv = s->dv;
        starts(a, w, w.back, dS1);
        NSD_TRY(launch(kOutput, s, a, st));
        a = common;  // dv
        a.rev = true;
        a.q = k;
        a.k = q;
        a.v = up;
        a.out = grp > 1 ? (void *)w.dv : dV;
        a.out32 = grp > 1;
        a.ldo = grp > 1 ? (int64_t)s->heads * s->dv : s->ldv;
        a.s_score = a.s_update = s->scale;
        a.s_inter = 1.f;
        a.sk = s->dv;
        a.sv = 1;
        starts(a, w, w.back, dS1);
        a.end = w.cut() ? nullptr : dS0;
        a.end_by_seq = true;
        NSD_TRY(launch(with_decay(a, s->d <= s->dv, v, w.forth, S0), s, a, st));
        if (grp > 1 && ntok > 0) {
            const unsigned blocks = (unsigned)std::min(ntok, 1 << 16);
            auto sum = [&](auto t) {
                using T = decltype(t);
                decay_heads_kernel<T><<<blocks, kSumThreads, 0, st>>>(
                    ntok, nseq, seqptr, s->kv_heads, grp, s->d, w.dk, static_cast<T *>(dK), s->ldk);
                decay_heads_kernel<T><<<blocks, kSumThreads, 0, st>>>(
                    ntok, nseq, seqptr, s->kv_heads, grp, s->dv, w.dv, static_cast<T *>(dV), s->ldv);
            };
            if (s->dtype == NSD_F32) sum(float());
            else sum(Bf16());
            NSD_TRY(check_launch("decay_heads_kernel"));
        }
    }
    if (ddecay == nullptr) return NSD_OK;
    decay_sums_kernel<<<s->heads, kSumThreads, 0, st>>>(nseq > 0 ? w.nseg : 0, s->heads, w.nvb, w.sums,
                                                       ddecay);
    return check_launch("decay_sums_kernel");
}

nsd_status nsd_attn_decay_step(int32_t nrows, const int32_t *slot, int32_t nslots,
                               const nsd_decay *s, const void *Q, const void *K, const void *V,
                               const float *decay, float *state, void *O, void *stream) {
    NSD_TRY(check_decay(s));
    NSD_REQUIRE(nrows >= 0 && nslots >= 0, "a negative size");
    if (nrows == 0) return NSD_OK;
    NSD_REQUIRE(Q && K && V && decay && O && (state || nslots == 0), "a NULL array");
    NSD_REQUIRE(slot || nrows <= nslots, "%d rows over %d states", nrows, nslots);
    const Areas of{nrows, s};
    NSD_TRY(check_apart({of.o(O), of.states(state, nslots)},
                        {of.q(Q), of.k(K), of.v(V), of.decay(decay), flat_area(slot, 4 * (int64_t)nrows)}));
    Step a{nrows, nslots, s->heads, s->heads / s->kv_heads, s->d, s->dv, 0, s->scale, slot, Q, K, V,
           s->ldq, s->ldk, s->ldv, s->ldo, decay, state, O};
    const bool four = s->dv % 4 == 0;
    // Lanes over a state's row: 128 columns a block, fewer where that leaves too few blocks (4
    // rows of 16 heads of 64 by 128: 5.1 us, with 128 columns 5.5; 16 rows: 6.1 with 64 columns,
    // 5.7 with 128).
    int cols = 128;
    while (cols > 32 && (int64_t)nrows * s->heads * ceil_div(s->dv, cols) < 256) cols /= 2;
    while (cols / 2 >= s->dv && cols > 32) cols /= 2;
    a.lanes = four ? cols / 4 : cols;
    const int64_t blocks = (int64_t)nrows * s->heads * ceil_div(s->dv, cols);
    if (blocks > UINT32_MAX / kStepThreads)
        return fail(NSD_ERR_TOO_LARGE, "%d rows of %d heads", nrows, s->heads);
    auto run = [&](auto t) {
        using T = decltype(t);
        if (four) decay_step_kernel<T, 4><<<blocks, kStepThreads, 0, as_stream(stream)>>>(a);
        else decay_step_kernel<T, 1><<<blocks, kStepThreads, 0, as_stream(stream)>>>(a);
    };
    if (s->dtype == NSD_F32) run(float());
    else run(Bf16());
    return check_launch("decay_step_kernel");
}

}  // extern "C"
