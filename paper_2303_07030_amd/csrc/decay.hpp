// Linear attention with a decay for each head: the scan over chunks of tokens that its
// forward pass and every gradient run, on the matrix cores.
//
//   S_t = e^g S_{t-1} + k_t^T v_t,   o_t = s q_t S_t
//
// A chunk of C tokens, with S the state before it, n = i - j and w = e^g:
//   O = [ s w^(i+1) Q S ] + [ s w^n (Q K^T) for n >= 0 ] V,
//   S = w^C S + (w^(C-1-j) K)^T V
// The gradients are the same scan with the roles changed.  With R the state that comes
// back from the tokens behind (R_t = w R_{t+1} + s q_t^T do_t):
//   dq: queries dO, keys V, values K, states S^T;   forwards
//   dk: queries V, keys dO, values Q, states R^T;   backwards
//   dv: queries K, keys Q, values dO, states R;     backwards
// (backwards, the state is held with its next decay in it, so that the state of no
// token is the upstream of the last state: powers i and C - j instead of i + 1 and
// C - 1 - j).  The gradient of g is the sum of do_t times the derivative of o_t, or of v_t
// times that of dv_t, or of q_t times that of dq_t: whichever scan is run, the
// derivative T of its state goes along,
//   d/dg: weights n w^n,  s w^(i+1) ((i+1) Q S + Q T);   T = w^C (T + C S) + sum
//   (C-1-j) w^(C-1-j) k^T v
// and what the segment's last T adds to what meets it from the other side is added.
//
// A block of four or eight waves takes a segment of a sequence, a head and 64 or 128
// columns of the values, 16 a wave.  A wave's own columns of the state stay in its
// registers, in 32 bits, in the layout that the products leave and, with the
// contraction's order within 32 places permuted (place() below), the next product
// takes.  Queries, keys (both ways round), transposed values and the scores are shared
// through LDS; the next chunk's rows are in flight meanwhile.
//
// bf16: products of bf16 rows are exact, and what is not a bf16 number (scores, states,
// decayed values) is a sum of three of them, 24 bits, as many as a 32-bit float has: the
// results are those of products in 32 bits.  fp32: fp32 products, half the chunk.
//
// A prompt of 65,536 tokens of 8 heads of 128 by 128 in bf16: the states 90 us, the outputs 220
// (2.4 TB/s of the rows' bytes).  Neither bytes nor products bound it alone: the vector units issue in
// 59% of the cycles (the parts of states and values, rows turned for LDS), the matrix cores are
// busy in 32%, and two blocks a CU do not lay the one over the other whole; of LDS's cycles 4%
// are conflicts.  A training step of 32,768 tokens of 16 heads of 64 by 128: states 68 us,
// outputs 172, dq and dk 146 each, dv with the gradient of g 295 (57% and 24%: two states leave
// three blocks of four waves a CU).
#pragma once

#include <type_traits>

#include "values.hpp"

namespace nsd {
namespace decay {

constexpr int kMaxWidth = 256;

template <class T>
constexpr int kChunkOf = sizeof(T) == 2 ? 64 : 32;

// One of the rows' matrices: head h of a query head is at (h / grp) * width.
struct Rows {
    const void *p;
    int64_t ld;
    int32_t width, grp;
};

struct Scan {
    int32_t ntok, nseq, H;
    const int32_t *seqptr;
    int32_t seg_len;          // tokens of a segment
    int32_t nseg;             // segment numbers there are (some of no tokens)
    Rows q, k, v;
    void *out;                // [ntok][..]: head h at h * v.width
    int64_t ldo;
    bool out32;               // a float for each query head, to be added up
    bool rev;
    float s_score, s_inter, s_update;
    const float *decay;       // g [H]
    // states [index][H][per], element (k, v) at k * sk + v * sv
    const float *start;       // NULL: zero
    float *end;               // NULL: not wanted
    bool start_by_seq, end_by_seq;
    int32_t sk, sv;
    int64_t per;
    // gradient of g: the rows that the outputs' derivatives meet, the states from the other side
    // that meet a segment's last one's, one sum for each block
    Rows up;
    const float *back;
    bool back_by_seq;
    float *sums;
};

// Segment `id`: sequence s has the numbers from seqptr[s] / seg_len + s on, which are enough for
// it whatever the lengths; those it does not need have no tokens.
struct Segment {
    int32_t seq, first, n;  // its first token and its tokens (0: none)
    bool on;                // it is one: also the first of an empty sequence
    __device__ __forceinline__ Segment(const Scan &a, int id) {
        int lo = 0, hi = a.nseq - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (max(a.seqptr[mid], 0) / a.seg_len + mid <= id) lo = mid;
            else hi = mid - 1;
        }
        seq = lo;
        const int begin = max(a.seqptr[lo], 0), end = min(a.seqptr[lo + 1], a.ntok);
        const int c = id - (begin / a.seg_len + lo);
        const int64_t at = begin + (int64_t)c * a.seg_len;
        on = c == 0 || (c > 0 && at < end);
        first = (int)min(at, (int64_t)a.ntok);
        n = on ? (int)max(min((int64_t)end - at, (int64_t)a.seg_len), (int64_t)0) : 0;
    }
};

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));

// Eight values of a lane: places of 32 of the contraction, of row (lane % 16).
template <class T>
struct Frag;
template <>
struct Frag<Bf16> {
    u32x4v v;
};
template <>
struct Frag<float> {
    float v[8];
};

template <class T>
__device__ __forceinline__ Frag<T> fragment(const T *p) {
    Frag<T> f;
    __builtin_memcpy(&f, __builtin_assume_aligned(p, 16), sizeof f);
    return f;
}

// c[4 g + r][n] += sum of a[4 g + r][.] b[n][.]: rows of a in the lane's four values, the row
// of b by lane % 16.
__device__ __forceinline__ void mma(f32x4v &c, const Frag<Bf16> &a, const Frag<Bf16> &b) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, a.v),
                                                __builtin_bit_cast(bf16x8v, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x4v &c, const Frag<float> &a, const Frag<float> &b) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
}

// x as a sum of N numbers of T (one is enough in 32 bits).
template <class T, int N>
constexpr int kParts = sizeof(T) == 2 ? N : 1;

// The parts but the last are cut, not rounded: an upper half is a bf16 number as it stands,
// what is left is exact, and eight bits of 24 are gone with each.
template <class T, int N, int M>
__device__ __forceinline__ void split(const float (&x)[M], T (&part)[kParts<T, N>][M]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < M; ++e) part[0][e] = x[e];
    } else {
        float left[M];
#pragma unroll
        for (int e = 0; e < M; ++e) left[e] = x[e];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t pair[M / 2];
#pragma unroll
            for (int e = 0; e < M; e += 2) {
                if (i + 1 < N) {
                    const uint32_t a = __float_as_uint(left[e]), b = __float_as_uint(left[e + 1]);
                    pair[e / 2] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                    left[e] -= __uint_as_float(a & 0xFFFF0000u);
                    left[e + 1] -= __uint_as_float(b & 0xFFFF0000u);
                } else {
                    const Bf16 two[2] = {narrowed<Bf16>(left[e]), narrowed<Bf16>(left[e + 1])};
                    __builtin_memcpy(&pair[e / 2], two, 4);
                }
            }
            __builtin_memcpy(part[i], pair, sizeof pair);
        }
    }
}
template <class T, int N>
__device__ __forceinline__ void split(const float (&x)[8], Frag<T> (&f)[kParts<T, N>]) {
    T part[kParts<T, N>][8];
    split<T, N, 8>(x, part);
#pragma unroll
    for (int i = 0; i < kParts<T, N>; ++i) __builtin_memcpy(&f[i], part[i], sizeof f[i]);
}

// Where value k of a row lies in LDS, k a multiple of four: of 32 values lane group g takes 4 g
// to 4 g + 3 and 16 + 4 g to 16 + 4 g + 3, as the products leave a state's rows.
__device__ __forceinline__ int place(int k) {
    const int u = k % 32 / 4;
    return k / 32 * 32 + (u % 4) * 8 + (u / 4) * 4;
}

// Banks.  LDS has 64 of them; a read of 16 bytes a lane takes lanes 0-3, 12-15, 20-27 at once,
// then 4-11, 16-19, 28-31, and so on (found by counting conflicts over row distances), a write
// of 8 bytes 16 consecutive lanes over half of them.  The 16 bytes of a row that a lane
// group reads are therefore turned by bits of the row's number, so that neither reads
// nor writes (Stage's) of bf16 meet: of the cycles of LDS none are conflicts in scans of states,
// 4 to 7% in those of outputs and 13% where the scores are SHORT (45% without it, in outputs).

// Of rows by token, KD values and 16 bytes apart.
template <class T>
__device__ __forceinline__ int turned(int row) {
    return sizeof(T) == 2 ? ((row >> 2 ^ row >> 3) & 1) * 8 : 0;
}

// Place j of row `row` of rows of C places (128 bytes).
template <class T>
__device__ __forceinline__ int spread(int row, int j) {
    constexpr int B = 16 / sizeof(T);
    const int x = sizeof(T) == 2 ? (row >> 2 & 1) | ((row >> 1 ^ row >> 2) & 2) | ((row << 1 ^ row >> 2) & 4)
                                 : row >> 1 & 7;
    return row * kChunkOf<T> + ((j / B ^ x) * B | j % B);
}

// Place of the score of row i and column j.  SHORT (of bf16): rows of 32 places, the columns from
// 32 on, which have rows from 32 on alone, behind the others; a quarter less, but two writes meet
// on a bank.
template <class T, bool SHORT>
__device__ __forceinline__ int score_place(int i, int j) {
    if constexpr (!SHORT) {
        return spread<T>(i, j);
    } else {
        const int row = i + (j & 32), u = row >> 2 & 3;
        return row * 32 + ((j >> 3 & 3) ^ u ^ (u << 1 & 2)) * 8 + (j & 7);
    }
}
template <class T, bool SHORT>
constexpr int kScores = SHORT ? 96 * 32 : kChunkOf<T> * kChunkOf<T>;

// A lane's fragments of rows of C places: row 16 tile + lane % 16, places 32 f + 8 (lane / 16) on.
// Two addresses for all of them, the rest known at compile time (or the same for all lanes).
template <class T>
struct Spread {
    const T *p;
    int other;  // bf16: of odd f + tile; fp32: of the second half of the places
    __device__ __forceinline__ Spread(const T *rows, int n16, int g)
        : p(rows + spread<T>(n16, 8 * g)),
          other(spread<T>(n16, 8 * g + (sizeof(T) == 2 ? 32 : 4)) - spread<T>(n16, 8 * g)) {}
    __device__ __forceinline__ Frag<T> at(int tile, int f) const {
        Frag<T> x;
        const int off = tile * 16 * kChunkOf<T>;
#pragma unroll
        for (int b = 0; b < (int)sizeof(T) / 2; ++b) {
            const bool odd = sizeof(T) == 2 ? (f ^ tile) & 1 : b;
            __builtin_memcpy(reinterpret_cast<char *>(&x) + 16 * b,
                             __builtin_assume_aligned(p + off + (odd ? other : 0), 16), 16);
        }
        return x;
    }
};

// The same of SHORT scores, part after part.
struct ShortScores {
    const Bf16 *p;
    __device__ __forceinline__ ShortScores(const Bf16 *scores, int n16, int g)
        : p(scores + score_place<Bf16, true>(n16, 8 * g)) {}
    __device__ __forceinline__ Frag<Bf16> at(int tile, int f) const {
        return fragment(p + tile / 4 * kScores<Bf16, true> + (16 * (tile % 4) + 32 * f) * 32);
    }
};

// A chunk's rows of one matrix on their way to LDS: four rows and four columns a unit.
// TAIL: the rows' widths are no multiples of four.
template <class T, int W, int THREADS, bool TAIL>
struct Stage {
    static constexpr int C = kChunkOf<T>;
    static constexpr int CV = 4;
    static constexpr int PIECES = W / CV;
    static constexpr int UNITS = C / 4 * PIECES;
    static constexpr int U = (UNITS + THREADS - 1) / THREADS;
    static constexpr bool EXACT = UNITS % THREADS == 0;
    static constexpr int WD = CV * sizeof(T) / 4;
    uint32_t x[U][4][WD];  // as they were loaded: nothing waits for them before clear()

    // (threads beyond the units repeat the last one, and store nothing)
    static __device__ __forceinline__ int unit(int tid, int u) {
        const int n = tid + u * THREADS;
        return EXACT ? n : min(n, UNITS - 1);
    }
    // (neighbouring lanes take either half of the same eight rows)
    static __device__ __forceinline__ int row_of(int n) { return (n / (2 * PIECES) * 2 + n % 2) * 4; }
    // Rows i < len (at least one) from token t0 on, or back; columns from col0 on.  Nothing here
    // depends on a lane's place: what is beyond a row or the chunk reads a neighbour of it,
    // and is cleared by clear().  A whole chunk's four rows have one place and four bases.
    __device__ __forceinline__ void load(int tid, const Rows &m, int h, int col0, int64_t t0, bool rev, int len) {
        const char *base = reinterpret_cast<const char *>(
            static_cast<const T *>(m.p) + (rev ? t0 - (len - 1) : t0) * m.ld +
            (int64_t)(h / m.grp) * m.width + col0);
        const int width = m.width - col0;
        const uint32_t row = (uint32_t)m.ld * sizeof(T);  // bytes
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i0 = row_of(unit(tid, u)), c = unit(tid, u) / 2 % PIECES * CV;
            if (!TAIL && len == C) {
                const uint32_t at = (uint32_t)(rev ? C - 4 - i0 : i0) * row + min(c, width - CV) * sizeof(T);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    __builtin_memcpy(x[u][r], base + (uint64_t)((uint32_t)(rev ? 3 - r : r) * row) + at, sizeof x[u][r]);
                continue;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = min(i0 + r, len - 1);
                const uint32_t at = (uint32_t)(rev ? len - 1 - i : i) * row;
                if constexpr (!TAIL) {
                    __builtin_memcpy(x[u][r], base + (at + min(c, width - CV) * sizeof(T)), sizeof x[u][r]);
                } else {
                    T t[CV];
#pragma unroll
                    for (int e = 0; e < CV; ++e)
                        __builtin_memcpy(&t[e], base + (at + min(c + e, width - 1) * sizeof(T)), sizeof(T));
                    __builtin_memcpy(x[u][r], t, sizeof t);
                }
            }
        }
    }
    __device__ __forceinline__ void clear(int tid, int width, int len) {
        if (len == C && width >= W) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i0 = row_of(unit(tid, u)), c = unit(tid, u) / 2 % PIECES * CV;
#pragma unroll
            for (int d = 0; d < WD; ++d) {
                const int e = TAIL ? c + d * (CV / WD) : c;  // the first value of the four bytes
                uint32_t keep = e < width ? ~0u : 0u;
                if (TAIL && sizeof(T) == 2 && e + 1 == width) keep = 0xFFFFu;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[u][r][d] &= i0 + r < len ? keep : 0u;
            }
        }
    }
    // rows of ld values, columns in the order of place()
    __device__ __forceinline__ void store(int tid, T *to, int ld) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!EXACT && tid + u * THREADS >= UNITS) continue;
            const int i0 = row_of(unit(tid, u)), c = unit(tid, u) / 2 % PIECES * CV;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                __builtin_memcpy(__builtin_assume_aligned(to + i0 * ld + (place(c) ^ turned<T>(i0)) + r * ld, 8), x[u][r],
                                 sizeof x[u][r]);
        }
    }
    // columns as rows of C places
    __device__ __forceinline__ void store_transposed(int tid, T *to) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!EXACT && tid + u * THREADS >= UNITS) continue;
            const int i0 = row_of(unit(tid, u)), c = unit(tid, u) / 2 % PIECES * CV;
            // (two columns of a multiple of four keep their 16 bytes' places, the others turn one bit)
            T *const at[2] = {to + spread<T>(c, i0), to + spread<T>(c + 2, i0) - 2 * C};
#pragma unroll
            for (int e = 0; e < CV; ++e) {
                uint32_t t[WD];
                if constexpr (sizeof(T) == 2) {
                    const uint32_t half = e % 2 ? 0x07060302u : 0x05040100u;
                    t[0] = __builtin_amdgcn_perm(x[u][1][e / 2], x[u][0][e / 2], half);
                    t[1] = __builtin_amdgcn_perm(x[u][3][e / 2], x[u][2][e / 2], half);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) t[r] = x[u][r][e];
                }
                __builtin_memcpy(__builtin_assume_aligned(at[e / 2] + e * C, 8), t, sizeof t);
            }
        }
    }
    __device__ __forceinline__ bool finite() const {
        bool all = true;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int d = 0; d < WD; ++d) {
                if constexpr (sizeof(T) == 4) {
                    uint32_t top = 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = max(top, x[u][r][d] & 0x7F800000u);
                    all = all && top < 0x7F800000u;
                } else {
                    typedef uint16_t two __attribute__((ext_vector_type(2)));
                    two top = {0, 0};
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        top = __builtin_elementwise_max(top, __builtin_bit_cast(two, x[u][r][d] & 0x7F807F80u));
                    all = all && top.x < 0x7F80 && top.y < 0x7F80;
                }
            }
        return all;
    }
};

// What a scan does: outputs; the states at the segments' ends alone; outputs and the gradient
// of g.
enum Kind { kOutput, kState, kDerivative };

// LDS of a block: queries, keys (the scores take their place; DERIV's parts the queries' as well),
// keys and values by columns.
template <class T, int KD, int NW, Kind KIND>
struct Shared {
    static constexpr int C = kChunkOf<T>;
    static constexpr int VB = NW * 16;
    static constexpr int LDK = KD + 16 / sizeof(T);
    static constexpr int OP = kParts<T, 3>;  // parts of scores; behind them those of DERIV's
    static constexpr int SP = KIND == kDerivative ? 2 * OP : OP;
    static constexpr int Q = KIND == kState ? 0 : C * LDK;
    static constexpr bool SHORT = KIND == kDerivative && sizeof(T) == 2;
    static constexpr int AT = KIND == kDerivative ? 0 : Q;  // where the scores are put
    static constexpr int PART = kScores<T, SHORT>;
    // Blocks of four waves take their values from LDS before the scores are put there, over keys
    // and values: three blocks a CU have room for the scores' parts.
    static constexpr bool OVER = KIND != kState && NW == 4;
    static constexpr int QKV = 2 * Q + (OVER ? VB * C : 0);
    static constexpr int ROWS = KIND == kState ? 0 : QKV > AT + SP * PART ? QKV : AT + SP * PART;
    // Wide keys by columns take the queries' place when those were read: three blocks of four waves
    // a CU instead of two (a training step, whose dq and dk have keys of 128, 1,019 us for 1,065).
    static constexpr bool LATE = KIND == kOutput && NW == 4 && KD > 64;
    static_assert(!LATE || KD * C <= Q, "keys by columns in the queries' place");
    static constexpr int KT_END = ROWS + (LATE ? 0 : KD * C);
    static constexpr int V = OVER ? 2 * Q : KT_END;
    static constexpr int VALUES = OVER ? KT_END : KT_END + VB * C;
};

// Waves of a SIMD, which say how many registers one may have: two blocks of eight waves a CU
// where the state leaves room for it (a prompt 334 us, with one block 398; a training step 1,019
// and 1,050, one of 5,003 tokens in fp32 182 and 195), three of four waves with the gradient of g
// in bf16 (the step 1,019 us, with two 1,105) and where wide keys leave them the LDS.
constexpr int waves_of(int kd, int nw, Kind kind) {
    const bool two_states = kind == kDerivative;
    if (kd > 128) return 1;
    if (nw == 4) return two_states == (kd <= 64) ? 3 : 2;
    return two_states && kd > 64 ? 2 : 4;
}

// KD: width of queries and keys, padded; NW: waves, 16 columns of the values each; blocks: of
// the segments' heads' columns, nvb for each head.
template <class T, int KD, int NW, Kind KIND, bool TAIL>
__global__ __launch_bounds__(NW * kWave, waves_of(KD, NW, KIND)) void scan_kernel(Scan a, int32_t nvb) {
    using Sh = Shared<T, KD, NW, KIND>;
    constexpr int C = Sh::C, VB = Sh::VB, LDK = Sh::LDK;
    constexpr int KT = KD / 16, KF = KD / 32, IT = C / 16, JF = C / 32;
    constexpr int OP = Sh::OP, SP = Sh::SP, NP = kParts<T, 3>;
    constexpr bool DERIV = KIND == kDerivative;
    constexpr int GR = KT < IT ? KT : IT;  // rows of the state that a step of their products takes
    __shared__ __align__(16) T lds[Sh::VALUES];
    T *const ldsQ = lds;
    T *const ldsK = ldsQ + Sh::Q;
    T *const ldsP = lds + Sh::AT;
    constexpr bool LATE = Sh::LATE;
    T *const ldsKt = LATE ? lds : lds + Sh::ROWS;
    T *const ldsVt = lds + Sh::V;
    __shared__ float power[C + 2], power_less[C + 2];
    __shared__ float weight[2 * C];  // s_score w^n at C + n, 0 below C
    __shared__ __align__(16) float behind[2 * C];  // s_update w^(C - 1 - j (+ 1)) at j, 0 from C on
    // A byte for each wave, not 0 where it staged a value that is not finite.  Its wave writes it
    // for every chunk, so that nothing clears it; between the others' reads of one chunk's and
    // the next write lies the barrier at the chunk's end.
    __shared__ __align__(8) uint8_t unusual[NW];
    __shared__ float wave_sum[NW];

    const int lane = threadIdx.x % kWave, n16 = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int unit = (int)xcd_contiguous_tile();
    const int vb = unit % nvb, h = unit / nvb % a.H, id = unit / nvb / a.H;
    const Segment seg(a, id);
    if (!seg.on) {
        if (DERIV && threadIdx.x == 0) a.sums[unit] = 0.f;
        return;
    }
    const int rev = a.rev ? 1 : 0;
    const int col0 = vb * VB, colw = wave * 16;  // first columns: the block's; the wave's in it
    if (threadIdx.x < C + 2) {
        // Powers of the decay, and what they are less than 1: near 1 the roundings of a power
        // itself would add up over the thousands of chunks that multiply it.
        const int n = threadIdx.x;
        const double x = n ? exp((double)a.decay[h] * (double)n) : 1.0;
        power[n] = (float)x;
        power_less[n] = (float)(x - 1.0);
        if (n >= rev && n < C + rev) behind[C - 1 + rev - n] = a.s_update * (float)x;
        if (n < C) {
            behind[C + n] = weight[n] = 0.f;
            weight[C + n] = a.s_score * (float)x;
        }
    }
    // this lane's part of the state: rows 16 kt + 4 g + r, column n16 of the wave's
    f32x4v S[KT], D[KT];  // (D: of DERIV alone)
    auto each_state = [&](const float *from, bool by_seq, auto f) {
        const float *const p = from + ((int64_t)(by_seq ? seg.seq : id) * a.H + h) * a.per;
        const int c = col0 + colw + n16;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int k = 16 * kt + 4 * g + r;
                const uint32_t at = (uint32_t)(min(k, a.k.width - 1) * a.sk + min(c, a.v.width - 1) * a.sv);
                f(kt, r, k < a.k.width && c < a.v.width, p + at);
            }
    };
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        S[kt] = f32x4v{0.f, 0.f, 0.f, 0.f};
        if (DERIV) D[kt] = f32x4v{0.f, 0.f, 0.f, 0.f};
    }
    if (a.start)
        each_state(a.start, a.start_by_seq, [&](int kt, int r, bool in, const float *p) {
            const float x = *p;
            S[kt][r] = in ? x : 0.f;
        });

    Stage<T, KD, NW * kWave, TAIL> xq, xk;
    Stage<T, VB, NW * kWave, TAIL> xv;
    const int64_t first = rev ? (int64_t)seg.first + seg.n - 1 : seg.first;
    const int dir = rev ? -1 : 1;
    float dsum = 0.f;
    int single = 0;  // tokens that are still taken one by one
    int pos = 0, len = 0, next = 0, next_len = min(C, seg.n);
    // States alone leave registers for the next chunk's rows, on their way while one is multiplied
    // (128 by 128, a prompt: 94 us, 102 without).  Other scans have the other blocks of a CU to
    // hide them: with outputs' rows ahead as well a prompt took 384 us in place of 334, a
    // training step 1,050 in place of 1,013, and keys of up to 64 gained nothing by them (1,019 and
    // 1,013; 8,192 tokens of 8 heads of 64 by 128 in fp32, forwards: 103 and 91).
    constexpr bool AHEAD = KIND == kState;
    auto load = [&](int tid) {
        const int64_t t0 = first + (int64_t)next * dir;
        if (KIND != kState) xq.load(tid, a.q, h, 0, t0, a.rev, next_len);
        xk.load(tid, a.k, h, 0, t0, a.rev, next_len);
        xv.load(tid, a.v, h, col0, t0, a.rev, next_len);
    };
    for (;;) {
        // What follows from the thread's number is found again for each chunk: kept across the
        // loop it would take more registers than the state.
        int tid = threadIdx.x;
        opaque(tid);
        if (AHEAD && next < seg.n) load(tid);
        if (len > 0) {
            const int n16 = tid % 16, g = tid % kWave / 16;
            // this lane's places in what the products read: all others are a constant from them
            const Spread<T> by_k(ldsKt, n16, g), by_v(ldsVt, n16, g);
            const std::conditional_t<Sh::SHORT, ShortScores, Spread<T>> by_p(ldsP, n16, g);
            const T *const byQ = ldsQ + n16 * LDK + (8 * g ^ turned<T>(n16));
            const T *const byK = byQ + (ldsK - ldsQ);

            Frag<T> vf[JF];  // the wave's columns of the values
            auto take_values = [&]() {
#pragma unroll
                for (int f = 0; f < JF; ++f) vf[f] = by_v.at(wave, f);
            };
            f32x4v O[IT], E[IT];  // (E: of DERIV, the outputs' derivatives)
            if constexpr (KIND != kState) {
                // ---- scores: tile (it, jt) of 16 x 16, jt <= it, shared out among the waves
                constexpr int TILES = IT * (IT + 1) / 2;
                constexpr int ROUNDS = (TILES + NW - 1) / NW;
                float p[ROUNDS][4];
                auto it_of = [](int t) { return t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0; };
                const int apart = n16 - 4 * g;  // of the lane's row and its first column in a tile
#pragma unroll
                for (int u = 0; u < ROUNDS; ++u) {
                    const int tile = u * NW + wave, it = it_of(tile), jt = tile - it * (it + 1) / 2;
                    if (tile >= TILES) break;
                    f32x4v acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int f = 0; f < KF; ++f)
                        mma(acc, fragment(byK + 16 * jt * LDK + 32 * f), fragment(byQ + 16 * it * LDK + 32 * f));
                    const float *const w = weight + C + 16 * (it - jt) + apart;
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[u][r] = acc[r] * w[-r];
                    if (it == jt)  // later tokens: 0, whatever their products are
#pragma unroll
                        for (int r = 0; r < 4; ++r) p[u][r] = apart >= r ? p[u][r] : 0.f;
                }
                // ---- from the state
                auto from_state = [&](const f32x4v (&state)[KT], f32x4v (&O)[IT]) {
#pragma unroll
                    for (int f = 0; f < KF; ++f) {
                        Frag<T> qf[IT];
#pragma unroll
                        for (int it = 0; it < IT; ++it) qf[it] = fragment(byQ + 16 * it * LDK + 32 * f);
                        Frag<T> sf[NP];
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = state[2 * f + e / 4][e % 4];
                        split<T, 3>(x, sf);
#pragma unroll
                        for (int s = 0; s < NP; ++s)
#pragma unroll
                            for (int it = 0; it < IT; ++it) mma(O[it], sf[s], qf[it]);
                    }
                };
                if constexpr (DERIV || LATE) {
#pragma unroll
                    for (int it = 0; it < IT; ++it) O[it] = f32x4v{0.f, 0.f, 0.f, 0.f};
                    from_state(S, O);
                }
                if constexpr (DERIV) {  // (i + 1) times that, and from its derivative
#pragma unroll
                    for (int it = 0; it < IT; ++it)
#pragma unroll
                        for (int r = 0; r < 4; ++r) E[it][r] = O[it][r] * (float)(16 * it + n16 + 1 - rev);
                    from_state(D, E);
                }
                if constexpr (Sh::OVER) take_values();
                __syncthreads();  // the keys were read: the scores take their place
                if (LATE) xk.store_transposed(tid, ldsKt);
#pragma unroll
                for (int u = 0; u < ROUNDS; ++u) {
                    const int tile = u * NW + wave, it = it_of(tile), jt = tile - it * (it + 1) / 2;
                    if (tile >= TILES) break;
                    T part[SP][4];
                    split<T, 3, 4>(p[u], reinterpret_cast<T(&)[OP][4]>(part));
                    if constexpr (DERIV) {
                        float y[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) y[r] = p[u][r] * (float)(16 * (it - jt) + apart - r);
                        split<T, 3, 4>(y, reinterpret_cast<T(&)[OP][4]>(part[OP]));
                    }
#pragma unroll
                    for (int s = 0; s < SP; ++s) {
                        T *const to = ldsP + s * Sh::PART;
                        __builtin_memcpy(__builtin_assume_aligned(
                                             to + score_place<T, Sh::SHORT>(16 * it + n16, 16 * jt + 4 * g), 8),
                                         part[s], 4 * sizeof(T));
                        if (jt == it && it % 2 == 0) {  // the rest of 32 columns
                            const T none[4] = {T(0), T(0), T(0), T(0)};
                            __builtin_memcpy(__builtin_assume_aligned(
                                                 to + score_place<T, Sh::SHORT>(16 * it + n16, 16 * jt + 16 + 4 * g), 8),
                                             none, sizeof none);
                        }
                    }
                }
                if constexpr (!DERIV && !LATE) {
#pragma unroll
                    for (int it = 0; it < IT; ++it) O[it] = f32x4v{0.f, 0.f, 0.f, 0.f};
                    from_state(S, O);
                }
            }
            if (LATE) __syncthreads();
            // ---- the state behind the chunk
            if constexpr (!Sh::OVER) take_values();
            const float keep = power[len], less = power_less[len];
            if (keep > 0.5f) {  // a slow decay by what it takes away
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if constexpr (DERIV) {
                            const float x = __builtin_fmaf((float)len, S[kt][r], D[kt][r]);
                            D[kt][r] = __builtin_fmaf(x, less, x);
                        }
                        S[kt][r] = __builtin_fmaf(S[kt][r], less, S[kt][r]);
                    }
            } else {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if constexpr (DERIV) D[kt][r] = __builtin_fmaf((float)len, S[kt][r], D[kt][r]) * keep;
                        S[kt][r] *= keep;
                    }
            }
            if constexpr (KIND != kState) {
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int i = 16 * it + n16;
                    const float w = a.s_inter * power[i + 1 - rev];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        O[it][r] *= w;
                        if constexpr (DERIV) E[it][r] *= w;
                    }
                }
            }
#pragma unroll
            for (int f = 0; f < JF; ++f) {
                Frag<T> vs[NP], vd[NP];
                T v[8];
                __builtin_memcpy(v, &vf[f], sizeof v);
                float x[8];
                if (len == C) {
                    __builtin_memcpy(x, __builtin_assume_aligned(behind + 32 * f + 8 * g, 16), sizeof x);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = behind[C - len + 32 * f + 8 * g + e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= widened(v[e]);
                split<T, 3>(x, vs);
                if constexpr (DERIV) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= (float)max(len - 1 + rev - (32 * f + 8 * g + e), 0);
                    split<T, 3>(x, vd);
                }
#pragma unroll
                for (int kg = 0; kg < KT / GR; ++kg) {
                    Frag<T> kf[GR];
#pragma unroll
                    for (int i = 0; i < GR; ++i) kf[i] = by_k.at(kg * GR + i, f);
#pragma unroll
                    for (int s = 0; s < NP; ++s)
#pragma unroll
                        for (int i = 0; i < GR; ++i) {
                            mma(S[kg * GR + i], kf[i], vs[s]);
                            if constexpr (DERIV) mma(D[kg * GR + i], kf[i], vd[s]);
                        }
                }
            }
            // ---- from the chunk's own tokens
            if constexpr (KIND != kState) {
                if (!LATE) __syncthreads();
#pragma unroll
                for (int f = 0; f < JF; ++f)
#pragma unroll
                    for (int s = 0; s < SP; ++s) {
                        Frag<T> pf[IT];
#pragma unroll
                        for (int it = 2 * f; it < IT; ++it) pf[it] = by_p.at(s * IT + it, f);
#pragma unroll
                        for (int it = 2 * f; it < IT; ++it)
                            mma(s < OP ? O[it] : E[it], vf[f], pf[it]);
                    }
            }
            // ---- outputs: row i by lane % 16, four columns each
            if constexpr (KIND != kState) {
                const int c = col0 + colw + 4 * g, left = TAIL ? a.v.width - c : 4;
                // rows from the chunk's first token on, or to it: a base and the lane's place
                const int64_t t0 = first + (int64_t)pos * dir - (a.rev ? C - 1 : 0);
                const uint32_t row = a.rev ? 15 - n16 : n16;
                auto place_of = [&](auto *p, int64_t ld, int64_t head, int it) {
                    return p + (t0 + (a.rev ? C - 16 - 16 * it : 16 * it)) * ld + head +
                           (row * (uint32_t)ld + (uint32_t)c);
                };
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    if (16 * it + n16 >= len || c >= a.v.width) continue;
                    const float x[4] = {O[it][0], O[it][1], O[it][2], O[it][3]};
                    if constexpr (DERIV) {
                        float up[4];
                        load_left<4, T>(place_of(static_cast<const T *>(a.up.p), a.up.ld,
                                                 (int64_t)(h / a.up.grp) * a.up.width, it), left, up);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            dsum = r < left ? __builtin_fmaf(E[it][r], up[r], dsum) : dsum;
                    }
                    if (a.out32) {
                        store_left<4, float>(place_of(static_cast<float *>(a.out), a.ldo,
                                                      (int64_t)h * a.v.width, it), left, x);
                    } else {
                        store_left<4, T>(place_of(static_cast<T *>(a.out), a.ldo,
                                                  (int64_t)h * a.v.width, it), left, x);
                    }
                }
            }
            __syncthreads();
        }
        if (next >= seg.n) break;
        // ---- the next chunk's rows to LDS
        if (!AHEAD) load(tid);
        pos = next;
        len = next_len;
        for (;;) {
            xk.clear(tid, a.k.width, len);
            xv.clear(tid, a.v.width - col0, len);
            if (KIND != kState) {
                xq.clear(tid, a.q.width, len);
                xq.store(tid, ldsQ, LDK);
                xk.store(tid, ldsK, LDK);
            }
            if (!LATE) xk.store_transposed(tid, ldsKt);
            xv.store_transposed(tid, ldsVt);
            if (KIND != kState) {
                const bool bad = __ballot(!xv.finite()) != 0;
                if (tid % kWave == 0) unusual[wave] = bad;
            }
            __syncthreads();
            // A product with a score of 0 keeps an infinite or missing number of a later token
            // out of an earlier one's output no more than a sum would: such chunks go token by
            // token.
            if (KIND == kState || len == 1) break;
            std::conditional_t<NW == 8, uint64_t, uint32_t> any;
            static_assert(sizeof any == NW, "a byte for each wave");
            __builtin_memcpy(&any, unusual, NW);
            if (any == 0) break;
            single = len;
            len = 1;
            __syncthreads();
        }
        if (single > 0) --single;
        next = pos + len;
        next_len = single > 0 ? 1 : min(C, seg.n - next);
    }
    if (a.end)
        each_state(a.end, a.end_by_seq, [&](int kt, int r, bool in, const float *p) {
            if (in) *const_cast<float *>(p) = S[kt][r];
        });
    if constexpr (DERIV) {  // what the segment adds to the states behind it
        if (a.back)
            each_state(a.back, a.back_by_seq, [&](int kt, int r, bool in, const float *p) {
                const float x = *p;
                dsum = in ? __builtin_fmaf(D[kt][r], x, dsum) : dsum;
            });
#pragma unroll
        for (int m = 1; m < kWave; m <<= 1) dsum += __shfl_xor(dsum, m, kWave);
        if (lane == 0) wave_sum[wave] = dsum;
        __syncthreads();
        if (threadIdx.x == 0) {
            float t = 0.f;
            for (int w = 0; w < NW; ++w) t += wave_sum[w];
            a.sums[unit] = t;
        }
    }
}

// Columns of the values that a block takes.  128 share the scores of 128: a prompt of 65,536
// tokens of 8 heads of 128 334 us, with 64 columns a block 342, 8,192 tokens of heads of 256 159
// and 220, a training step of 5,003 tokens in fp32 182 and 192.  But two states in parts of bf16
// leave a block of eight waves too few registers: a training step of 32,768 tokens of 64 by 128
// 1,019 us with 64 columns for the scan with the gradient of g, 1,149 with 128 (the gradient of four
// sequences of 8,192 tokens of 128 by 128: 1,422 and 1,474; heads of 256, whose block has a CU
// for itself, go the other way, 871 and 773).
constexpr int block_columns(Kind kind, bool bf16, int width) {
    return width > 64 && !(kind == kDerivative && bf16) ? 128 : 64;
}

nsd_status launch_scan_f32(Kind kind, const Scan &a, hipStream_t st);
nsd_status launch_scan_bf16(Kind kind, const Scan &a, hipStream_t st);

template <class T, int KD, int NW, Kind KIND>
nsd_status launch_one(const Scan &a, hipStream_t st) {
    const int nvb = (int)ceil_div(a.v.width, NW * 16);
    const int64_t blocks = (int64_t)a.nseg * a.H * nvb;
    if (blocks == 0) return NSD_OK;
    if (a.k.width % 4 == 0 && a.v.width % 4 == 0)  // whole pieces of the rows, at any address
        scan_kernel<T, KD, NW, KIND, false><<<blocks, NW * kWave, 0, st>>>(a, nvb);
    else
        scan_kernel<T, KD, NW, KIND, true><<<blocks, NW * kWave, 0, st>>>(a, nvb);
    return check_launch("scan_kernel");
}

template <class T, int KD, Kind KIND>
nsd_status launch_columns(const Scan &a, hipStream_t st) {
    constexpr bool kBf16 = sizeof(T) == 2;
    if constexpr (block_columns(KIND, kBf16, kMaxWidth) == 128)
        if (block_columns(KIND, kBf16, a.v.width) == 128) return launch_one<T, KD, 8, KIND>(a, st);
    return launch_one<T, KD, 4, KIND>(a, st);
}

template <class T, Kind KIND>
nsd_status launch_kind(const Scan &a, hipStream_t st) {
    if (a.k.width <= 32) return launch_columns<T, 32, KIND>(a, st);
    if (a.k.width <= 64) return launch_columns<T, 64, KIND>(a, st);
    if (a.k.width <= 128) return launch_columns<T, 128, KIND>(a, st);
    return launch_columns<T, 256, KIND>(a, st);
}

template <class T>
nsd_status launch_any(Kind kind, const Scan &a, hipStream_t st) {
    switch (kind) {
        case kOutput: return launch_kind<T, kOutput>(a, st);
        case kState: return launch_kind<T, kState>(a, st);
        default: return launch_kind<T, kDerivative>(a, st);
    }
}

}  // namespace decay
}  // namespace nsd
