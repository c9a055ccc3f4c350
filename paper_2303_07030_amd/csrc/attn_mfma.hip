// Differential attention over stored keys in bfloat16, on the matrix cores.
//
// A wave takes 32 entries of a row at a time for a slab of key heads: as many
// as make at most 128 columns and, with the query heads that read them, at
// most 8 query heads.  The 16 rows of a matrix product are those heads' two
// maps.  That is worth it although a row of the mask shares its keys with no
// other row: one product instruction replaces dozens of conversions and sums
// over lanes (16 heads over 4 key heads, d = 64: the vector form took 15
// instructions an entry and head, this takes about 2).
//
//   S^T = K Q^T      K's rows as they are gathered: lane (n, g) holds 8 columns
//                    32 c + 8 g.. of key n.  Q^T holds each head's halves on
//                    the columns of its key head and zeros elsewhere, so heads
//                    of one slab do not mix.  The product gives lane (n, g) the
//                    scores of row n (a head's map) at keys 4 g + i: a softmax
//                    in the lane, and two exchanges for the row's maximum.
//   O  += P V        P's operand is those very registers: as two tiles of 16
//                    keys, lane (n, g) has 8 keys of row n, and the order in
//                    which a product takes its 32 keys is free as long as V's
//                    operand has the same.  V is loaded 8 columns a lane and 8
//                    keys in turn, and paired by byte permutes: no LDS.
//
// Rows of the product are ordered so that lane group g ends with both maps of
// heads 2 g and 2 g + 1: the difference needs no exchange.  Weights go into the
// products as three bfloat16 numbers, each the nearest to what those before leave:
// the 24 bits of a 32-bit float.  The output is a difference of two maps that may
// nearly cancel, and the row sums of a gradient's weights cancel always; with two
// numbers (16 bits) what is left of such sums is wrong by up to 2^-17 of their
// terms, more than the output's own rounding.
//
// Zeros in Q^T meet other heads' keys: a key that is not finite there would make
// 0 times infinity.  A row whose sums come out NaN is therefore walked again
// with the products taken half by half of one head, everything else masked.
//
// Bound by HBM where a cache is read once (sixteen tokens over 24K keys each, 4 key
// heads of d = 64: 201 us, 4.2 TB/s of rows in random order; 194 with weights of 16
// bits), by issue and latency at two waves a SIMD where rows share keys (a training
// step of 8192 rows, a window of 256 and 16 keys more, 8 heads over 4: 1.31 ms; 1.25
// with weights of 16 bits).  At these widths (d = 64, dv = 128) the kernels need a
// few registers more than two waves leave them: 12 to 84 bytes of scratch a lane, 96
// to 164 where the key columns do not fill their chunks.
#include "attn.hpp"
#include "attn_mfma.hpp"

namespace nsd {
namespace attn {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t bf16_t;

__device__ __forceinline__ f32x4v mma(u32x4 a, u32x4 b, f32x4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ u32x4 load16(const bf16_t *p) {
    u32x4 r;
    __builtin_memcpy(&r, p, 16);
    return r;
}

// Eight weights as sums of three bfloat16 numbers.
struct Weights {
    u32x4 part[3];
    __device__ __forceinline__ explicit Weights(const float (&p)[8]) {
        bf16x8 h[3];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            float left = p[t];
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                h[i][t] = static_cast<__bf16>(left);
                left -= static_cast<float>(h[i][t]);
            }
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) part[i] = __builtin_bit_cast(u32x4, h[i]);
    }
};

// Column j of 8 rows of 8 columns, as a product's operand.
__device__ __forceinline__ u32x4 column(const u32x4 (&v)[8], int j) {
    const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], sel);
    return r;
}

// The value of another lane.
__device__ __forceinline__ float from_lane(float v, int lane) { return __shfl(v, lane); }
__device__ __forceinline__ int from_lane(int v, int lane) { return __shfl(v, lane); }

// What a wave's lanes hold of its slab.  The 16 product rows are R = 8 >> lrh
// mask rows of up to 1 << lrh heads of two maps each.
struct Geo {
    int n, g;              // lane = 16 g + n
    int kv0, hsl;          // first key head of the slab, key heads in it
    int h0, RH;            // first query head, query heads (at most 8)
    int Dl, Wl;            // columns of the slab in K and in V
    int sub, hx, kvl, map; // mask row, head, key head within the slab, map of row n
    bool used;             // row n is one

    __device__ __forceinline__ Geo(const Shape &s, const Slab &b, int slab) {
        const int lane = threadIdx.x % kWave;
        n = lane % 16;
        g = lane / 16;
        const int part = slab % b.nsub;
        kv0 = slab / b.nsub * b.hs;
        hsl = min(b.hs, s.Hk - kv0);
        h0 = kv0 * s.grp + part * 8;
        RH = b.hs == 1 ? min(s.grp - part * 8, 8) : hsl * s.grp;
        Dl = hsl * 2 * s.d;
        Wl = hsl * s.dv;
        const int y = 2 * (n >> 2) + (n & 1), x = y & ((1 << b.lrh) - 1);
        sub = y >> b.lrh;
        map = (n >> 1) & 1;
        used = x < RH;
        hx = h0 + min(x, RH - 1);
        kvl = hx / s.grp - kv0;
    }
};

// Where lane group g's 8 columns of 32-column chunk c of L columns start: past
// the end it steps back to the last 8 (its first `dup` are another lane's), a
// chunk that has none reads the first.
struct Piece {
    int start, dup;
    bool on;
};
__device__ __forceinline__ Piece piece(int col, int L) {
    Piece p;
    p.on = col < L;
    p.start = p.on ? min(col, L - 8) : 0;
    p.dup = p.on ? col - p.start : 0;
    return p;
}
// Bits of the piece's columns within [lo, lo + len) that are this lane's own.
__device__ __forceinline__ u32x4 piece_mask(const Piece &p, int lo, int len) {
    u32x4 m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a = 2 * i, c = p.start + a - lo;
        const uint32_t x = p.on && a >= p.dup && c >= 0 && c < len ? 0xFFFFu : 0u;
        const uint32_t y = p.on && a + 1 >= p.dup && c + 1 >= 0 && c + 1 < len ? 0xFFFF0000u : 0u;
        m[i] = x | y;
    }
    return m;
}

// Orders a wave's LDS accesses (the hardware takes them in order: this is for the
// compiler).
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The rows of a tile's 32 keys as a product's operand: lane (n, g) needs 8 columns
// of key n, but a load whose neighbouring lanes read different rows takes four
// times the accesses of one that reads rows in order (a tile of 16 KB: 640
// against 256).  So rows are loaded in order, 2 N loads of 64 pieces of 8
// columns, and turned in LDS; a piece's place is xored with its row's number,
// which leaves neither side a bank conflict.  FULL: L = 32 N.
template <int N, bool FULL>
struct KeyCols {
    static constexpr int P = 4 * N;             // pieces of a row
    static constexpr int kWords = 32 * P;       // 16-byte words of a wave's tile
    int off;      // of the piece that this lane loads
    u32x4 edge;   // of the one chunk that L ends in
    int L;
    __device__ __forceinline__ KeyCols(int lane, int L_) : L(L_) {
        off = piece(8 * (lane % P), L).start;
        if (!FULL) edge = piece_mask(piece(L / 32 * 32 + 8 * (lane / 16), L), 0, L);
    }
    __device__ __forceinline__ bool has(int c) const { return FULL || 32 * c < L; }
    // Where piece p of row r lies in the tile.
    static __device__ __forceinline__ int place(int r, int p) {
        return r * P + (p ^ (N == 1 ? r >> 2 & 3 : N == 2 ? r >> 1 & 7 : r & 15));
    }
    // Row i at base + idx_i ld, idx_i held by lane i; `two`: the last 16 exist.
    __device__ __forceinline__ void load(const bf16_t *base, int64_t ld, int idx, bool two,
                                         u32x4 (&x)[2 * N]) const {
        const int lane = threadIdx.x % kWave;
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = load16(base + (int64_t)from_lane(idx, (64 * i + lane) / P) * ld + off);
#pragma unroll
        for (int i = N; i < 2 * N; ++i) x[i] = u32x4{0, 0, 0, 0};
        if (two) {
#pragma unroll
            for (int i = N; i < 2 * N; ++i)
                x[i] = load16(base + (int64_t)from_lane(idx, (64 * i + lane) / P) * ld + off);
        }
    }
    __device__ __forceinline__ void turn(const u32x4 (&x)[2 * N], u32x4 *tile) const {
        const int lane = threadIdx.x % kWave;
        wave_fence();  // the tile before has been read
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) tile[place((64 * i + lane) / P, lane % P)] = x[i];
        wave_fence();
    }
    // k^T q of 16 rows of the tile.
    __device__ __forceinline__ f32x4v dot(const u32x4 *tile, int n, int g, int half,
                                          const u32x4 (&q)[N]) const {
        f32x4v s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (!has(c)) continue;
            const u32x4 k = tile[place(16 * half + n, 4 * c + g)];
            s = mma(!FULL && c == L / 32 ? k & edge : k, q[c], s);
        }
        return s;
    }
    // The same of the columns [lo, lo + len) alone, the others not read.
    __device__ __forceinline__ f32x4v dot_of(const u32x4 *tile, int n, int g, int half, int lo,
                                             int len, const u32x4 (&q)[N]) const {
        f32x4v s = {0.f, 0.f, 0.f, 0.f};
        opaque(g);  // masks made here, not kept through the kernel
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (!has(c)) continue;
            const u32x4 m = piece_mask(piece(32 * c + 8 * g, L), lo, len);
            s = mma(tile[place(16 * half + n, 4 * c + g)] & m, q[c], s);
        }
        return s;
    }
};

// Row n's operand: `len` values at `p` on the columns [lo, lo + len) of L, zeros
// elsewhere.  ALIGNED: len and lo are multiples of 8, a piece is in or out.
template <int N, bool FULL>
__device__ __forceinline__ void row_operand(const KeyCols<N, FULL> &cols, int g, const bf16_t *p,
                                            int lo, int len, bool used, bool aligned,
                                            u32x4 (&q)[N]) {
    opaque(g);  // a row's conditions are made again, not kept
#pragma unroll
    for (int c = 0; c < N; ++c) {
        q[c] = u32x4{0, 0, 0, 0};
        if (!cols.has(c)) continue;
        const Piece pc = piece(32 * c + 8 * g, cols.L);
        if (aligned) {
            if (used && pc.on && pc.start >= lo && pc.start < lo + len)
                q[c] = load16(p + pc.start - lo);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int at = pc.start + e - lo;
                if (used && pc.on && e >= pc.dup && at >= 0 && at < len)
                    q[c][e / 2] |= (uint32_t)p[at] << (16 * (e & 1));
            }
        }
    }
}

__device__ __forceinline__ uint32_t low_bits(int k) { return k >= 32 ? ~0u : (1u << k) - 1u; }

// This lane's 8 entries of a tile: 4 g + i of either half.
__device__ __forceinline__ int tile_entry(int g, int t) { return 4 * g + (t & 3) + (t & 4) * 4; }

// 32 keys and who uses them.  A group is up to R consecutive rows, of which lane
// l knows row row0 + l % 8 by its entries [lo, hi), and row row0 + sub by what is
// marked "own".
struct Tile {
    int idx;        // key l % 32
    float bias;     // its bias
    uint32_t used;  // keys in use
    uint32_t bits;  // own: the keys that are entries of the row
    int start;      // own: the first of those entries
    int row0, lo, hi;
    bool last;      // of its group
    __device__ __forceinline__ bool in(int g, int t) const {
        return (bits & used) >> tile_entry(g, t) & 1;
    }
    __device__ __forceinline__ int entry(int g, int t) const {
        return start + __popc(bits & low_bits(tile_entry(g, t)));
    }
    __device__ __forceinline__ bool has(int row) const {  // row0 + row has entries
        return from_lane(hi, row) > from_lane(lo, row);
    }
};

__device__ __forceinline__ int or_lanes(int v, int n) {  // over groups of 8 or 32 lanes
    auto other = [](float x) { return __float_as_int(x); };
    v |= other(lane_xor<1>(__int_as_float(v)));
    v |= other(lane_xor<2>(__int_as_float(v)));
    v |= other(lane_xor<4>(__int_as_float(v)));
    if (n > 8) {
        v |= other(lane_xor<8>(__int_as_float(v)));
        v |= other(lane_xor<16>(__int_as_float(v)));
    }
    return v;
}
__device__ __forceinline__ int sum_8(int v) {
    auto other = [](float x) { return __float_as_int(x); };
    v += other(lane_xor<1>(__int_as_float(v)));
    v += other(lane_xor<2>(__int_as_float(v)));
    return v + other(lane_xor<4>(__int_as_float(v)));
}
__device__ __forceinline__ int min_8(int v) {
    auto other = [](float x) { return __float_as_int(x); };
    v = min(v, other(lane_xor<1>(__int_as_float(v))));
    v = min(v, other(lane_xor<2>(__int_as_float(v))));
    return min(v, other(lane_xor<4>(__int_as_float(v))));
}

// A walk over one item's entries, tile by tile, R rows together.
//
// In runs: a tile is 32 consecutive entries, whichever of the group's rows they
// are of.  Shared: rows that are near often store the same columns (windows,
// documents); a tile is then 32 consecutive columns from the lowest that a row
// has next, and a key serves every row that stores it.  Groups whose rows all
// have 32 entries and more are tried: a shared tile has to hold kShared entries,
// and where it does not, 32 of the first unfinished row are taken; after kTries
// of those no more is tried.  (A window of 256: tiles a row 9 -> 2.4.)
constexpr int kShared = 48, kTries = 2;

struct Walk {
    const int32_t *idx, *segidx, *segptr;
    const float *bias;
    int nseg, b0, R, sub;
    bool may_share, done;
    // the group
    int row0, p, end, lo, hi, cur, tries;
    bool shared;
    // the next group
    int nrow0, nlo, nhi, nend;
    // loaded for the next tile
    int c[4], first;
    float b;

    __device__ __forceinline__ Walk(const int32_t *idx_, const int32_t *segidx_,
                                    const int32_t *segptr_, const float *bias_, int nseg_, int R_,
                                    int sub_, bool may_share_)
        : idx(idx_), segidx(segidx_), segptr(segptr_), bias(bias_), nseg(nseg_), R(R_), sub(sub_),
          may_share(may_share_), done(false) {}

    // All rows of the item [a0, b0_).
    __device__ __forceinline__ void begin(int a0, int b0_) {
        b0 = b0_;
        fetch_group(a0);
        enter(a0);
        load();
    }
    // The entries [a0, b0_) of one row.
    __device__ __forceinline__ void begin_row(int row, int a0, int b0_) {
        b0 = b0_;
        nrow0 = row;
        nlo = threadIdx.x % 8 == 0 ? a0 : b0;
        nhi = nend = b0;
        enter(a0);
        load();
    }

    __device__ __forceinline__ void fetch_group(int at) {
        const int l = threadIdx.x % 8;
        nrow0 = segidx[at];
        const int rows = min(R, nseg - nrow0);
        const bool one = l < rows;
        nlo = one ? max(segptr[nrow0 + l], at) : b0;
        nhi = one ? max(min(segptr[nrow0 + l + 1], b0), nlo) : b0;
        nend = min(segptr[nrow0 + rows], b0);
    }
    __device__ __forceinline__ void enter(int at) {
        row0 = nrow0;
        lo = cur = nlo;
        hi = nhi;
        end = nend;
        p = at;
        tries = 0;
        const bool small = (int)(threadIdx.x % 8) < R && hi - lo < 32;
        shared = may_share && R > 1 && __ballot(small) == 0;
        if (end < b0) fetch_group(end);
        else nrow0 = -1;
    }
    __device__ __forceinline__ void load() {
        const int lane = threadIdx.x % kWave;
        if (!shared) {
            const int e = p + min(lane % 32, b0 - 1 - p);
            c[0] = idx[e];
            b = bias ? bias[e] : 0.f;
            return;
        }
        first = cur < hi ? idx[cur] : INT32_MAX;
#pragma unroll
        for (int r = 0; r < 8; r += 2) {
            if (r >= R) break;
            const int row = r + lane / 32, e = from_lane(cur, row);
            c[r / 2] = lane % 32 < from_lane(hi, row) - e ? idx[e + lane % 32] : INT32_MAX;
        }
    }

    __device__ __forceinline__ Tile make() {
        const int lane = threadIdx.x % kWave, l = lane % 8;
        Tile t;
        t.row0 = row0;
        t.lo = lo;
        t.hi = hi;
        if (!shared) {
            t.idx = c[0];
            t.bias = b;
            t.used = (uint32_t)__ballot(lane % 32 < end - p && b != -INFINITY);
            const int olo = from_lane(lo, sub), ohi = from_lane(hi, sub);
            t.bits = low_bits(min(max(ohi - p, 0), 32)) & ~low_bits(min(max(olo - p, 0), 32));
            t.start = max(olo, p);
            t.last = end - p <= 32;
            p = t.last ? end : p + 32;
        } else {
            const int lowest = __builtin_amdgcn_readfirstlane(min_8(first));
            int mine = 0;  // keys of row row0 + l
            bool share = false;
            if (tries < kTries) {
#pragma unroll
                for (int r = 0; r < 8; r += 2) {
                    if (r >= R) break;
                    // past the row's end c is INT32_MAX, which no column is
                    const uint32_t k = (uint32_t)c[r / 2] - (uint32_t)lowest;
                    const bool near = k < 32u && c[r / 2] != INT32_MAX;
                    const int v = or_lanes(near ? (int)(1u << k) : 0, 32);
                    const int x = from_lane(v, l % 2 * 32);
                    mine = l / 2 == r / 2 ? x : mine;
                }
                const int held = sum_8(__popc(mine)), left = sum_8(hi - cur);
                share = __builtin_amdgcn_readfirstlane(held) >= kShared ||
                        __builtin_amdgcn_readfirstlane(held) ==
                            __builtin_amdgcn_readfirstlane(left);
                tries += !share;
            }
            t.idx = (int)((uint32_t)lowest + lane % 32);  // past the last column: not used
            if (!share) {
                const int row =
                    __builtin_ctz((uint32_t)__ballot(cur < hi) & 0xFFu);  // the first with any left
                mine = l == row ? (int)low_bits(min(hi - cur, 32)) : 0;
#pragma unroll
                for (int r = 0; r < 8; r += 2) {  // each in turn: an index would put c in memory
                    if (r >= R) break;
                    const int x = from_lane(c[r / 2], row % 2 * 32 + lane % 32);
                    t.idx = row / 2 == r / 2 ? x : t.idx;
                }
            }
            t.bias = 0.f;
            t.used = (uint32_t)__builtin_amdgcn_readfirstlane(or_lanes(mine, 8));
            t.bits = (uint32_t)from_lane(mine, sub);
            t.start = from_lane(cur, sub);
            cur += __popc(mine);
            t.last = __ballot(cur < hi) == 0;
        }
        if (t.last) {
            if (nrow0 < 0) done = true;
            else enter(end);
        }
        if (!done) load();
        return t;
    }
};

// The rows of an item, one by one.
template <class F>
__device__ __forceinline__ void for_rows(const int32_t *segidx, const int32_t *segptr, int p,
                                         int b0, F f) {
    while (p < b0) {
        const int row = segidx[p], end = min(segptr[row + 1], b0);
        f(row, p, end);
        p = end;
    }
}

// One row's entries from p on, for a walk of that row alone: `own` lanes use them.
__device__ __forceinline__ Tile alone(const int32_t *idx, const float *bias, int p, int end,
                                      bool own) {
    const int l = threadIdx.x % 32, e = p + min(l, end - 1 - p);
    Tile t = {};
    t.idx = idx[e];
    t.bias = bias ? bias[e] : 0.f;
    t.used = (uint32_t)__ballot(l < end - p && t.bias != -INFINITY);
    t.bits = own ? low_bits(min(end - p, 32)) : 0u;
    t.start = p;
    return t;
}

// An unused entry stands for a used one (if there is any): what it loads exists
// and is used anyway.
__device__ __forceinline__ int stand_in(int idx, uint32_t bits) {
    const int first = __builtin_amdgcn_readlane(idx, bits ? __builtin_ctz(bits) : 0);
    return bits >> (threadIdx.x % 32) & 1 ? idx : first;
}
__device__ __forceinline__ float over_groups_max(float v) {
    v = fmaxf(v, lane_xor<16>(v));
    return fmaxf(v, lane_xor<32>(v));
}
__device__ __forceinline__ float over_groups_sum(float v) {
    v += lane_xor<16>(v);
    return v + lane_xor<32>(v);
}

// Columns 128 v + 8 n .. of rows that are weighted and summed, and the products.
template <int NV>
struct SumCols {
    int off[NV];  // from the slab's first column
    bool on[NV];
    __device__ __forceinline__ SumCols(int n, int L) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const Piece p = piece(128 * v + 8 * n, L);
            off[v] = p.start;
            on[v] = p.on;
        }
    }
    // This lane's columns of its 8 entries' rows: row e at base + idx_e ld, idx_e
    // held by lane e.  `two`: the last four exist.
    __device__ __forceinline__ void load(const bf16_t *base, int64_t ld, int idx, int g, bool two,
                                         u32x4 (&x)[NV][8]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const bf16_t *row = base + (int64_t)from_lane(idx, tile_entry(g, t)) * ld;
#pragma unroll
            for (int v = 0; v < NV; ++v) x[v][t] = load16(row + off[v]);
        }
#pragma unroll
        for (int t = 4; t < 8; ++t)
#pragma unroll
            for (int v = 0; v < NV; ++v) x[v][t] = u32x4{0, 0, 0, 0};
        if (two) {
#pragma unroll
            for (int t = 4; t < 8; ++t) {
                const bf16_t *row = base + (int64_t)from_lane(idx, tile_entry(g, t)) * ld;
#pragma unroll
                for (int v = 0; v < NV; ++v) x[v][t] = load16(row + off[v]);
            }
        }
    }
};

// acc += w rows.
template <int NV>
__device__ __forceinline__ void weigh(const u32x4 (&x)[NV][8], const Weights &w,
                                      f32x4v (&acc)[NV][8]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u32x4 b = column(x[v], j);
#pragma unroll
            for (int i = 0; i < 3; ++i) acc[v][j] = mma(w.part[i], b, acc[v][j]);
            // the paired columns are made one at a time: made all at once they
            // take as many registers again as the rows
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

template <int NV>
__device__ __forceinline__ void clear(f32x4v (&acc)[NV][8]) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[v][j] = f32x4v{0.f, 0.f, 0.f, 0.f};
}

// NaN if some sum is not finite.
template <int NV>
__device__ __forceinline__ float taint(const f32x4v (&acc)[NV][8]) {
    float z = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) z = __builtin_fmaf(acc[v][j][i], 0.f, z);
    return z;
}
// Rows of unused keys as zeros.
template <int NV>
__device__ __forceinline__ void drop_unused(u32x4 (&x)[NV][8], int g, uint32_t used) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const uint32_t m = used >> tile_entry(g, t) & 1 ? ~0u : 0u;
#pragma unroll
        for (int v = 0; v < NV; ++v) x[v][t] &= u32x4{m, m, m, m};
    }
}

// One row's group, of the first product rows alone.
__device__ __forceinline__ Tile row_tile(int row, int lo, int hi) {
    Tile t = {};
    t.row0 = row;
    t.lo = lo;
    t.hi = threadIdx.x % 8 == 0 ? hi : lo;
    return t;
}

// ------------------------------------------------------------ forward

template <int NC, int NV, bool FULL>
struct Fwd {
    const FwdArgs &a;
    const Slab &b;
    const Geo geo;
    const KeyCols<NC, FULL> kc;
    const SumCols<NV> vc;
    const bf16_t *K, *V;
    u32x4 q[NC], k[2 * NC], x[NV][8];  // a row's operand; a tile's keys and values
    f32x4v acc[NV][8];
    float m, l;
    u32x4 *tile;

    __device__ __forceinline__ Fwd(const FwdArgs &a_, const Slab &b_, int slab, u32x4 *tile_)
        : a(a_), b(b_), geo(a_.s, b_, slab), kc(threadIdx.x % kWave, geo.Dl),
          vc(geo.n, geo.Wl), tile(tile_) {
        K = static_cast<const bf16_t *>(a.K) + (int64_t)geo.kv0 * 2 * a.s.d;
        V = static_cast<const bf16_t *>(a.V) + (int64_t)geo.kv0 * a.s.dv;
    }

    __device__ __forceinline__ void load_query(int64_t row) {
        row = min(row, (int64_t)a.nrows - 1);
        const bf16_t *Q = static_cast<const bf16_t *>(a.Q) + row * a.s.ldq +
                          ((int64_t)geo.hx * 2 + geo.map) * a.s.d;
        row_operand(kc, geo.g, Q, (geo.kvl * 2 + geo.map) * a.s.d, a.s.d, geo.used,
                    a.s.d % 8 == 0, q);
    }
    __device__ __forceinline__ void load_keys(int idx, bool two) {
        kc.load(K, a.s.ldk, idx, two, k);
    }
    __device__ __forceinline__ void load_values(int idx, bool two) {
        vc.load(V, a.s.ldv, idx, geo.g, two, x);
    }
    __device__ __forceinline__ void reset() {
        clear(acc);
        m = -INFINITY;
        l = 0.f;
    }

    // Scores of the keys loaded, half by half if `apart`.
    __device__ __forceinline__ void scores(bool apart, f32x4v &s0, f32x4v &s1) const {
        kc.turn(k, tile);
        if (!apart) {
            s0 = kc.dot(tile, geo.n, geo.g, 0, q);
            s1 = kc.dot(tile, geo.n, geo.g, 1, q);
            return;
        }
        for (int h = 0; h < geo.hsl * 2; ++h) {
            const bool own = geo.kvl * 2 + geo.map == h || h == 0;
            const f32x4v x0 = kc.dot_of(tile, geo.n, geo.g, 0, h * a.s.d, a.s.d, q);
            const f32x4v x1 = kc.dot_of(tile, geo.n, geo.g, 1, h * a.s.d, a.s.d, q);
            s0 = own ? x0 : s0;
            s1 = own ? x1 : s1;
        }
    }

    // The tile's weights into the rows' sums.
    __device__ __forceinline__ void absorb(f32x4v s0, f32x4v s1, const Tile &c) {
        float s[8], top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 8; ++t) s[t] = (t < 4 ? s0[t] : s1[t - 4]) * a.s.scale;
        if (a.bias) {
#pragma unroll
            for (int t = 0; t < 8; ++t) s[t] += from_lane(c.bias, tile_entry(geo.g, t));
        }
        if (!__all((c.bits & c.used) == ~0u)) {
#pragma unroll
            for (int t = 0; t < 8; ++t) s[t] = c.in(geo.g, t) ? s[t] : -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) top = fmaxf(top, s[t]);
        top = over_groups_max(top);
        if (__any(top > m)) {
            const float mn = fmaxf(m, top);
            const float f = exp_diff(m, finite_max(mn));
            l *= f;
            m = mn;
            float fr[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fr[i] = from_lane(f, 4 * geo.g + i);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[v][j][i] *= fr[i];
        }
        const float ms = finite_max(m);
        float w[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            w[t] = exp_diff(s[t], ms);
            l += w[t];
        }
        weigh(x, Weights(w), acc);
    }

    // Whether a sum is not finite: a row's own doing, or another's or another
    // head's times 0.
    __device__ __forceinline__ bool tainted() const {
        const float z = taint(acc) + l * 0.f;
        return __any(z != z);
    }
    // The entries [p, end) of a row again, by itself and half by half, what it does
    // not use masked.
    __device__ __forceinline__ void walk_apart(int row, int p, int end, int at) {
        const Tile c = row_tile(row, p, end);
        load_query(row);
        reset();
        for (; p < end; p += min(32, end - p)) {
            const Tile t = alone(a.colind, a.bias, p, end, geo.sub == 0);
            if (t.used == 0) continue;
            const int idx = stand_in(t.idx, t.used);
            load_keys(idx, true);
            load_values(idx, true);
            drop_unused(x, geo.g, t.used);
            f32x4v s0, s1;
            scores(true, s0, s1);
            absorb(s0, s1, t);
        }
        finish(c, at);
    }

    template <class F>
    __device__ __forceinline__ void each_piece(const Tile &c, F f) const {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int r = (2 * geo.g + y) >> b.lrh, x = (2 * geo.g + y) & ((1 << b.lrh) - 1);
            const bool has = c.has(r);
            if (x >= geo.RH || !has) continue;
            const int head = (geo.h0 + x) / a.s.grp - geo.kv0;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int kvl = b.hs == 1 ? 0 : vc.off[v] / a.s.dv;
                if (vc.on[v] && kvl == head)
                    f(c.row0 + r, geo.h0 + x, v, y, vc.off[v] - kvl * a.s.dv);
            }
        }
    }

    // The group's rows into O, or into partial `at`.
    __device__ __forceinline__ void finish(const Tile &c, int at) {
        const float ls = over_groups_sum(l);
        const bool has = c.has(geo.sub);  // by every lane: it reads across them
        const bool own = geo.g == 0 && geo.used && has;
        const float st[2] = {m, ls};
        if (at >= 0) {
            const int ld = 4 + 2 * a.s.dv;
            float *o = a.part + (int64_t)at * a.s.H * ld;
            if (own) __builtin_memcpy(o + (int64_t)geo.hx * ld + 2 * geo.map, st, 8);
            each_piece(c, [&](int, int h, int v, int y, int col) {
                float x1[8], x2[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x1[j] = acc[v][j][y];
                    x2[j] = acc[v][j][2 + y];
                }
                float *p = o + (int64_t)h * ld + 4 + col;
                store_values<float, 8>(p, x1);
                store_values<float, 8>(p + a.s.dv, x2);
            });
            return;
        }
        float inv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = from_lane(ls, 4 * geo.g + i);
            inv[i] = x == 0.f ? 0.f : 1.f / x;
        }
        each_piece(c, [&](int row, int h, int v, int y, int col) {
            const float i1 = inv[y], i2 = a.lambda[h] * inv[2 + y];
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = acc[v][j][y] * i1 - acc[v][j][2 + y] * i2;
            store_values<bf16_t, 8>(static_cast<bf16_t *>(a.O) + row * a.s.ldo +
                                        (int64_t)h * a.s.dv + col, o);
        });
        if (a.stat && own)
            __builtin_memcpy(a.stat + ((int64_t)(c.row0 + geo.sub) * a.s.H + geo.hx) * 4 +
                                 2 * geo.map, st, 8);
    }
};

// Four consecutive items and one slab a block: rows that are near share keys.
struct Unit {
    int64_t item;
    int slab;
    __device__ __forceinline__ Unit(int64_t nmain, int nslab) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const int64_t q = near_block(blockIdx.x, (int)nmain);
        item = q / nslab * kAttnWaves + wave;
        slab = (int)(q % nslab);
    }
};

// Waves a SIMD that a kernel's registers must allow.
constexpr int waves(int nc, int nv) { return nc * nv <= 4 ? 2 : 1; }

// A tile's loads are issued while the tile before it is worked on: its keys (and
// the next row's query) once the scores have read the ones before, its values
// once the sums have; its entries' indexes two tiles ahead.
template <int NC, int NV, bool FULL, bool DECODE>
__global__ __launch_bounds__(kAttnThreads, waves(NC, NV)) void mfma_fwd_kernel(FwdArgs a, Slab b) {
    if (!DECODE && (int64_t)blockIdx.x >= a.nmain) {
        for_empty(a.plan, a.nrows, a.all_empty, a.nmain,
                  [&](int64_t row) { empty_row<bf16_t>(a, row); });
        return;
    }
    const Unit u(a.nmain, b.nslab);
    if (u.item >= (DECODE ? (int64_t)a.nrows * a.nsplit : (int64_t)a.plan.nitems)) return;
    __shared__ u32x4 tiles[kAttnWaves][KeyCols<NC, FULL>::kWords];
    Fwd<NC, NV, FULL> f(a, b, u.slab, tiles[threadIdx.x / kWave]);
    int at = -1;  // the partial that a chunk or split leaves
    Walk walk(a.colind, a.rowidx, a.rowptr, a.bias, a.nrows, 8 >> b.lrh, f.geo.sub,
              a.bias == nullptr);
    if constexpr (DECODE) {
        const int row = (int)(u.item / a.nsplit), j = (int)(u.item - (int64_t)row * a.nsplit);
        const int r0 = a.rowptr[row], r1 = a.colind ? a.rowptr[row + 1] : r0;
        const int p0 = (int)min((int64_t)r0 + (int64_t)j * a.per, (int64_t)r1);
        const int b0 = j + 1 == a.nsplit ? r1 : (int)min((int64_t)p0 + a.per, (int64_t)r1);
        if (a.nsplit > 1) at = (int)u.item;
        if (p0 >= b0) {
            f.reset();
            f.finish(row_tile(row, 0, 1), at);  // nothing: the empty sums
            return;
        }
        walk.begin_row(row, p0, b0);
    } else {
        if (a.plan.nchunks > 0) at = a.plan.chunk_ord[u.item];
        walk.begin(a.plan.item_ptr[u.item], a.plan.item_ptr[u.item + 1]);
    }
    Tile c = walk.make(), n = c;
    f.load_query((int64_t)c.row0 + f.geo.sub);
    int idx = stand_in(c.idx, c.used);
    f.load_keys(idx, c.used >> 16 != 0);
    f.load_values(idx, c.used >> 16 != 0);
    f.reset();
    bool more = !walk.done, bad = false;
    if (more) n = walk.make();
    while (true) {
        f32x4v s0, s1;
        f.scores(false, s0, s1);
        if (more) {
            idx = stand_in(n.idx, n.used);
            f.load_keys(idx, n.used >> 16 != 0);
            if (c.last) f.load_query((int64_t)n.row0 + f.geo.sub);
        }
        if (c.used) f.absorb(s0, s1, c);
        if (more) f.load_values(idx, n.used >> 16 != 0);
        if (c.last) {
            bad |= f.tainted();
            f.finish(c, at);
            f.reset();
        }
        if (!more) break;
        c = n;
        more = !walk.done;
        if (more) n = walk.make();
    }
    if (!bad) return;
    if constexpr (DECODE) {
        const int row = c.row0;
        f.walk_apart(row, __builtin_amdgcn_readfirstlane(walk.lo), walk.b0, at);
    } else {
        for_rows(a.rowidx, a.rowptr, a.plan.item_ptr[u.item], walk.b0,
                 [&](int row, int p, int end) { f.walk_apart(row, p, end, at); });
    }
}

// ------------------------------------------------------------ backward, rows

// Coefficients of an entry and head as they lie in memory: first (a^1, t, a^2,
// t), then, once D is known, (ds^1, a^1 - lambda a^2, ds^2, 1 if the entry is
// used): row n's lane writes and reads its own pair in both.
template <int NC, int NV, bool FULL>
struct Rows {
    const BwdArgs &a;
    const Slab &b;
    const Geo geo;
    const KeyCols<NC, FULL> kc;
    const KeyCols<4 * NV, false> wc;  // V by rows
    const bf16_t *K, *V;
    u32x4 q[NC], o[4 * NV], k[2 * NC], v[8 * NV];
    float m, inv, D;
    u32x4 *tile;  // keys, then values

    __device__ __forceinline__ Rows(const BwdArgs &a_, const Slab &b_, int slab, u32x4 *tile_)
        : a(a_), b(b_), geo(a_.s, b_, slab), kc(threadIdx.x % kWave, geo.Dl),
          wc(threadIdx.x % kWave, geo.Wl), tile(tile_) {
        K = static_cast<const bf16_t *>(a.K) + (int64_t)geo.kv0 * 2 * a.s.d;
        V = static_cast<const bf16_t *>(a.V) + (int64_t)geo.kv0 * a.s.dv;
    }

    __device__ __forceinline__ void load_operands(int64_t row) {
        row = min(row, (int64_t)a.nseg - 1);
        const bf16_t *Q = static_cast<const bf16_t *>(a.Q) + row * a.s.ldq +
                          ((int64_t)geo.hx * 2 + geo.map) * a.s.d;
        row_operand(kc, geo.g, Q, (geo.kvl * 2 + geo.map) * a.s.d, a.s.d, geo.used,
                    a.s.d % 8 == 0, q);
        const bf16_t *O = static_cast<const bf16_t *>(a.dO) + row * a.s.ldo +
                          (int64_t)geo.hx * a.s.dv;
        row_operand(wc, geo.g, O, geo.kvl * a.s.dv, a.s.dv, geo.used, a.s.dv % 8 == 0, o);
    }
    __device__ __forceinline__ void begin(int64_t row) {
        row = min(row, (int64_t)a.nseg - 1);
        float st[2];
        __builtin_memcpy(st, a.stat + (row * a.s.H + geo.hx) * 4 + 2 * geo.map, 8);
        m = finite_max(st[0]);
        inv = st[1] == 0.f ? 0.f : 1.f / st[1];
        D = 0.f;
    }
    __device__ __forceinline__ void load_keys(int idx, bool two) {
        kc.load(K, a.s.ldk, idx, two, k);
        wc.load(V, a.s.ldv, idx, two, v);
    }

    // Scores and t of the keys loaded, half by half if `apart`.
    __device__ __forceinline__ void products(bool apart, f32x4v (&s)[2], f32x4v (&t)[2]) const {
        kc.turn(k, tile);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (!apart) {
                s[e] = kc.dot(tile, geo.n, geo.g, e, q);
            } else {
                for (int h = 0; h < geo.hsl * 2; ++h) {
                    const f32x4v x =
                        kc.dot_of(tile, geo.n, geo.g, e, h * a.s.d, a.s.d, q);
                    s[e] = geo.kvl * 2 + geo.map == h || h == 0 ? x : s[e];
                }
            }
        }
        wc.turn(v, tile);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (!apart) {
                t[e] = wc.dot(tile, geo.n, geo.g, e, o);
            } else {
                for (int h = 0; h < geo.hsl; ++h) {
                    const f32x4v x =
                        wc.dot_of(tile, geo.n, geo.g, e, h * a.s.dv, a.s.dv, o);
                    t[e] = geo.kvl == h || h == 0 ? x : t[e];
                }
            }
        }
    }

    // The pairs of a tile's entries (those of masked ones are not read again); D's
    // terms added up.
    __device__ __forceinline__ void absorb(const f32x4v (&sc)[2], const f32x4v (&tc)[2],
                                           const Tile &c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = c.in(geo.g, e);
            float s = sc[e / 4][e % 4] * a.s.scale;
            if (a.bias) s += from_lane(c.bias, tile_entry(geo.g, e));
            const float w = in ? exp_diff(s, m) * inv : 0.f;
            const float t = in ? tc[e / 4][e % 4] : 0.f;
            D = __builtin_fmaf(w, t, D);
            if (in && geo.used) {
                const float y[2] = {w, t};
                __builtin_memcpy(a.coef + ((int64_t)c.entry(geo.g, e) * a.s.H + geo.hx) * 4 +
                                     2 * geo.map, y, 8);
            }
        }
    }

    // The entries [p, end) of a row again, by itself and half by half.
    __device__ __forceinline__ void walk_apart(int row, int p, int end, float *out) {
        load_operands(row);
        begin(row);
        for (; p < end; p += min(32, end - p)) {
            const Tile t = alone(a.other, a.bias, p, end, geo.sub == 0);
            if (t.used == 0) continue;
            load_keys(stand_in(t.idx, t.used), true);
            f32x4v s[2], u[2];
            products(true, s, u);
            absorb(s, u, t);
        }
        const float sum = over_groups_sum(D);
        if (geo.g == 0 && geo.used && geo.sub == 0) out[(int64_t)geo.hx * 2 + geo.map] = sum;
    }
};

// dq of rows whose D is known, and their entries' last coefficients.
template <int NK>
struct RowSums {
    const BwdArgs &a;
    const Slab &b;
    const Geo &geo;
    const SumCols<NK> qc;
    const bf16_t *K;
    u32x4 x[NK][8];
    f32x4v acc[NK][8];

    __device__ __forceinline__ RowSums(const BwdArgs &a_, const Slab &b_, const Geo &g)
        : a(a_), b(b_), geo(g), qc(g.n, g.Dl) {
        K = static_cast<const bf16_t *>(a.K) + (int64_t)g.kv0 * 2 * a.s.d;
    }

    __device__ __forceinline__ float row_D(int64_t row) const {
        row = min(row, (int64_t)a.nseg - 1);
        return a.D[(row * a.s.H + geo.hx) * 2 + geo.map];
    }
    __device__ __forceinline__ float *pair(const Tile &c, int e) const {
        return a.coef + ((int64_t)c.entry(geo.g, e) * a.s.H + geo.hx) * 4 + 2 * geo.map;
    }
    __device__ __forceinline__ void load_pairs(const Tile &c, float (&y)[8][2]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e][0] = y[e][1] = 0.f;
            if (c.in(geo.g, e)) __builtin_memcpy(y[e], pair(c, e), 8);
        }
    }
    __device__ __forceinline__ void load_keys(int idx, bool two) {
        qc.load(K, a.s.ldk, idx, geo.g, two, x);
    }
    // ds of the tile, from its pairs; the pairs are overwritten.
    __device__ __forceinline__ void last_pairs(const Tile &c, float D, float lambda,
                                               const float (&y)[8][2], float (&ds)[8]) const {
        const float f = geo.map ? -lambda : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = c.in(geo.g, e);
            const float other = lane_xor<2>(y[e][0]);  // the other map's weight
            ds[e] = f * y[e][0] * (y[e][1] - D);
            ds[e] = in ? ds[e] : 0.f;
            const float out[2] = {ds[e],
                                  geo.map ? (in ? 1.f : 0.f) : y[e][0] - lambda * other};
            if (geo.used && c.bits >> tile_entry(geo.g, e) & 1)
                __builtin_memcpy(pair(c, e), out, 8);
        }
    }
    __device__ __forceinline__ void absorb(const float (&ds)[8]) {
        weigh(x, Weights(ds), acc);
    }
    // The entries [p, end) of a row again, by itself, from the last pairs.
    __device__ __forceinline__ void walk_apart(int row, int p, int end, int at) {
        const Tile c = row_tile(row, p, end);
        clear(acc);
        for (; p < end; p += min(32, end - p)) {
            const Tile t = alone(a.other, a.bias, p, end, geo.sub == 0);
            if (t.used == 0) continue;
            float y[8][2], ds[8];
            load_pairs(t, y);
            load_keys(stand_in(t.idx, t.used), true);
            drop_unused(x, geo.g, t.used);
#pragma unroll
            for (int e = 0; e < 8; ++e) ds[e] = y[e][0];
            absorb(ds);
        }
        finish(c, at);
    }

    // The group's rows into dQ, or into partial `at`.
    __device__ __forceinline__ void finish(const Tile &c, int at) const {
        const int d2 = 2 * a.s.d;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int r = (2 * geo.g + y) >> b.lrh, x = (2 * geo.g + y) & ((1 << b.lrh) - 1);
            const bool has = c.has(r);
            if (x >= geo.RH || !has) continue;
            const int h = geo.h0 + x, head = h / a.s.grp - geo.kv0;
#pragma unroll
            for (int v = 0; v < NK; ++v) {
                const int kvl = b.hs == 1 ? 0 : qc.off[v] / d2, col = qc.off[v] - kvl * d2;
                if (!qc.on[v] || kvl != head) continue;
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    o[j] = col + j < a.s.d ? acc[v][j][y] : acc[v][j][2 + y];
                if (at >= 0) {
                    store_values<float, 8>(a.part + ((int64_t)at * a.s.H + h) * d2 + col, o);
                    continue;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] *= a.s.scale;
                store_values<bf16_t, 8>(static_cast<bf16_t *>(a.dQ) +
                                            (int64_t)(c.row0 + r) * a.s.ldq + (int64_t)h * d2 +
                                            col, o);
            }
        }
    }
};

// First pass over rows: every entry's pair and the rows' D (a chunk's part).
template <int NC, int NV, bool FULL>
__global__ __launch_bounds__(kAttnThreads, waves(NC, NV)) void mfma_weight_kernel(
    BwdArgs a, Slab b) {
    if ((int64_t)blockIdx.x >= a.nmain) {
        for_empty(a.plan, a.nseg, a.all_empty, a.nmain,
                  [&](int64_t row) { empty_row<bf16_t>(a, row); });
        return;
    }
    const Unit u(a.nmain, b.nslab);
    if (u.item >= a.plan.nitems) return;
    __shared__ u32x4 tiles[kAttnWaves][std::max(KeyCols<NC, FULL>::kWords, 128 * 4 * NV)];
    Rows<NC, NV, FULL> f(a, b, u.slab, tiles[threadIdx.x / kWave]);
    const int chunk = a.plan.nchunks > 0 ? a.plan.chunk_ord[u.item] : -1;
    Walk walk(a.other, a.idx, a.ptr, a.bias, a.nseg, 8 >> b.lrh, f.geo.sub, a.bias == nullptr);
    walk.begin(a.plan.item_ptr[u.item], a.plan.item_ptr[u.item + 1]);
    Tile c = walk.make(), n = c;
    f.load_operands((int64_t)c.row0 + f.geo.sub);
    f.begin((int64_t)c.row0 + f.geo.sub);
    int idx = stand_in(c.idx, c.used);
    f.load_keys(idx, c.used >> 16 != 0);
    float *out = chunk >= 0 ? a.part_D : a.D;
    bool more = !walk.done, bad = false;
    if (more) n = walk.make();
    while (true) {
        f32x4v s[2], t[2];
        f.products(false, s, t);
        if (more) {
            idx = stand_in(n.idx, n.used);
            f.load_keys(idx, n.used >> 16 != 0);
            if (c.last) f.load_operands((int64_t)n.row0 + f.geo.sub);
        }
        if (c.used) f.absorb(s, t, c);
        if (c.last) {
            bad |= __any(f.D != f.D);
            const int64_t at = chunk >= 0 ? chunk : (int64_t)c.row0 + f.geo.sub;
            const bool has = c.has(f.geo.sub);
            const float sum = over_groups_sum(f.D);
            if (f.geo.g == 0 && f.geo.used && has)
                out[(at * a.s.H + f.geo.hx) * 2 + f.geo.map] = sum;
            if (more) f.begin((int64_t)n.row0 + f.geo.sub);
        }
        if (!more) break;
        c = n;
        more = !walk.done;
        if (more) n = walk.make();
    }
    if (!bad) return;
    for_rows(a.idx, a.ptr, a.plan.item_ptr[u.item], walk.b0, [&](int row, int p, int end) {
        f.walk_apart(row, p, end, out + (int64_t)(chunk >= 0 ? chunk : row) * a.s.H * 2);
    });
}

// Second pass over rows, D known: the entries' last coefficients and dq.
template <int NK>
__global__ __launch_bounds__(kAttnThreads, NK == 1 ? 2 : 1) void mfma_row_kernel(
    BwdArgs a, Slab b) {
    const Unit u(a.nmain, b.nslab);
    if (u.item >= a.plan.nitems) return;
    const Geo geo(a.s, b, u.slab);
    RowSums<NK> sums(a, b, geo);
    const float lambda = a.lambda[geo.hx];
    const int chunk = a.plan.nchunks > 0 ? a.plan.chunk_ord[u.item] : -1;
    Walk walk(a.other, a.idx, a.ptr, a.bias, a.nseg, 8 >> b.lrh, geo.sub, a.bias == nullptr);
    walk.begin(a.plan.item_ptr[u.item], a.plan.item_ptr[u.item + 1]);
    Tile c = walk.make(), n = c;
    float D = sums.row_D((int64_t)c.row0 + geo.sub), nD = D, y[8][2], ny[8][2];
    sums.load_pairs(c, y);
    sums.load_keys(stand_in(c.idx, c.used), c.used >> 16 != 0);
    clear(sums.acc);
    bool more = !walk.done, bad = false;
    if (more) n = walk.make();
    while (true) {
        if (more) {
            sums.load_pairs(n, ny);
            if (c.last) nD = sums.row_D((int64_t)n.row0 + geo.sub);
        }
        float ds[8];
        sums.last_pairs(c, D, lambda, y, ds);
        if (c.used) sums.absorb(ds);
        if (more) sums.load_keys(stand_in(n.idx, n.used), n.used >> 16 != 0);
        if (c.last) {
            const float z = taint(sums.acc);
            bad |= __any(z != z);
            sums.finish(c, chunk);
            clear(sums.acc);
        }
        if (!more) break;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            y[t][0] = ny[t][0];
            y[t][1] = ny[t][1];
        }
        D = nD;
        c = n;
        more = !walk.done;
        if (more) n = walk.make();
    }
    if (!bad) return;
    for_rows(a.idx, a.ptr, a.plan.item_ptr[u.item], walk.b0,
             [&](int row, int p, int end) { sums.walk_apart(row, p, end, chunk); });
}

// D of the long rows, and their dq, from the chunks' sums: one block for a row
// and head.
__global__ __launch_bounds__(64) void mfma_join_D_kernel(BwdArgs a) {
    int64_t row, first, n;
    long_segment(a.plan, a.ptr, 0, blockIdx.x, row, first, n);
    for (int c = threadIdx.x; c < 2 * a.s.H; c += 64) {
        float s = 0.f;
#pragma unroll 8
        for (int64_t j = 0; j < n; ++j) s += a.part_D[(first + j) * 2 * a.s.H + c];
        a.D[row * 2 * a.s.H + c] = s;
    }
}
__global__ __launch_bounds__(kAttnThreads) void mfma_join_row_kernel(BwdArgs a) {
    int64_t row, first, n;
    const int h = blockIdx.x % a.s.H, W = 2 * a.s.d;
    long_segment(a.plan, a.ptr, 0, blockIdx.x / a.s.H, row, first, n);
    for (int c = threadIdx.x; c < W; c += kAttnThreads) {
        float s = 0.f;
#pragma unroll 8
        for (int64_t j = 0; j < n; ++j) s += a.part[((first + j) * a.s.H + h) * W + c];
        static_cast<bf16_t *>(a.dQ)[row * a.s.ldq + (int64_t)h * W + c] =
            narrow<bf16_t>(s * a.s.scale);
    }
}

// ------------------------------------------------------------ backward, columns

// dk and dv of a slab of key heads.  The product rows are four pairs of a column
// and a key head (so many columns at once as their number allows), four
// coefficients each: ds^1, a^1 - lambda a^2, ds^2 and one that is not used; lane
// group g ends with pair g's sums.
template <int NK, int NV>
struct ColSums {
    const BwdArgs &a;
    const Slab &b;
    int n, g, kv0, hsl, lhs;
    SumCols<NK> qc;
    SumCols<NV> oc;
    int qh[NK], oh[NV], qcol[NK], ocol[NV];  // a piece's key head and column in it
    bool weighs;
    int64_t first;  // the coefficient of product row n in an entry's
    u32x4 qx[NK][8], ox[NV][8];
    f32x4v dk[NK][8], dv[NV][8];

    __device__ __forceinline__ ColSums(const BwdArgs &a_, const Slab &b_, int slab)
        : a(a_), b(b_), n(threadIdx.x % 16), g(threadIdx.x % kWave / 16), kv0(slab * b_.hs),
          hsl(min(b_.hs, a_.s.Hk - slab * b_.hs)), lhs(b_.hs == 1 ? 0 : b_.hs == 2 ? 1 : 2),
          qc(n, hsl * 2 * a_.s.d), oc(n, hsl * a_.s.dv) {
        const int d2 = 2 * a.s.d, dv1 = a.s.dv, grp = a.s.grp;
#pragma unroll
        for (int v = 0; v < NK; ++v) {
            qh[v] = b.hs == 1 ? 0 : qc.off[v] / d2;
            qcol[v] = qc.off[v] - qh[v] * d2;
            qc.off[v] = (kv0 + qh[v]) * grp * d2 + qcol[v];
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            oh[v] = b.hs == 1 ? 0 : oc.off[v] / dv1;
            ocol[v] = oc.off[v] - oh[v] * dv1;
            oc.off[v] = (kv0 + oh[v]) * grp * dv1 + ocol[v];
        }
        const int head = n / 4 & ((1 << lhs) - 1);
        weighs = head < hsl && n % 4 != 3;
        first = (int64_t)(kv0 + min(head, hsl - 1)) * grp * 4 + n % 4;
    }
    // The column (within a group) of product row n's pair.
    __device__ __forceinline__ int sub() const { return n / 4 >> lhs; }

    __device__ __forceinline__ void positions(const Tile &c, int (&pos)[8]) const {
#pragma unroll
        for (int t = 0; t < 8; ++t) pos[t] = c.in(g, t) ? a.perm[c.entry(g, t)] : 0;
    }
    // Weights of query head gi of each key head.
    __device__ __forceinline__ void load_weights(const Tile &c, const int (&pos)[8], int gi,
                                                 float (&w)[8]) const {
        const float *C = a.coef + first + gi * 4;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            w[t] = 0.f;
            if (weighs && c.in(g, t)) w[t] = C[(int64_t)pos[t] * a.s.H * 4];
        }
    }
    __device__ __forceinline__ void load_q(int idx, bool two, int gi) {
        qc.load(static_cast<const bf16_t *>(a.Q) + (int64_t)gi * 2 * a.s.d, a.s.ldq, idx, g, two,
                qx);
    }
    __device__ __forceinline__ void load_o(int idx, bool two, int gi) {
        oc.load(static_cast<const bf16_t *>(a.dO) + (int64_t)gi * a.s.dv, a.s.ldo, idx, g, two,
                ox);
    }
    __device__ __forceinline__ void reset() {
        clear(dk);
        clear(dv);
    }
    __device__ __forceinline__ bool tainted() const {
        const float z = taint(dk) + taint(dv);
        return __any(z != z);
    }
    // The entries [p, end) of a column again, by itself; one whose key is masked (its
    // last coefficient is 0) brings nothing, whatever its row holds.
    __device__ __forceinline__ void walk_apart(int col, int p, int end, int at) {
        const Tile c = row_tile(col, p, end);
        reset();
        for (; p < end; p += min(32, end - p)) {
            Tile t = alone(a.other, nullptr, p, end, sub() == 0);
            const int64_t pos32 = a.perm[p + min((int)(threadIdx.x % 32), end - 1 - p)];
            const float live = a.coef[(pos32 * a.s.H + kv0 * a.s.grp) * 4 + 3];
            t.used &= (uint32_t)__ballot(live != 0.f);
            if (t.used == 0) continue;
            const int idx = stand_in(t.idx, t.used);
            int pos[8];
            positions(t, pos);
            for (int gi = 0; gi < a.s.grp; ++gi) {
                float w[8];
                load_weights(t, pos, gi, w);
                load_q(idx, true, gi);
                load_o(idx, true, gi);
                drop_unused(qx, g, t.used);
                drop_unused(ox, g, t.used);
                const Weights parts(w);
                weigh(qx, parts, dk);
                weigh(ox, parts, dv);
            }
        }
        finish(c, at);
    }

    // The group's columns, or partial `at`.
    __device__ __forceinline__ void finish(const Tile &c, int at) const {
        const int r = g >> lhs, head = g & ((1 << lhs) - 1), d2 = 2 * a.s.d;
        const bool has = c.has(r);
        if (!has || head >= hsl) return;
        const int64_t col = c.row0 + r, kv = kv0 + head;
        float *part = a.part + ((int64_t)at * a.s.Hk + kv) * (d2 + a.s.dv);
        bf16_t *K = static_cast<bf16_t *>(a.dK) + col * a.s.ldk + kv * d2;
        bf16_t *V = static_cast<bf16_t *>(a.dV) + col * a.s.ldv + kv * a.s.dv;
#pragma unroll
        for (int v = 0; v < NK; ++v) {
            if (!qc.on[v] || qh[v] != head) continue;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                o[j] = (qcol[v] + j < a.s.d ? dk[v][j][0] : dk[v][j][2]) * a.s.scale;
            if (at >= 0) store_values<float, 8>(part + qcol[v], o);
            else store_values<bf16_t, 8>(K + qcol[v], o);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!oc.on[v] || oh[v] != head) continue;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = dv[v][j][1];
            if (at >= 0) store_values<float, 8>(part + d2 + ocol[v], o);
            else store_values<bf16_t, 8>(V + ocol[v], o);
        }
    }
};

template <int NK, int NV>
__global__ __launch_bounds__(kAttnThreads, NK * NV == 1 ? 2 : 1) void mfma_col_kernel(
    BwdArgs a, Slab b) {
    if ((int64_t)blockIdx.x >= a.nmain) {
        for_empty(a.plan, a.nseg, a.all_empty, a.nmain,
                  [&](int64_t col) { empty_column<bf16_t>(a, col); });
        return;
    }
    const Unit u(a.nmain, b.nslab);
    if (u.item >= a.plan.nitems) return;
    ColSums<NK, NV> f(a, b, u.slab);
    const int chunk = a.plan.nchunks > 0 ? a.plan.chunk_ord[u.item] : -1, grp = a.s.grp;
    Walk walk(a.other, a.idx, a.ptr, nullptr, a.nseg, 4 >> f.lhs, f.sub(), a.bias == nullptr);
    walk.begin(a.plan.item_ptr[u.item], a.plan.item_ptr[u.item + 1]);
    // a tile is taken once for every query head of a key head
    Tile c = walk.make(), n = c;
    int pos[8], npos[8], idx = stand_in(c.idx, c.used), nidx = idx, gi = 0;
    float w[8];
    f.positions(c, pos);
    f.load_weights(c, pos, 0, w);
    f.load_q(idx, c.used >> 16 != 0, 0);
    f.load_o(idx, c.used >> 16 != 0, 0);
    f.reset();
    bool more = !walk.done, bad = false;
    if (more) n = walk.make();
    while (true) {
        const Weights parts(w);
        const bool turn = gi + 1 == grp;  // to the next tile
        const int ngi = turn ? 0 : gi + 1;
        const bool go = !turn || more;
        if (turn && more) {
            f.positions(n, npos);
            nidx = stand_in(n.idx, n.used);
        }
        const bool two = (turn ? n.used : c.used) >> 16 != 0;
        const int at = turn ? nidx : idx;
        weigh(f.qx, parts, f.dk);
        if (go) f.load_q(at, two, ngi);
        weigh(f.ox, parts, f.dv);
        if (go) f.load_o(at, two, ngi);
        if (go) {
            if (turn) f.load_weights(n, npos, 0, w);
            else f.load_weights(c, pos, ngi, w);
        }
        if (turn && c.last) {
            bad |= f.tainted();
            f.finish(c, chunk);
            f.reset();
        }
        if (!go) break;
        gi = ngi;
        if (!turn) continue;
        c = n;
        idx = nidx;
#pragma unroll
        for (int t = 0; t < 8; ++t) pos[t] = npos[t];
        more = !walk.done;
        if (more) n = walk.make();
    }
    if (!bad) return;
    for_rows(a.idx, a.ptr, a.plan.item_ptr[u.item], walk.b0,
             [&](int col, int p, int end) { f.walk_apart(col, p, end, chunk); });
}

// ------------------------------------------------------------ dispatch

template <int N>
using Int = std::integral_constant<int, N>;

// Chunks of 32 key columns and groups of 128 value columns that a slab needs.
template <class F>
void with_cols(const Slab &b, F f) {
    if (b.nv == 1) {
        if (b.nc == 1) f(Int<1>(), Int<1>());
        else if (b.nc == 2) f(Int<2>(), Int<1>());
        else if (b.nc == 4) f(Int<4>(), Int<1>());
        else f(Int<8>(), Int<1>());
    } else {
        if (b.nc == 8) f(Int<8>(), Int<2>());
        else f(Int<4>(), Int<2>());
    }
}

}  // namespace

// Which form is faster, by the query heads of a key head.  Measured at 4M entries,
// dv = 2 d, the vector form / this one, us, forward and gradient:
//   heads      a random 60 a row        a window of 32          a window of 256
//   8 over 4, d = 64
//          1453/1329  4588/5273    1283/582  3900/3420     931/428  2800/2303
//   16 over 4, d = 32
//          1282/716   5240/4486    1173/705  4873/3973     929/410  2869/2383
//   4 over 4, d = 64
//          1076/1442  2479/4181     645/396  1910/2063     492/631  1386/2221
//   8 over 8, d = 16
//           549/671   1373/2149     294/585  1145/2087     259/432   750/1646
// One query head a key head leaves half the product rows empty, and the backward
// passes have as many coefficients: the vector form, on windows too (but for a
// narrow one at d = 64).  From two on this one; where it loses is a gradient of
// two heads without shared columns, and slabs of few columns (4 over 2, d = 16:
// 214/250 and 1140/1295 at 60 a row).
bool cores_pay(const nsd_attn *s) { return fits_cores(s) && s->heads >= 2 * s->kv_heads; }

Slab make_slab(const nsd_attn *s) {
    const int grp = s->heads / s->kv_heads;
    Slab b;
    b.hs = 1;
    b.nsub = (int32_t)ceil_div(grp, 8);
    // heads whose columns are whole 16-byte pieces lie side by side; four at most,
    // one for each group of lanes in the column pass
    if (s->d % 8 == 0 && s->dv % 8 == 0)
        while (b.hs < 4 && b.hs < s->kv_heads && (b.hs + 1) * grp <= 8 &&
               (b.hs + 1) * std::max(2 * s->d, s->dv) <= 128)
            ++b.hs;
    const int D = b.hs * 2 * s->d, W = b.hs * s->dv;
    b.nv = W <= 128 ? 1 : 2;
    b.nc = 1;
    while (32 * b.nc < D) b.nc *= 2;
    if (b.nv == 2) b.nc = std::max(b.nc, 4);
    b.full = s->d % 8 == 0 && D == 32 * b.nc && s->kv_heads % b.hs == 0;
    b.nslab = (int32_t)ceil_div(s->kv_heads, b.hs) * b.nsub;
    b.lrh = 0;
    while (1 << b.lrh < std::min(b.hs * grp, 8)) ++b.lrh;
    return b;
}

Slab one_row(Slab b) {
    b.lrh = 3;
    return b;
}

Slab column_slab(Slab b) {
    b.nslab /= b.nsub;
    b.nsub = 1;
    return b;
}

int64_t mfma_blocks(int64_t items, const Slab &b) {
    return ceil_div(items, kAttnWaves) * b.nslab;
}

void mfma_forward(const FwdArgs &a, const Slab &b, int64_t blocks, bool decode, hipStream_t st) {
    with_cols(b, [&](auto NC, auto NV) {
        const dim3 g((unsigned)blocks), t(kAttnThreads);
        if (decode) {
            if (b.full) mfma_fwd_kernel<NC(), NV(), true, true><<<g, t, 0, st>>>(a, b);
            else mfma_fwd_kernel<NC(), NV(), false, true><<<g, t, 0, st>>>(a, b);
        } else {
            if (b.full) mfma_fwd_kernel<NC(), NV(), true, false><<<g, t, 0, st>>>(a, b);
            else mfma_fwd_kernel<NC(), NV(), false, false><<<g, t, 0, st>>>(a, b);
        }
    });
}

void mfma_rows(const BwdArgs &a, const Slab &b, int64_t blocks, hipStream_t st) {
    const dim3 t(kAttnThreads);
    with_cols(b, [&](auto NC, auto NV) {
        const dim3 g((unsigned)blocks);
        if (b.full) mfma_weight_kernel<NC(), NV(), true><<<g, t, 0, st>>>(a, b);
        else mfma_weight_kernel<NC(), NV(), false><<<g, t, 0, st>>>(a, b);
    });
    if (a.nmain == 0) return;
    const unsigned nlong = (unsigned)a.plan.nlong;
    if (nlong > 0) mfma_join_D_kernel<<<nlong, 64, 0, st>>>(a);
    const dim3 g((unsigned)a.nmain);
    if (b.nc == 8) mfma_row_kernel<2><<<g, t, 0, st>>>(a, b);
    else mfma_row_kernel<1><<<g, t, 0, st>>>(a, b);
    if (nlong > 0) mfma_join_row_kernel<<<nlong * a.s.H, kAttnThreads, 0, st>>>(a);
}

void mfma_columns(const BwdArgs &a, const Slab &b, int64_t blocks, hipStream_t st) {
    const dim3 g((unsigned)blocks), t(kAttnThreads);
    if (b.nc == 8 && b.nv == 2) mfma_col_kernel<2, 2><<<g, t, 0, st>>>(a, b);
    else if (b.nc == 8) mfma_col_kernel<2, 1><<<g, t, 0, st>>>(a, b);
    else if (b.nv == 2) mfma_col_kernel<1, 2><<<g, t, 0, st>>>(a, b);
    else mfma_col_kernel<1, 1><<<g, t, 0, st>>>(a, b);
}

}  // namespace attn
}  // namespace nsd
