// One step of AdamW over many tensors in one launch, its two states per weight
// held in 32 bits or in 8.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   w = w (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
//
// HBM-bound: every array is read and written once (200M weights in bf16 with
// 32-bit copies: 1.02 ms, 5.3 TB/s; with 8-bit states and no copies 420 to 430
// us, 4.5 TB/s).  With 8-bit states the instructions are as close: steps without
// a pause between them draw the engine clock from 2.1 GHz to 1.6 for some ten of
// them, and take up to 650 us there, 460 after forty.
// The tensors' entries are cut into chunks of kChunk, one workgroup each, found
// through a list that the plan holds, so that tensors of one value and of
// billions share a launch and a step has no pass over the host's list.  A wave
// takes 256 consecutive entries, a lane four of them: the 256 are also what
// shares a scale in the 8-bit states, so that the largest of a block is one
// butterfly of a wave.
//
// States in 8 bits: m as e4m3 and v as e5m2, each over a 32-bit scale that
// takes the block's largest value to the format's largest.  A value is rounded
// to one of its two neighbours at random, up with the probability that keeps
// its mean.  To nearest, a state whose step is smaller than half a code's
// distance (v moves by 1 - b2 of its distance to g^2, and codes of v lie a
// quarter of their value apart) would never move.  e5m2's range, 2^31 down
// from the block's largest, keeps every v whose square root is more than 2^-16
// of the largest; one that is not zero is not rounded to zero (but with its whole
// block, at a scale below 2^-126), which would leave a step of m / eps.  The
// random bits are a hash of the step, the tensor and the entry: a step is
// reproducible, and needs no generator's state.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>
#include <type_traits>

#include "nsd_internal.hpp"

namespace nsd {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kStateBlock = NSD_ADAMW_BLOCK;
constexpr int kPer = 4;  // entries per lane and block
constexpr int kChunkBlocks = 16;
constexpr int64_t kChunk = kChunkBlocks * kStateBlock;
static_assert(kStateBlock == kPer * kWave, "a wave takes one block of states");

// What a workgroup needs of its tensor.
struct AdamTensor {
    void *p;
    float *master;
    const void *g;
    void *m, *v;
    float *m_scale, *v_scale;
    int32_t n;
    float wd;
    int32_t kind;  // Kind
    int32_t pad;
};
struct AdamChunk {
    int32_t tensor, first;  // the tensor, and the first entry in it
};

// Types of the weights (with or without a 32-bit copy) and of the gradients.
enum Kind { kF32 = 0, kBf16 = 1, kCopied = 2, kKinds = 3 };

struct AdamScalars {
    float b1, c1, b2, c2;  // b and 1 - b
    float eps, lr;
    float log_b1, log_b2;
    float rate, root;  // lr / (1 - b1^t) and 1 / sqrt(1 - b2^t), for t of the host
    uint32_t step;
    const int32_t *step_dev;
    const float *lr_dev, *grad_scale;
};

typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32a1 __attribute__((aligned(1)));

// An address read from the table, known to be of global memory: accesses
// through a plain pointer would be flat ones, which wait for LDS as well.
template <class T>
using Global = __attribute__((address_space(1))) T *;
template <class T, class U>
__device__ __forceinline__ Global<T> global(U *p) {
    return (Global<T>)p;
}

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float from_bf16(uint32_t b) { return __uint_as_float(b << 16); }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return from_bf16(x); }

// Four consecutive values from entry i of an array; entries past the end
// (`left` are there) read 0 and are not written.  FULL: all four exist.
template <bool FULL, class T>
__device__ __forceinline__ void load4(const void *q, int64_t i, int left, float (&x)[kPer]) {
    using V = std::conditional_t<sizeof(T) == 4, f32x4, u16x4>;
    if (FULL) {
        const V t = *global<const V>(static_cast<const T *>(q) + i);
        x[0] = widen((T)t.x); x[1] = widen((T)t.y); x[2] = widen((T)t.z); x[3] = widen((T)t.w);
    } else {
        const auto p = global<const T>(static_cast<const T *>(q) + i);
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = e < left ? widen((T)p[e]) : 0.f;
    }
}
template <bool FULL, class T>
__device__ __forceinline__ void store4(void *q, int64_t i, int left, const T (&x)[kPer]) {
    using V = std::conditional_t<sizeof(T) == 4, f32x4, u16x4>;
    if (FULL) {
        const V t = {x[0], x[1], x[2], x[3]};
        *global<V>(static_cast<T *>(q) + i) = t;
    } else {
        const auto p = global<T>(static_cast<T *>(q) + i);
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (e < left) p[e] = x[e];
    }
}
template <bool FULL>
__device__ __forceinline__ uint32_t load_codes(const void *q, int64_t i, int left) {
    const auto p = global<const uint8_t>(static_cast<const uint8_t *>(q) + i);
    if (FULL) return *(Global<const u32a1>)p;
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < left) c |= (uint32_t)p[e] << (8 * e);
    return c;
}
template <bool FULL>
__device__ __forceinline__ void store_codes(void *q, int64_t i, int left, uint32_t c) {
    const auto p = global<uint8_t>(static_cast<uint8_t *>(q) + i);
    if (FULL) {
        *(Global<u32a1>)p = c;
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (e < left) p[e] = (uint8_t)(c >> (8 * e));
    }
}

// A product and a sum that are rounded by themselves (no fused multiply-add).
__device__ __forceinline__ float mul_r(float x, float y) {
#pragma clang fp contract(off)
    return x * y;
}
__device__ __forceinline__ float add_r(float x, float y) {
#pragma clang fp contract(off)
    return x + y;
}

// Largest of a wave, in every lane (NaN is left out: its own code says it).
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, lane_xor<1>(x));
    x = fmaxf(x, lane_xor<2>(x));
    x = fmaxf(x, lane_xor<4>(x));
    x = fmaxf(x, lane_xor<8>(x));
    x = fmaxf(x, lane_xor<16>(x));
    return fmaxf(x, lane_xor<32>(x));
}

// The block's scale and its inverse (0: every value is below 2^-126 / top).
__device__ __forceinline__ float block_scale(const float (&x)[kPer], float inv_top, float &inv) {
    const float top = wave_max(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])),
                                     fmaxf(fabsf(x[2]), fabsf(x[3]))));
    const float s = top * inv_top;
    const bool zero = s < 0x1p-126f;
    inv = zero ? 0.f : 1.f / s;
    return zero ? 0.f : s;
}

// y >= 0 to a code of MANT mantissa bits, smallest normal 2^LOW, largest code
// MAX: the bits that the code drops carry into those it keeps by 16 random ones
// (and half a unit of those).  Below the smallest normal, codes are 2^(LOW -
// MANT) apart (a second moment's at least the first, where it is not zero), and
// NaN becomes the format's: all so rare (a ten-thousandth of a normal
// distribution's m) that a wave takes them apart (200M weights: 70 of
// 476 us saved, the step being bound by its instructions).
template <int MANT, int LOW, uint32_t MAX>
__device__ __forceinline__ void encode(const float (&y)[kPer], const uint32_t (&rnd)[kPer],
                                       uint32_t (&code)[kPer]) {
    constexpr int DROP = 23 - MANT;
    constexpr float kLow = MANT == 3 ? 0x1p-6f : 0x1p-14f;
    bool rare = false;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const uint32_t carry = (rnd[e] << (DROP - 16)) | (1u << (DROP - 17));
        const uint32_t t = __float_as_uint(y[e]) + carry - ((uint32_t)(126 + LOW) << 23);
        code[e] = min(t >> DROP, MAX);
        rare |= !(y[e] >= kLow);
    }
    if (!__any(rare)) return;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const float frac = ((float)rnd[e] + 0.5f) * 0x1p-16f;
        constexpr float kSub = MANT == 3 ? 512.f : 65536.f;
        const uint32_t small = (uint32_t)(int)floorf(add_r(y[e] * kSub, frac));
        code[e] = y[e] < kLow ? min(small, MAX) : code[e];
        if (MANT == 2) code[e] = y[e] > 0.f ? max(code[e], 1u) : code[e];
        code[e] = y[e] == y[e] ? code[e] : 0x7Fu;
    }
}

// Four values' codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t encode_m(const float (&x)[kPer], float inv,
                                             const uint32_t (&rnd)[kPer]) {
    float y[kPer];
    uint32_t r[kPer], c[kPer], out = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        y[e] = mul_r(fabsf(x[e]), inv);
        r[e] = rnd[e] & 0xFFFFu;
    }
    encode<3, -6, 0x7Eu>(y, r, c);
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        out |= (c[e] | (__float_as_uint(x[e]) >> 24 & 0x80u)) << (8 * e);
    return out;
}
__device__ __forceinline__ uint32_t encode_v(const float (&x)[kPer], float inv,
                                             const uint32_t (&rnd)[kPer]) {
    float y[kPer];
    uint32_t r[kPer], c[kPer], out = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        y[e] = mul_r(x[e], inv);
        r[e] = rnd[e] >> 16;
    }
    encode<2, -14, 0x7Bu>(y, r, c);
#pragma unroll
    for (int e = 0; e < kPer; ++e) out |= c[e] << (8 * e);
    return out;
}

__device__ __forceinline__ void decode_m(uint32_t c, float (&x)[kPer]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    x[0] = lo.x; x[1] = lo.y; x[2] = hi.x; x[3] = hi.y;
}
__device__ __forceinline__ void decode_v(uint32_t c, float (&x)[kPer]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)c, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)c, true);
    x[0] = lo.x; x[1] = lo.y; x[2] = hi.x; x[3] = hi.y;
}

struct StepScalars {
    float lr, rate, root, gscale;
    uint32_t key;
};

// One block of 256 entries (fewer at a tensor's end), one wave.
template <int KIND, class G, bool EIGHT, bool FULL>
__device__ __forceinline__ void adam_block(const AdamTensor &t, const AdamScalars &a,
                                           const StepScalars &s, int64_t i, int left) {
    using P = std::conditional_t<KIND == kF32, float, uint16_t>;
    float g[kPer], w[kPer], m[kPer], v[kPer];
    const int64_t blk = i / kStateBlock;  // the same in every lane of the wave
    load4<FULL, G>(t.g, i, left, g);
    if constexpr (KIND == kCopied) load4<FULL, float>(t.master, i, left, w);
    else load4<FULL, P>(t.p, i, left, w);
    float sm = 1.f, sv = 1.f;
    if constexpr (EIGHT) {
        sm = global<const float>(t.m_scale)[blk];
        sv = global<const float>(t.v_scale)[blk];
        decode_m(load_codes<FULL>(t.m, i, left), m);
        decode_v(load_codes<FULL>(t.v, i, left), v);
    } else {
        load4<FULL, float>(t.m, i, left, m);
        load4<FULL, float>(t.v, i, left, v);
    }
    const float decay = s.lr * t.wd;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        // each product and sum of the states rounded by itself: what a block's
        // codes are then follows from the inputs alone
        const float gr = mul_r(g[e], s.gscale);
        if constexpr (EIGHT) {
            m[e] = mul_r(m[e], sm);
            v[e] = mul_r(v[e], sv);
        }
        m[e] = add_r(mul_r(m[e], a.b1), mul_r(gr, a.c1));
        v[e] = add_r(mul_r(v[e], a.b2), mul_r(mul_r(gr, a.c2), gr));
    }
    // the root and the quotient to one unit in the last place; the hardware's root
    // takes normal numbers, smaller ones are scaled
    float sq[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) sq[e] = __builtin_amdgcn_sqrtf(v[e]);
    if (__any(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < 0x1p-126f)) {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (v[e] < 0x1p-126f) sq[e] = __builtin_amdgcn_sqrtf(v[e] * 0x1p32f) * 0x1p-16f;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        // the decay joins the step and both leave the weight at once: 1 - lr wd,
        // rounded by itself, is off by up to 2^-25, the same way at every step.  (An
        // infinite weight stays so.)
        const float den = sq[e] * s.root + a.eps;
        const float step = s.rate * (m[e] * __builtin_amdgcn_rcpf(den));
        const float held = __builtin_amdgcn_fmed3f(w[e], -FLT_MAX, FLT_MAX);
        w[e] -= __builtin_fmaf(held, decay, step);
    }
    uint32_t rnd[kPer];
    if constexpr (EIGHT || KIND == kBf16) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) rnd[e] = mix32((uint32_t)(i + e) * 0x9E3779B1u + s.key);
    }
    if constexpr (EIGHT) {
        float im, iv;
        sm = block_scale(m, 1.f / 448.f, im);
        sv = block_scale(v, 1.f / 57344.f, iv);
        store_codes<FULL>(t.m, i, left, encode_m(m, im, rnd));
        store_codes<FULL>(t.v, i, left, encode_v(v, iv, rnd));
        if (threadIdx.x % kWave == 0) {
            global<float>(t.m_scale)[blk] = sm;
            global<float>(t.v_scale)[blk] = sv;
        }
    } else {
        store4<FULL, float>(t.m, i, left, m);
        store4<FULL, float>(t.v, i, left, v);
    }
    if constexpr (KIND == kF32) {
        store4<FULL, float>(t.p, i, left, w);
    } else {
        uint16_t b[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if constexpr (KIND == kCopied) {  // the copy keeps what nearest drops
                const __bf16 r = static_cast<__bf16>(w[e]);
                b[e] = __builtin_bit_cast(uint16_t, r);
            } else {  // at random: a step is mostly below half a unit of bf16
                const uint32_t u = __float_as_uint(w[e]) +
                                   (mix32(rnd[e] ^ 0x9E3779B1u) & 0xFFFFu);
                b[e] = w[e] == w[e] ? (uint16_t)(u >> 16) : (uint16_t)0x7FC0u;
            }
        }
        store4<FULL, uint16_t>(t.p, i, left, b);
        if constexpr (KIND == kCopied) store4<FULL, float>(t.master, i, left, w);
    }
}

template <int KIND, class G, bool EIGHT>
__device__ __forceinline__ void adam_chunk(const AdamTensor &t, const AdamScalars &a,
                                           const StepScalars &s, int64_t first) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t end = min(first + kChunk, (int64_t)t.n);
    for (int64_t b = first + wave * kStateBlock; b < end;
         b += kAdamThreads / kWave * kStateBlock) {
        const int64_t i = b + lane * kPer;
        if (b + kStateBlock <= t.n) adam_block<KIND, G, EIGHT, true>(t, a, s, i, kPer);
        else adam_block<KIND, G, EIGHT, false>(t, a, s, i, (int)max((int64_t)t.n - i, (int64_t)0));
    }
}

template <bool EIGHT>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(
    const AdamTensor *__restrict__ tensors, const AdamChunk *__restrict__ chunks, AdamScalars a) {
    const AdamChunk c = chunks[blockIdx.x];
    const AdamTensor t = tensors[c.tensor];
    StepScalars s;
    s.lr = a.lr_dev ? *a.lr_dev : a.lr;
    s.gscale = a.grad_scale ? *a.grad_scale : 1.f;
    uint32_t step = a.step;
    s.rate = a.rate;
    s.root = a.root;
    if (a.step_dev) {
        step = (uint32_t)*a.step_dev;
        s.root = 1.f / sqrtf(-expm1f((float)step * a.log_b2));
    }
    if (a.step_dev || a.lr_dev) s.rate = s.lr / -expm1f((float)step * a.log_b1);
    s.key = mix32(step * 0x9E3779B1u + (uint32_t)c.tensor);
    switch (t.kind) {
        case kF32: adam_chunk<kF32, float, EIGHT>(t, a, s, c.first); break;
        case kBf16: adam_chunk<kBf16, float, EIGHT>(t, a, s, c.first); break;
        case kCopied: adam_chunk<kCopied, float, EIGHT>(t, a, s, c.first); break;
        case kKinds + kF32: adam_chunk<kF32, uint16_t, EIGHT>(t, a, s, c.first); break;
        case kKinds + kBf16: adam_chunk<kBf16, uint16_t, EIGHT>(t, a, s, c.first); break;
        case kKinds + kCopied: adam_chunk<kCopied, uint16_t, EIGHT>(t, a, s, c.first); break;
    }
}

nsd_status check_tensors(int32_t n, const nsd_adamw_tensor *ts, int32_t state_bits,
                         int64_t *chunks) {
    NSD_REQUIRE(n >= 0, "negative number of tensors");
    NSD_REQUIRE(n == 0 || ts != nullptr, "tensors is NULL");
    NSD_REQUIRE(state_bits == 8 || state_bits == 32, "states of %d bits (8 or 32)", state_bits);
    *chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        const nsd_adamw_tensor &t = ts[i];
        NSD_REQUIRE(t.n >= 0, "tensor %d: negative length", i);
        if (t.n > INT32_MAX - kChunk)
            return fail(NSD_ERR_TOO_LARGE, "tensor %d: %lld values", i, (long long)t.n);
        NSD_REQUIRE((t.param_dtype == NSD_F32 || t.param_dtype == NSD_BF16) &&
                        (t.grad_dtype == NSD_F32 || t.grad_dtype == NSD_BF16),
                    "tensor %d: unknown type", i);
        NSD_REQUIRE(t.master == nullptr || t.param_dtype == NSD_BF16,
                    "tensor %d: a 32-bit copy of 32-bit weights", i);
        NSD_REQUIRE(t.n == 0 || (t.param && t.grad && t.m && t.v), "tensor %d: a NULL array", i);
        NSD_REQUIRE(t.n == 0 || state_bits == 32 || (t.m_scale && t.v_scale),
                    "tensor %d: 8-bit states without scales", i);
        *chunks += ceil_div(t.n, kChunk);
    }
    // a launch's threads are counted in 32 bits
    if (*chunks > UINT32_MAX / kAdamThreads)
        return fail(NSD_ERR_TOO_LARGE, "%lld chunks", (long long)*chunks);
    return NSD_OK;
}

// An array of a tensor: its bytes, and whether a step writes it.
struct AdamArray {
    uintptr_t lo, hi;
    int32_t tensor;
    bool written;
};

// No array that a step writes may share memory with another: workgroups take
// them in any order.  (Gradients may share theirs.)
nsd_status check_apart(int32_t n, const nsd_adamw_tensor *ts, int32_t state_bits) {
    if (n == 0) return NSD_OK;
    constexpr int kArrays = 7;
    AdamArray *all = static_cast<AdamArray *>(std::malloc((size_t)n * kArrays * sizeof(AdamArray)));
    if (all == nullptr) return fail(NSD_ERR_HIP, "no host memory for %d tensors", n);
    size_t count = 0;
    for (int32_t i = 0; i < n; ++i) {
        const nsd_adamw_tensor &t = ts[i];
        auto add = [&](const void *p, int64_t values, int64_t bytes, bool written) {
            const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
            if (p && values > 0) all[count++] = {lo, lo + (uintptr_t)(values * bytes), i, written};
        };
        const int64_t state = state_bits / 8;
        add(t.param, t.n, t.param_dtype == NSD_BF16 ? 2 : 4, true);
        add(t.master, t.n, 4, true);
        add(t.grad, t.n, t.grad_dtype == NSD_BF16 ? 2 : 4, false);
        add(t.m, t.n, state, true);
        add(t.v, t.n, state, true);
        if (state_bits == 8) {
            add(t.m_scale, ceil_div(t.n, kStateBlock), 4, true);
            add(t.v_scale, ceil_div(t.n, kStateBlock), 4, true);
        }
    }
    std::sort(all, all + count, [](const AdamArray &x, const AdamArray &y) { return x.lo < y.lo; });
    // of the arrays before, the one that ends last, and the one that is written
    size_t any = 0, written = count, a = count, b = count;
    for (size_t i = 0; i < count && a == count; ++i) {
        if (written < count && all[i].lo < all[written].hi) a = written, b = i;
        else if (i > 0 && all[i].written && all[i].lo < all[any].hi) a = any, b = i;
        if (i > 0 && all[i].hi > all[any].hi) any = i;
        if (all[i].written && (written == count || all[i].hi > all[written].hi)) written = i;
    }
    const int32_t ta = a < count ? all[a].tensor : -1, tb = b < count ? all[b].tensor : -1;
    std::free(all);
    NSD_REQUIRE(ta < 0, "arrays of tensors %d and %d share memory that a step writes", ta, tb);
    return NSD_OK;
}

// Table: the tensors' records, then the chunks' (device and host alike).
size_t table_bytes(int32_t n, int64_t chunks) {
    return (size_t)n * sizeof(AdamTensor) + (size_t)chunks * sizeof(AdamChunk);
}

}  // namespace

}  // namespace nsd

using namespace nsd;

extern "C" {

nsd_status nsd_adamw_plan_size(int32_t ntensors, const nsd_adamw_tensor *tensors, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_REQUIRE(ntensors >= 0, "negative number of tensors");
    NSD_REQUIRE(ntensors == 0 || tensors != nullptr, "tensors is NULL");
    int64_t chunks = 0;
    for (int32_t i = 0; i < ntensors; ++i) {
        NSD_REQUIRE(tensors[i].n >= 0, "tensor %d: negative length", i);
        chunks += ceil_div(tensors[i].n, kChunk);
    }
    *bytes = std::max<size_t>(table_bytes(ntensors, chunks), 256);
    return NSD_OK;
}

nsd_status nsd_adamw_plan_build(int32_t ntensors, const nsd_adamw_tensor *tensors,
                                int32_t state_bits, nsd_adamw_plan *plan, void *table,
                                size_t table_size, void *stream) {
    NSD_REQUIRE(plan != nullptr, "plan is NULL");
    int64_t nchunks;
    NSD_TRY(check_tensors(ntensors, tensors, state_bits, &nchunks));
    const size_t need = table_bytes(ntensors, nchunks);
    if (need > 0 && (table == nullptr || table_size < need))
        return fail(NSD_ERR_WORKSPACE, "table %zu bytes at %p, need %zu", table_size, table, need);
    NSD_REQUIRE((reinterpret_cast<uintptr_t>(table) & 7) == 0, "table is not 8-byte aligned");
    NSD_TRY(check_apart(ntensors, tensors, state_bits));
    if (need > 0) {
        char *host = static_cast<char *>(std::malloc(need));
        if (host == nullptr) return fail(NSD_ERR_HIP, "no host memory for %zu bytes", need);
        AdamTensor *ts = reinterpret_cast<AdamTensor *>(host);
        AdamChunk *cs = reinterpret_cast<AdamChunk *>(host + (size_t)ntensors * sizeof(AdamTensor));
        for (int32_t i = 0; i < ntensors; ++i) {
            const nsd_adamw_tensor &t = tensors[i];
            const int kind = t.param_dtype == NSD_F32 ? kF32 : t.master ? kCopied : kBf16;
            ts[i] = AdamTensor{t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale,
                               (int32_t)t.n, t.weight_decay,
                               kind + (t.grad_dtype == NSD_BF16 ? kKinds : 0), 0};
            for (int64_t b = 0; b < t.n; b += kChunk) *cs++ = AdamChunk{i, (int32_t)b};
        }
        hipError_t e = hipMemcpyAsync(table, host, need, hipMemcpyHostToDevice, as_stream(stream));
        if (e == hipSuccess) e = hipStreamSynchronize(as_stream(stream));
        std::free(host);
        NSD_TRY(check_hip(e, "copy of the tensor table"));
    }
    plan->ntensors = ntensors;
    plan->nchunks = (int32_t)nchunks;
    plan->state_bits = state_bits;
    plan->table = table;
    return NSD_OK;
}

nsd_status nsd_adamw_step(const nsd_adamw_plan *plan, const nsd_adamw *h, void *stream) {
    NSD_REQUIRE(plan != nullptr && h != nullptr, "plan or hyperparameters are NULL");
    NSD_REQUIRE(plan->nchunks >= 0 && plan->ntensors >= 0 &&
                    (plan->state_bits == 8 || plan->state_bits == 32) &&
                    (plan->nchunks == 0 || plan->table),
                "plan is not built (nsd_adamw_plan_build)");
    NSD_REQUIRE(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1,
                "beta %g, %g outside [0, 1)", h->beta1, h->beta2);
    NSD_REQUIRE(h->eps >= 1e-30 && std::isfinite(h->eps), "eps %g below 1e-30", h->eps);
    NSD_REQUIRE(h->lr_dev || std::isfinite(h->lr), "lr is not finite");
    NSD_REQUIRE(h->step_dev || h->step >= 1, "step %d (the first step is 1)", h->step);
    if (plan->nchunks == 0) return NSD_OK;
    AdamScalars a;
    a.b1 = (float)h->beta1;
    a.c1 = (float)(1.0 - h->beta1);
    a.b2 = (float)h->beta2;
    a.c2 = (float)(1.0 - h->beta2);
    a.eps = (float)h->eps;
    a.lr = (float)h->lr;
    a.log_b1 = (float)std::log(h->beta1);
    a.log_b2 = (float)std::log(h->beta2);
    const int32_t t = h->step_dev ? 1 : h->step;
    a.rate = (float)(h->lr / (1.0 - std::pow(h->beta1, t)));
    a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t)));
    a.step = (uint32_t)t;
    a.step_dev = h->step_dev;
    a.lr_dev = h->lr_dev;
    a.grad_scale = h->grad_scale;
    const AdamTensor *ts = static_cast<const AdamTensor *>(plan->table);
    const AdamChunk *cs = reinterpret_cast<const AdamChunk *>(ts + plan->ntensors);
    if (plan->state_bits == 8)
        adamw_kernel<true><<<plan->nchunks, kAdamThreads, 0, as_stream(stream)>>>(ts, cs, a);
    else
        adamw_kernel<false><<<plan->nchunks, kAdamThreads, 0, as_stream(stream)>>>(ts, cs, a);
    return check_launch("adamw_kernel");
}

}  // extern "C"
