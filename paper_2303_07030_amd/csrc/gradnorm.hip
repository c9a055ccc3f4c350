// The norm of many tensors' gradients and the factor that clips them.
//
//   norm = |f| sqrt(sum g^2) or the largest |f g|,  scale = f min(1, max / (norm + 1e-6))
//
// HBM-bound: the gradients are read once.  Tensors are cut into chunks of kChunk
// values, one workgroup each, found through the plan's list; a chunk leaves one
// partial in 64 bits.  A second launch joins them: one block for each tensor,
// and one more that adds up every chunk's partial by itself instead of waiting
// for the tensors' sums, so that nothing needs a counter or an atomic and every
// sum has one order.  Squares in 64 bits cost two instructions a value at half
// and quarter rate, far below what a value's bytes take.
//
// 200 million values of 24 tensors in bf16: 94 us (4.3 TB/s) and 6.1 for the join; scaled in
// place 169 (4.7 TB/s).  300 tensors of 2 million values in fp32: 4.8 and 2.7 us, launches.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <type_traits>

#include "values.hpp"

namespace nsd {

namespace {

constexpr int kGradThreads = 256;
constexpr int64_t kChunk = 8192;

struct GradTensor {
    int32_t first_chunk, nchunks;
};
struct GradChunk {  // all that a block needs, so that it waits for one read before the values'
    void *g;
    int32_t n, dtype;
};

// Largest magnitudes are compared as bits: in their order a NaN is above infinity.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

template <bool MAX>
struct Partial {
    double sum = 0.0;
    uint32_t top = 0;
    __device__ __forceinline__ void take(float x) {
        if constexpr (MAX) top = max(top, magnitude(x));
        else sum = __builtin_fma((double)x, (double)x, sum);
    }
    __device__ __forceinline__ void join(double v) {  // another partial, as value() gave it
        if constexpr (MAX) top = max(top, magnitude((float)v));
        else sum += v;
    }
    __device__ __forceinline__ double value() const {
        return MAX ? (double)__uint_as_float(top) : sum;
    }
    __device__ __forceinline__ void over_wave() {
#pragma unroll
        for (int m = 1; m < kWave; m <<= 1) {
            if constexpr (MAX) top = max(top, (uint32_t)__shfl_xor((int)top, m, kWave));
            else sum += __shfl_xor(sum, m, kWave);
        }
    }
};

template <bool MAX, int THREADS>
__device__ __forceinline__ void over_block(Partial<MAX> &p) {
    __shared__ double of_wave[THREADS / kWave];
    p.over_wave();
    if (threadIdx.x % kWave == 0) of_wave[threadIdx.x / kWave] = p.value();
    __syncthreads();
    p = Partial<MAX>();
    for (int w = 0; w < THREADS / kWave; ++w) p.join(of_wave[w]);
}

template <bool MAX, class T>
__device__ __forceinline__ void take_chunk(Partial<MAX> &p, const T *g, int end) {
    constexpr int N = 16 / sizeof(T);
    Partial<MAX> q[4];  // independent sums: a chain of one would wait for every value
    constexpr int step = kGradThreads * N;
    for (int b = 0; b < end; b += 4 * step) {
        float x[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = b + u * step + (int)threadIdx.x * N;
            load_left<N, T>(g + min(i, end), max(min(end - i, N), 0), x[u]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u].take(x[u][e]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) p.join(q[u].value());
}

template <bool MAX>
__global__ __launch_bounds__(kGradThreads) void grad_chunk_kernel(
    const GradChunk *__restrict__ chunks, double *part) {
    const GradChunk c = chunks[blockIdx.x];
    Partial<MAX> p;
    if (c.dtype == NSD_F32) take_chunk<MAX, float>(p, static_cast<const float *>(c.g), c.n);
    else take_chunk<MAX, Bf16>(p, static_cast<const Bf16 *>(c.g), c.n);
    over_block<MAX, kGradThreads>(p);
    if (threadIdx.x == 0) part[blockIdx.x] = p.value();
}

constexpr int kJoinThreads = 512;

template <bool MAX>
__global__ __launch_bounds__(kJoinThreads) void grad_join_kernel(
    const GradTensor *__restrict__ tensors, const double *__restrict__ part, int32_t nchunks,
    const float *grad_scale, double max_norm, double *norm, float *scale, double *norms) {
    int first = 0, n = nchunks;
    if (blockIdx.x > 0) {
        first = tensors[blockIdx.x - 1].first_chunk;
        n = tensors[blockIdx.x - 1].nchunks;
    }
    Partial<MAX> p;
    for (int i = threadIdx.x; i < n; i += 8 * kJoinThreads) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = i + u * kJoinThreads < n ? part[first + i + u * kJoinThreads] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) p.join(v[u]);
    }
    over_block<MAX, kJoinThreads>(p);
    if (threadIdx.x > 0) return;
    const double f = grad_scale ? (double)*grad_scale : 1.0;
    const double v = (MAX ? p.value() : sqrt(p.value())) * fabs(f);
    if (blockIdx.x > 0) {
        norms[blockIdx.x - 1] = v;
    } else {
        *norm = v;
        // (a norm that is not a number, but no infinite one without a bound, shows in the factor)
        const double c = v != v ? v : max_norm < HUGE_VAL ? max_norm / (v + 1e-6) : 1.0;
        *scale = (float)(f * (c > 1.0 ? 1.0 : c));
    }
}

template <class T>
__device__ __forceinline__ void scale_chunk(T *g, int end, float s) {
    constexpr int N = 16 / sizeof(T);
    constexpr int step = kGradThreads * N;
    for (int b = 0; b < end; b += 4 * step) {
        float x[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = b + u * step + (int)threadIdx.x * N;
            load_left<N, T>(g + min(i, end), max(min(end - i, N), 0), x[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = b + u * step + (int)threadIdx.x * N;
#pragma unroll
            for (int e = 0; e < N; ++e) x[u][e] *= s;
            store_left<N, T>(g + min(i, end), max(min(end - i, N), 0), x[u]);
        }
    }
}

__global__ __launch_bounds__(kGradThreads) void grad_scale_kernel(
    const GradChunk *__restrict__ chunks, const float *__restrict__ scale) {
    const float s = *scale;
    if (s == 1.f) return;
    const GradChunk c = chunks[blockIdx.x];
    if (c.dtype == NSD_F32) scale_chunk<float>(static_cast<float *>(c.g), c.n, s);
    else scale_chunk<Bf16>(static_cast<Bf16 *>(c.g), c.n, s);
}

nsd_status check_grads(int32_t n, const nsd_grad_tensor *ts, int64_t *chunks) {
    NSD_REQUIRE(n >= 0, "negative number of tensors");
    NSD_REQUIRE(n == 0 || ts != nullptr, "tensors is NULL");
    *chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        NSD_REQUIRE(ts[i].n >= 0, "tensor %d: negative length", i);
        if (ts[i].n > INT32_MAX - kChunk)
            return fail(NSD_ERR_TOO_LARGE, "tensor %d: %lld values", i, (long long)ts[i].n);
        NSD_REQUIRE(known_dtype(ts[i].dtype), "tensor %d: unknown type", i);
        NSD_REQUIRE(ts[i].n == 0 || ts[i].grad, "tensor %d: a NULL array", i);
        NSD_REQUIRE((reinterpret_cast<uintptr_t>(ts[i].grad) & (dtype_bytes(ts[i].dtype) - 1)) == 0,
                    "tensor %d: not at an address of its type", i);
        *chunks += ceil_div(ts[i].n, kChunk);
    }
    // a launch's threads are counted in 32 bits; so are the tensors' blocks
    if (*chunks > UINT32_MAX / kGradThreads || n >= (int32_t)(UINT32_MAX / kJoinThreads))
        return fail(NSD_ERR_TOO_LARGE, "%d tensors of %lld chunks", n, (long long)*chunks);
    return NSD_OK;
}

// 1 where some tensors share memory, 0 where none do, -1 without host memory.
int share_memory(int32_t n, const nsd_grad_tensor *ts) {
    if (n < 2) return 0;
    struct Span {
        uintptr_t lo, hi;
    };
    Span *all = static_cast<Span *>(std::malloc((size_t)n * sizeof(Span)));
    if (all == nullptr) return -1;
    size_t count = 0;
    for (int32_t i = 0; i < n; ++i) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(ts[i].grad);
        if (ts[i].n > 0) all[count++] = {lo, lo + (uintptr_t)ts[i].n * dtype_bytes(ts[i].dtype)};
    }
    std::sort(all, all + count, [](const Span &x, const Span &y) { return x.lo < y.lo; });
    int shared = 0;
    for (size_t i = 1; i < count; ++i) shared |= all[i].lo < all[i - 1].hi;
    std::free(all);
    return shared;
}

size_t grad_table_bytes(int32_t n, int64_t chunks) {
    return (size_t)n * sizeof(GradTensor) + (size_t)chunks * sizeof(GradChunk);
}

nsd_status check_plan(const nsd_grad_plan *p) {
    NSD_REQUIRE(p != nullptr && p->ntensors >= 0 && p->nchunks >= 0 &&
                    (p->ntensors == 0 || p->table),
                "plan is not built (nsd_grad_plan_build)");
    return NSD_OK;
}

const GradTensor *tensors_of(const nsd_grad_plan *p) {
    return static_cast<const GradTensor *>(p->table);
}
const GradChunk *chunks_of(const nsd_grad_plan *p) {
    return reinterpret_cast<const GradChunk *>(tensors_of(p) + p->ntensors);
}

}  // namespace

}  // namespace nsd

using namespace nsd;

extern "C" {

nsd_status nsd_grad_plan_size(int32_t ntensors, const nsd_grad_tensor *tensors, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    int64_t chunks;
    NSD_TRY(check_grads(ntensors, tensors, &chunks));
    *bytes = std::max<size_t>(grad_table_bytes(ntensors, chunks), 256);
    return NSD_OK;
}

nsd_status nsd_grad_plan_build(int32_t ntensors, const nsd_grad_tensor *tensors,
                               nsd_grad_plan *plan, void *table, size_t table_size,
                               void *stream) {
    NSD_REQUIRE(plan != nullptr, "plan is NULL");
    int64_t nchunks;
    NSD_TRY(check_grads(ntensors, tensors, &nchunks));
    const size_t need = grad_table_bytes(ntensors, nchunks);
    if (need > 0 && (table == nullptr || table_size < need))
        return fail(NSD_ERR_WORKSPACE, "table %zu bytes at %p, need %zu", table_size, table, need);
    NSD_REQUIRE((reinterpret_cast<uintptr_t>(table) & 7) == 0, "table is not 8-byte aligned");
    const int shared = share_memory(ntensors, tensors);
    if (shared < 0) return fail(NSD_ERR_HIP, "no host memory for %d tensors", ntensors);
    if (need > 0) {
        char *host = static_cast<char *>(std::malloc(need));
        if (host == nullptr) return fail(NSD_ERR_HIP, "no host memory for %zu bytes", need);
        GradTensor *ts = reinterpret_cast<GradTensor *>(host);
        GradChunk *cs = reinterpret_cast<GradChunk *>(host + (size_t)ntensors * sizeof(GradTensor));
        int32_t at = 0;
        for (int32_t i = 0; i < ntensors; ++i) {
            const nsd_grad_tensor &t = tensors[i];
            const int32_t own = (int32_t)ceil_div(t.n, kChunk);
            ts[i] = GradTensor{at, own};
            for (int32_t c = 0; c < own; ++c)
                cs[at++] = GradChunk{static_cast<char *>(t.grad) + c * kChunk * dtype_bytes(t.dtype),
                                     (int32_t)std::min(kChunk, t.n - c * kChunk), t.dtype};
        }
        hipError_t e = hipMemcpyAsync(table, host, need, hipMemcpyHostToDevice, as_stream(stream));
        if (e == hipSuccess) e = hipStreamSynchronize(as_stream(stream));
        std::free(host);
        NSD_TRY(check_hip(e, "copy of the gradients' table"));
    }
    plan->ntensors = ntensors;
    plan->nchunks = (int32_t)nchunks;
    plan->shared = shared;
    plan->table = table;
    return NSD_OK;
}

nsd_status nsd_grad_norm_workspace_size(const nsd_grad_plan *plan, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_TRY(check_plan(plan));
    Carver c(nullptr);
    c.take<double>(plan->nchunks);
    *bytes = std::max<size_t>(c.bytes(), 256);
    return NSD_OK;
}

nsd_status nsd_grad_norm(const nsd_grad_plan *plan, const nsd_clip *h, double *norm, float *scale,
                         double *norms, void *ws, size_t ws_bytes, void *stream) {
    NSD_TRY(check_plan(plan));
    NSD_REQUIRE(h != nullptr, "options are NULL");
    NSD_REQUIRE(h->order == 2 || h->order == 0, "order %d (2, or 0 for the largest)", h->order);
    NSD_REQUIRE(h->max_norm > 0, "max_norm %g is not above 0", h->max_norm);
    NSD_REQUIRE(norm && scale, "norm or scale is NULL");
    size_t need;
    NSD_TRY(nsd_grad_norm_workspace_size(plan, &need));
    if (ws == nullptr || ws_bytes < need)
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, need);
    NSD_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    // (one block writes the factor while others still read what it is made of)
    NSD_TRY(check_apart({flat_area(norm, 8), flat_area(scale, 4), flat_area(norms, 8 * (int64_t)plan->ntensors),
                         flat_area(ws, (int64_t)need)},
                        {flat_area(h->grad_scale, 4),
                         flat_area(plan->table, (int64_t)grad_table_bytes(plan->ntensors, plan->nchunks))}));
    Carver c(ws);
    double *part = c.take<double>(plan->nchunks);
    const hipStream_t st = as_stream(stream);
    const GradTensor *ts = tensors_of(plan);
    auto launch = [&](auto max) -> nsd_status {
        constexpr bool MAX = decltype(max)::value;
        if (plan->nchunks > 0) {
            grad_chunk_kernel<MAX><<<plan->nchunks, kGradThreads, 0, st>>>(chunks_of(plan), part);
            NSD_TRY(check_launch("grad_chunk_kernel"));
        }
        grad_join_kernel<MAX><<<1 + (norms ? plan->ntensors : 0), kJoinThreads, 0, st>>>(
            ts, part, plan->nchunks, h->grad_scale, h->max_norm, norm, scale, norms);
        return check_launch("grad_join_kernel");
    };
    return h->order == 0 ? launch(std::true_type()) : launch(std::false_type());
}

nsd_status nsd_grad_clip(const nsd_grad_plan *plan, const float *scale, void *stream) {
    NSD_TRY(check_plan(plan));
    NSD_REQUIRE(scale != nullptr, "scale is NULL");
    NSD_REQUIRE(!plan->shared, "tensors that share memory would be scaled more than once");
    if (plan->nchunks == 0) return NSD_OK;
    grad_scale_kernel<<<plan->nchunks, kGradThreads, 0, as_stream(stream)>>>(
        chunks_of(plan), scale);
    return check_launch("grad_scale_kernel");
}

}  // extern "C"
