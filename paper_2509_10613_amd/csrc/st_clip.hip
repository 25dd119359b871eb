// The norm of all entries of many arrays, and the arrays scaled down to a bound.
//
// Bound by memory: one read for the norm, one read and one write for the scaling (the factor is known only after the whole first
// pass; what of the arrays the caches still hold is not read again): 1.64e9 bfloat16 entries into floats 2.74 ms, 4.8 TB/s.  The arrays' table travels as a kernel argument, so a call
// copies nothing and can be captured; kClipBatch arrays per launch.  A launch is one grid of workgroups that step through
// chunks of kChunk entries, whatever arrays these lie in, and leaves one partial sum of squares per workgroup; every workgroup of the
// scaling launches adds all partial sums in the same order, which is cheaper than a launch in between.
//
// Squares and sums are in double: the square of a large float or bfloat16 passes float's range, and the conversions hide
// behind the loads.
#include "st_dev.h"
#include "st_kernels.h"

namespace st {
namespace {

constexpr int kThreads = 256, kChunk = 16384;

struct Batch {
    const void* in[kClipBatch];
    void* out[kClipBatch];
    int64_t count[kClipBatch];
    uint32_t chunk[kClipBatch + 1];   // the array's first chunk
    uint8_t dt[kClipBatch], out_dt[kClipBatch];
    int n;
};

template <typename F>
__device__ __forceinline__ void by_type(int dt, F&& f)
{
    switch (dt) {
    case ST_F64: f(double{}); break;
    case ST_F32: f(float{}); break;
    case ST_BF16: f(bf16{}); break;
    default: f(f16{}); break;
    }
}

// The array a chunk lies in.
__device__ __forceinline__ int array_of(const Batch& b, uint32_t chunk)
{
    int lo = 0, hi = b.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (b.chunk[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The workgroup's sum, in every thread, in a fixed order.
template <int THREADS>
__device__ __forceinline__ double sum_block(double x, double* scratch)
{
#pragma unroll
    for (int o = 32; o > 0; o /= 2) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) s += scratch[i];
    __syncthreads();
    return s;
}

// The squares of n <= kChunk entries, one thread's share.
template <typename T, int THREADS>
__device__ __forceinline__ double squares(const T* p, int n)
{
    constexpr int E = kPer16<T>, U = 4;
    double sum[U] = {};
    int i = threadIdx.x * E;
    for (; i + (U - 1) * THREADS * E + E <= n; i += U * THREADS * E) {
        Vec<T, E> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_vec<T, E>(p + i + u * THREADS * E);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[u] = fma((double)v[u].v[e], (double)v[u].v[e], sum[u]);
    }
    for (; i < n; i += THREADS * E) {
        const Vec<T, E> v = n - i >= E ? load_vec<T, E>(p + i) : load_some<T, E>(p + i, n - i);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[0] = fma((double)v.v[e], (double)v.v[e], sum[0]);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// A: the product's type.
template <typename T, typename O, typename A, int THREADS>
__device__ __forceinline__ void scale(const T* p, O* q, int n, double factor)
{
    constexpr int E = kPer16<T>, U = 2;
    const A f = (A)factor;
    const bool same = factor == 1.0;
    auto put = [&](int i, const Vec<T, E>& v, int some) {
        Vec<O, E> r;
#pragma unroll
        for (int e = 0; e < E; ++e) r.v[e] = (O)(same ? (A)v.v[e] : (A)v.v[e] * f);
        if (some >= E) store_vec(q + i, r);
        else store_some(q + i, r, some);
    };
    int i = threadIdx.x * E;
    for (; i + (U - 1) * THREADS * E + E <= n; i += U * THREADS * E) {
        Vec<T, E> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_vec<T, E>(p + i + u * THREADS * E);
#pragma unroll
        for (int u = 0; u < U; ++u) put(i + u * THREADS * E, v[u], E);
    }
    for (; i < n; i += THREADS * E) put(i, n - i >= E ? load_vec<T, E>(p + i) : load_some<T, E>(p + i, n - i), n - i);
}

template <int THREADS>
__device__ __forceinline__ double chunk_squares(const Batch& b, uint32_t c)
{
    const int a = array_of(b, c);
    const int64_t first = (int64_t)(c - b.chunk[a]) * kChunk, left = b.count[a] - first;
    const int n = left < kChunk ? (int)left : kChunk;
    double s = 0;
    by_type(b.dt[a], [&](auto type) {
        using T = decltype(type);
        s = squares<T, THREADS>(static_cast<const T*>(b.in[a]) + first, n);
    });
    return s;
}

template <int THREADS>
__device__ __forceinline__ void chunk_scale(const Batch& b, uint32_t c, double factor)
{
    const int a = array_of(b, c);
    const int64_t first = (int64_t)(c - b.chunk[a]) * kChunk, left = b.count[a] - first;
    const int n = left < kChunk ? (int)left : kChunk;
    by_type(b.dt[a], [&](auto type) {
        by_type(b.out_dt[a], [&](auto out_type) {
            using T = decltype(type);
            using O = decltype(out_type);
            const T* from = static_cast<const T*>(b.in[a]) + first;
            O* to = static_cast<O*>(b.out[a]) + first;
            // The product in double, rounded once; of 16-bit entries that do not become doubles in float, which is within 2^-23 of it, unless
            // the factor is below float's normal numbers (entries near 1e38 of bfloat16).
            if constexpr (sizeof(T) == 2 && sizeof(O) != 8)
                if (factor >= __FLT_MIN__) return scale<T, O, float, THREADS>(from, to, n, factor);
            scale<T, O, double, THREADS>(from, to, n, factor);
        });
    });
}

// In place with factor 1 nothing is to be done.
__device__ __forceinline__ bool untouched(const Batch& b, uint32_t c, double factor)
{
    const int a = array_of(b, c);
    return factor == 1.0 && b.in[a] == b.out[a];
}

__device__ __forceinline__ double clip_factor(double norm, double bound)
{
    return norm > bound && norm <= __DBL_MAX__ ? bound / norm : 1.0;
}

__global__ __launch_bounds__(kThreads) void squares_kernel(Batch b, double* partial)
{
    __shared__ double scratch[kThreads / 64];
    double s = 0;
    for (uint32_t c = blockIdx.x; c < b.chunk[b.n]; c += gridDim.x) s += chunk_squares<kThreads>(b, c);
    s = sum_block<kThreads>(s, scratch);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* partial, int n, double* scratch)
{
    double s = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += partial[i];
    return sqrt(sum_block<kThreads>(s, scratch));
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double* partial, int n, double* norm)
{
    __shared__ double scratch[kThreads / 64];
    const double x = norm_of(partial, n, scratch);
    if (threadIdx.x == 0) *norm = x;
}

__global__ __launch_bounds__(kThreads) void scale_kernel(Batch b, const double* partial, int n, double bound, double* norm)
{
    __shared__ double scratch[kThreads / 64];
    const double x = norm_of(partial, n, scratch), factor = clip_factor(x, bound);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = x;   // (every launch writes the same)
    for (uint32_t c = blockIdx.x; c < b.chunk[b.n]; c += gridDim.x)
        if (!untouched(b, c, factor)) chunk_scale<kThreads>(b, c, factor);
}

}  // namespace

static int64_t launches(int64_t n) { return n == 0 ? 1 : (n + kClipBatch - 1) / kClipBatch; }
// A launch's workgroups: the call's share of kClipBlocks, 64 at least.
static int64_t blocks_of(int64_t n)
{
    const int64_t share = kClipBlocks / launches(n);
    return share < 64 ? 64 : share;
}

size_t clip_workspace(int64_t n) { return round_up((size_t)(launches(n) * blocks_of(n)) * sizeof(double), 256); }

hipError_t clip(const void* const* grads, void* const* out, const int64_t* counts, const int* dts, const int* out_dts, int64_t n,
                double max_norm, double* norm, void* ws, hipStream_t st)
{
    double* partial = static_cast<double*>(ws);
    const int64_t most = blocks_of(n);
    int partials = 0;
    hipError_t e;
    for (int pass = 0; pass < (out ? 2 : 1); ++pass)
        for (int64_t i = 0; i < n;) {
            Batch b;
            b.n = 0;
            uint64_t chunks = 0;
            for (; i < n && b.n < kClipBatch; ++i) {
                if (counts[i] == 0) continue;
                const uint64_t mine = ((uint64_t)counts[i] + kChunk - 1) / kChunk;
                b.in[b.n] = grads[i];
                b.out[b.n] = out ? out[i] : nullptr;
                b.count[b.n] = counts[i];
                b.chunk[b.n] = (uint32_t)chunks;
                b.dt[b.n] = (uint8_t)dts[i];
                b.out_dt[b.n] = (uint8_t)(out_dts ? out_dts[i] : dts[i]);
                chunks += mine;
                ++b.n;
            }
            if (b.n == 0) break;
            b.chunk[b.n] = (uint32_t)chunks;
            const unsigned blocks = (unsigned)(chunks < (uint64_t)most ? chunks : (uint64_t)most);
            if (pass == 0) {
                squares_kernel<<<blocks, kThreads, 0, st>>>(b, partial + partials);
                partials += (int)blocks;
            } else {
                scale_kernel<<<blocks, kThreads, 0, st>>>(b, partial, partials, max_norm, norm);
            }
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    if (!out || partials == 0) {
        norm_kernel<<<1, kThreads, 0, st>>>(partial, partials, norm);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace st
