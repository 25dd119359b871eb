// Softmax cross entropy of a linear read-out, and its gradients, in pieces of the classes.
//
// Forward: the logits z = h w^T are formed tile by tile on the matrix cores and reduced in registers to every row's maximum and sum
// of exponentials over the tile (and the target's logit); no logit is written.  Backward: the logits of a piece of the classes are formed
// again, their gradients G = u (exp(z - lse) - [class = target]) written as they are and transposed, and multiplied: grad_h += G w and
// grad_w = G^T h.
//
// All products are of one form, C[m, n] = sum_k A[m, k] B[n, k] with rows of A and B in whole steps of 128 bytes, so one main loop serves
// every type: a lane holds 16 consecutive bytes of a row, which are one matrix instruction's operand for 16-bit types and four or two
// instructions' for float and double (the order of k does not matter as long as both sides have the same).  The side whose index the
// result's rows run along is B: a lane then holds results that lie side by side in a row.
#include "st_dev.h"
#include "st_kernels.h"

namespace st {
namespace {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using f64x4 = __attribute__((ext_vector_type(4))) double;
using bf16x8 = __attribute__((ext_vector_type(8))) bf16;
using f16x8 = __attribute__((ext_vector_type(8))) f16;

template <typename T>
struct Types;
template <>
struct Types<bf16> {
    using Sum = float;
    using Frag = bf16x8;   // 16 bytes of a row
    using Acc = f32x4;     // a lane's part of a 16 x 16 tile
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Types<f16> {
    using Sum = float;
    using Frag = f16x8;
    using Acc = f32x4;
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Types<float> {
    using Sum = float;
    using Frag = f32x4;
    using Acc = f32x4;
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};
template <>
struct Types<double> {
    using Sum = double;
    using Frag = __attribute__((ext_vector_type(2))) double;
    using Acc = f64x4;
    static __device__ __forceinline__ Acc product(Frag a, Frag b, Acc c)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) c = __builtin_amdgcn_mfma_f64_16x16x4f64(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};
// The row of a 16 x 16 result tile that a lane's r-th number belongs to (its column is lane % 16).
template <typename T>
__device__ __forceinline__ int acc_row(int lane, int r)
{
    return sizeof(T) == 8 ? (lane >> 4) + 4 * r : (lane >> 4) * 4 + r;
}

__device__ __forceinline__ double exp_of(double x, double) { return exp(x); }
__device__ __forceinline__ float exp_of(float x, float) { return expf(x); }
// of logits that are sums of products of 16-bit numbers: the instruction's error is far below theirs
__device__ __forceinline__ float exp_of(float x, bf16) { return __expf(x); }
__device__ __forceinline__ float exp_of(float x, f16) { return __expf(x); }
__device__ __forceinline__ double log_of(double x) { return log(x); }
__device__ __forceinline__ float log_of(float x) { return logf(x); }

template <typename S>
__device__ __forceinline__ S lowest()
{
    return -(S)__builtin_inf();
}
// exp(x - m) where m may be the maximum of nothing
template <typename T, typename S>
__device__ __forceinline__ S exp_below(S x, S m)
{
    return m == lowest<S>() ? (S)0 : exp_of(x - m, T{});
}

// ------------------------------------------------------------------------------------------------ the products
constexpr int kThreads = 256, kTile = kTileRows, kWaveTile = 64, kSub = kWaveTile / 16;

struct Operands {
    const char *a, *b;
    int64_t a_pitch, b_pitch;   // bytes between rows
    int64_t m, n;               // rows
    int64_t steps;              // of kStepBytes along k
};

template <typename T>
using AccTile = typename Types<T>::Acc[kSub][kSub];

// One workgroup's 128 x 128 tile: four waves of 64 x 64.  acc[i][j]: 16 x 16 tile of rows m0 + i * 16, columns n0 + j * 16.
template <typename T>
__device__ __forceinline__ void multiply(const Operands& o, int64_t m0, int64_t n0, AccTile<T>& acc, char* lds)
{
    using Frag = typename Types<T>::Frag;
    constexpr int kLoads = kTile * kStepBytes / 16 / kThreads;   // 16-byte chunks per thread and side
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1;
#pragma unroll
    for (int i = 0; i < kSub; ++i)
#pragma unroll
        for (int j = 0; j < kSub; ++j) acc[i][j] = {0, 0, 0, 0};
    f32x4 ra[kLoads], rb[kLoads];
    const char *pa[kLoads], *pb[kLoads];
    int to[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int chunk = threadIdx.x + i * kThreads, row = chunk >> 3, c = chunk & 7;
        // rows behind the last are read from the last: their results are dropped
        pa[i] = o.a + (m0 + row < o.m ? m0 + row : o.m - 1) * o.a_pitch + c * 16;
        pb[i] = o.b + (n0 + row < o.n ? n0 + row : o.n - 1) * o.b_pitch + c * 16;
        to[i] = row * kStepBytes + ((c ^ (row & 7)) << 4);   // (the chunks of eight rows' same columns lie in different banks)
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        ra[i] = *reinterpret_cast<const f32x4*>(pa[i]);
        rb[i] = *reinterpret_cast<const f32x4*>(pb[i]);
    }
    for (int64_t s = 0; s < o.steps; ++s) {
        char* la = lds + (s & 1) * (2 * kTile * kStepBytes);
        char* lb = la + kTile * kStepBytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            *reinterpret_cast<f32x4*>(la + to[i]) = ra[i];
            *reinterpret_cast<f32x4*>(lb + to[i]) = rb[i];
        }
        __syncthreads();
        if (s + 1 < o.steps)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                ra[i] = *reinterpret_cast<const f32x4*>(pa[i] + (s + 1) * kStepBytes);
                rb[i] = *reinterpret_cast<const f32x4*>(pb[i] + (s + 1) * kStepBytes);
            }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            Frag fa[kSub], fb[kSub];
#pragma unroll
            for (int i = 0; i < kSub; ++i) {
                const int c = ((kk * 4 + (lane >> 4)) ^ (lane & 7)) << 4;
                fa[i] = *reinterpret_cast<const Frag*>(la + (wm * kWaveTile + i * 16 + (lane & 15)) * kStepBytes + c);
                fb[i] = *reinterpret_cast<const Frag*>(lb + (wn * kWaveTile + i * 16 + (lane & 15)) * kStepBytes + c);
            }
#pragma unroll
            for (int i = 0; i < kSub; ++i)
#pragma unroll
                for (int j = 0; j < kSub; ++j) acc[i][j] = Types<T>::product(fa[i], fb[j], acc[i][j]);
        }
        // (the next step writes the other half; a wave reaches that write of the step after next only past the next barrier)
    }
}
constexpr size_t kProductLds = 4 * kTile * kStepBytes;

// Forward: every row's maximum and sum of exponentials over the tile's classes (A: classes of w, B: rows of h).
template <typename T>
__global__ __launch_bounds__(kThreads) void stats_kernel(Operands o, const void* targets, int it, int64_t first_class, int64_t V,
                                                         typename Types<T>::Sum* part_max, typename Types<T>::Sum* part_sum,
                                                         typename Types<T>::Sum* hit)
{
    using S = typename Types<T>::Sum;
    __shared__ __align__(16) char lds[kProductLds];
    const int64_t m0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
    AccTile<T> acc;
    multiply<T>(o, m0, n0, acc, lds);
    __syncthreads();
    S* waves = reinterpret_cast<S*>(lds);   // [2 halves of the classes][2: maximum, sum][kTile]
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1;
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
        const int64_t row = n0 + wn * kWaveTile + j * 16 + (lane & 15);
        const int64_t target = row < o.n ? load_index(targets, row, it) : -1;
        const int64_t wanted = target >= 0 && target < V ? target - first_class - m0 - wm * kWaveTile : -1;
        S top = lowest<S>();
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = i * 16 + acc_row<T>(lane, r);
                if (m0 + wm * kWaveTile + at >= o.m) acc[i][j][r] = lowest<S>();
                else if (at == wanted) hit[row] = acc[i][j][r];
                // (a maximum that a NaN passes through)
                top = acc[i][j][r] > top || acc[i][j][r] != acc[i][j][r] ? acc[i][j][r] : top;
            }
#pragma unroll
        for (int x = 16; x < 64; x *= 2) {
            const S other = __shfl_xor(top, x);
            top = other > top || other != other ? other : top;
        }
        S sum = 0;
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += exp_below<T>(acc[i][j][r], top);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) {
            waves[(wm * 2 + 0) * kTile + wn * kWaveTile + j * 16 + lane] = top;
            waves[(wm * 2 + 1) * kTile + wn * kWaveTile + j * 16 + lane] = sum;
        }
    }
    __syncthreads();
    const int64_t row = n0 + threadIdx.x;
    if (threadIdx.x < kTile && row < o.n) {
        const S a = waves[threadIdx.x], b = waves[2 * kTile + threadIdx.x];
        const S top = b > a || b != b ? b : a;
        part_max[(int64_t)blockIdx.x * o.n + row] = top;
        part_sum[(int64_t)blockIdx.x * o.n + row] =
            waves[kTile + threadIdx.x] * exp_below<T>(a, top) + waves[3 * kTile + threadIdx.x] * exp_below<T>(b, top);
    }
}

// Backward: the gradients of the piece's logits, g[row][class] and gt[class][row], zeros up to whole steps.
template <typename T>
__global__ __launch_bounds__(kThreads) void grads_kernel(Operands o, const void* targets, int it, int64_t first_class,
                                                         const typename Types<T>::Sum* lse, const typename Types<T>::Sum* up, T* g,
                                                         int64_t g_pitch, T* gt, int64_t gt_pitch)
{
    using S = typename Types<T>::Sum;
    __shared__ __align__(16) char lds[kProductLds];
    const int64_t m0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
    AccTile<T> acc;
    multiply<T>(o, m0, n0, acc, lds);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1;
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
        const int64_t row = n0 + wn * kWaveTile + j * 16 + (lane & 15);
        const bool there = row < o.n;
        const int64_t target = there ? load_index(targets, row, it) : -1;
        const int64_t wanted = target - first_class - m0 - wm * kWaveTile;
        const S u = there ? up[row] : (S)0, l = there ? lse[row] : (S)0;
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = i * 16 + acc_row<T>(lane, r);
                const int64_t cls = m0 + wm * kWaveTile + at;
                // rows without a target (u is 0) stay 0 whatever their logits are
                const S p = exp_of(acc[i][j][r] - l, T{}) - (at == wanted ? (S)1 : (S)0);
                const T v = (T)(u != 0 && cls < o.m ? u * p : (S)0);
                if (there && cls < g_pitch) g[row * g_pitch + cls] = v;
                if (cls < o.m && row < gt_pitch) gt[cls * gt_pitch + row] = v;
            }
    }
}

// out[n][m] (pitch D): the first piece's results set the sum, the last one's leave it rounded, divided by the gradients' scaling.
template <typename T>
__global__ __launch_bounds__(kThreads) void product_kernel(Operands o, typename Types<T>::Sum* sum, T* out, int64_t D, bool first, bool last,
                                                           const typename Types<T>::Sum* unscale)
{
    using S = typename Types<T>::Sum;
    __shared__ __align__(16) char lds[kProductLds];
    const int64_t m0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
    AccTile<T> acc;
    multiply<T>(o, m0, n0, acc, lds);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wm = w >> 1, wn = w & 1;
    const S f = *unscale;
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
        const int64_t n = n0 + wn * kWaveTile + j * 16 + (lane & 15);
        if (n >= o.n) continue;
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t m = m0 + wm * kWaveTile + i * 16 + acc_row<T>(lane, r);
                if (m >= o.m) continue;
                S x = acc[i][j][r];
                if (!first) x += sum[n * D + m];
                if (last) out[n * D + m] = (T)(x * f);
                else sum[n * D + m] = x;
            }
    }
}

// ------------------------------------------------------------------------------------------------ copies
// dst[rows][pitch] = src[rows][cols], zeros behind the columns.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* src, T* dst, int64_t rows, int64_t cols, int64_t pitch)
{
    constexpr int E = kPer16<T>;
    const int64_t per_row = pitch / E, items = rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row, col = (i - row * per_row) * E;
        const int64_t left = cols - col;
        const Vec<T, E> v = left >= E ? load_vec<T, E>(src + row * cols + col) : load_some<T, E>(src + row * cols + col, (int)(left > 0 ? left : 0));
        store_vec(dst + row * pitch + col, v);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T* p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = T(0);
}

// dst[cols][pitch] = src[rows][cols] transposed, zeros behind the rows.  targets not null: rows without one are zeros, whatever they hold.
template <typename T>
__global__ __launch_bounds__(256) void transpose_kernel(const T* src, T* dst, int64_t rows, int64_t cols, int64_t pitch, const void* targets,
                                                        int it, int64_t V)
{
    constexpr int N = 64;
    __shared__ T tile[N][N + 16 / sizeof(T) / 2];
    const int64_t r0 = (int64_t)blockIdx.x * N, c0 = (int64_t)blockIdx.y * N;
    for (int i = threadIdx.x; i < N * N; i += 256) {
        const int64_t r = r0 + i / N, c = c0 + i % N;
        bool there = r < rows && c < cols;
        if (there && targets) {
            const int64_t t = load_index(targets, r, it);
            there = t >= 0 && t < V;
        }
        tile[i / N][i % N] = there ? src[r * cols + c] : T(0);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < N * N; i += 256) {
        const int64_t r = r0 + i % N, c = c0 + i / N;
        if (c < cols && r < pitch) dst[c * pitch + r] = tile[i % N][i / N];
    }
}

// ------------------------------------------------------------------------------------------------ rows
// Joins the tiles' maxima and sums of a piece with the running ones; after the last piece lse and the row's loss.
// A workgroup takes 64 rows, 16 threads each over the tiles.
template <typename T>
__global__ __launch_bounds__(1024) void join_kernel(const typename Types<T>::Sum* part_max, const typename Types<T>::Sum* part_sum, int64_t tiles,
                                                    int64_t rows, bool first, bool last, typename Types<T>::Sum* run_max,
                                                    typename Types<T>::Sum* run_sum, const typename Types<T>::Sum* hit, const void* targets, int it,
                                                    int64_t V, typename Types<T>::Sum* lse, typename Types<T>::Sum* losses)
{
    using S = typename Types<T>::Sum;
    __shared__ S tops[16][64], sums[16][64];
    const int lane = threadIdx.x & 63, seg = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 64 + lane;
    S top = lowest<S>(), sum = 0;
    auto add = [&](S t, S s) {
        const S m = t > top || t != t ? t : top;
        sum = sum * exp_below<T>(top, m) + s * exp_below<T>(t, m);
        top = m;
    };
    if (row < rows) {
        if (seg == 0 && !first) add(run_max[row], run_sum[row]);
        for (int64_t i = seg; i < tiles; i += 16) add(part_max[i * rows + row], part_sum[i * rows + row]);
    }
    tops[seg][lane] = top;
    sums[seg][lane] = sum;
    __syncthreads();
    if (seg != 0 || row >= rows) return;
    for (int i = 1; i < 16; ++i) add(tops[i][lane], sums[i][lane]);
    if (!last) {
        run_max[row] = top;
        run_sum[row] = sum;
        return;
    }
    const S l = top + log_of(sum);
    const int64_t target = load_index(targets, row, it);
    lse[row] = l;
    losses[row] = target >= 0 && target < V ? l - hit[row] : (S)0;
}

// The rows with a target and, unless reduction is ST_NONE, the sum or mean of their losses.  One workgroup.
template <typename S>
__global__ __launch_bounds__(1024) void reduce_kernel(const S* losses, const void* targets, int it, int64_t rows, int64_t V, int reduction, S* loss,
                                                      double* count)
{
    __shared__ double scratch[32];
    double sum = 0, n = 0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const int64_t t = load_index(targets, i, it);
        if (t >= 0 && t < V) {
            n += 1;
            if (reduction != ST_NONE) sum += (double)losses[i];
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o /= 2) {
        sum += __shfl_xor(sum, o);
        n += __shfl_xor(n, o);
    }
    if ((threadIdx.x & 63) == 0) {
        scratch[threadIdx.x >> 6] = sum;
        scratch[16 + (threadIdx.x >> 6)] = n;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = n = 0;
    for (int i = 0; i < 16; ++i) {
        sum += scratch[i];
        n += scratch[16 + i];
    }
    *count = n;
    if (reduction == ST_SUM) *loss = (S)sum;
    if (reduction == ST_MEAN) *loss = (S)(n > 0 ? sum / n : 0.0);
}

// Every row's upstream gradient, and scaling[0] = 1 / the factor it has been multiplied by: for f16 a power of two that takes the
// largest to 2^13 .. 2^14 (the gradients of a mean over thousands of rows would otherwise be subnormal).  One workgroup.
template <typename T>
__global__ __launch_bounds__(1024) void upstream_kernel(const typename Types<T>::Sum* grad, const void* targets, int it, int64_t rows, int64_t V,
                                                        int reduction, const double* count, typename Types<T>::Sum* up,
                                                        typename Types<T>::Sum* scaling)
{
    using S = typename Types<T>::Sum;
    __shared__ float tops[16];
    auto value = [&](int64_t i) {
        const int64_t t = load_index(targets, i, it);
        if (t < 0 || t >= V) return (S)0;
        if (reduction == ST_NONE) return grad[i];
        return reduction == ST_SUM ? grad[0] : (S)((double)grad[0] / *count);
    };
    S factor = 1;
    if constexpr (std::is_same_v<T, f16>) {
        float top = 0;
        for (int64_t i = threadIdx.x; i < rows; i += 1024) top = fmaxf(top, fabsf(value(i)));
#pragma unroll
        for (int o = 32; o > 0; o /= 2) top = fmaxf(top, __shfl_xor(top, o));
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
        for (int i = 0; i < 16; ++i) top = fmaxf(top, tops[i]);
        int e = 0;
        if (top > 0 && top <= 3.4028234e38f) {
            frexpf(top, &e);
            e = 14 - e;
            e = e > 126 ? 126 : e < -126 ? -126 : e;
        }
        factor = ldexpf(1.0f, e);
        if (threadIdx.x == 0) *scaling = ldexpf(1.0f, -e);
    } else {
        if (threadIdx.x == 0) *scaling = 1;
    }
    for (int64_t i = threadIdx.x; i < rows; i += 1024) up[i] = value(i) * factor;
}

unsigned blocks_for(int64_t items) { return (unsigned)((items + 255) / 256 < 16384 ? (items + 255) / 256 : 16384); }

#define ST_TRY(call)                               \
    do {                                           \
        (call);                                    \
        const hipError_t err_ = hipGetLastError(); \
        if (err_ != hipSuccess) return err_;       \
    } while (0)

// A matrix with rows in whole steps: the caller's, or a copy.
template <typename T>
hipError_t in_steps(const T* src, int64_t rows, int64_t cols, int64_t pitch, void* copy, const T** out, hipStream_t st)
{
    *out = src;
    if (cols == pitch && reinterpret_cast<uintptr_t>(src) % 16 == 0) return hipSuccess;
    *out = static_cast<const T*>(copy);
    ST_TRY((pack_kernel<T><<<blocks_for(rows * (pitch / kPer16<T>)), 256, 0, st>>>(src, static_cast<T*>(copy), rows, cols, pitch)));
    return hipSuccess;
}

template <typename T>
Operands operands(const T* a, int64_t a_cols, int64_t m, const T* b, int64_t b_cols, int64_t n, int64_t k)
{
    return {reinterpret_cast<const char*>(a), reinterpret_cast<const char*>(b), a_cols * (int64_t)sizeof(T), b_cols * (int64_t)sizeof(T), m, n,
            k * (int64_t)sizeof(T) / kStepBytes};
}
dim3 tiles_of(int64_t m, int64_t n) { return dim3((unsigned)((m + kTile - 1) / kTile), (unsigned)((n + kTile - 1) / kTile)); }

template <typename T>
hipError_t run_fwd(const EntropyPlan& p, const T* h, const T* w, const void* targets, void* loss, void* lse, double* rows, int reduction, int it,
                   unsigned char* ws, hipStream_t st)
{
    using S = typename Types<T>::Sum;
    if (p.T == 0) {
        ST_TRY((reduce_kernel<S><<<1, 1024, 0, st>>>(nullptr, nullptr, it, 0, p.V, reduction, static_cast<S*>(loss), rows)));
        return hipSuccess;
    }
    const T* hs;
    hipError_t e = in_steps(h, p.T, p.D, p.Dp, ws + p.off_h, &hs, st);
    if (e != hipSuccess) return e;
    S *run_max = reinterpret_cast<S*>(ws + p.off_max), *run_sum = reinterpret_cast<S*>(ws + p.off_sum), *hit = reinterpret_cast<S*>(ws + p.off_hit);
    const int64_t most = p.piece / kTile;
    S *part_max = reinterpret_cast<S*>(ws + p.off_part), *part_sum = part_max + most * p.T;
    // (the running maxima are dead where the losses of the rows are written: a thread reads its own first)
    S* losses = reduction == ST_NONE ? static_cast<S*>(loss) : run_max;
    for (int64_t i = 0; i < p.pieces; ++i) {
        const int64_t first = i * p.piece, n = p.V - first < p.piece ? p.V - first : p.piece;
        const T* wsrc;
        if ((e = in_steps(w + first * p.D, n, p.D, p.Dp, ws + p.off_w, &wsrc, st)) != hipSuccess) return e;
        const Operands o = operands(wsrc, p.Dp, n, hs, p.Dp, p.T, p.Dp);
        const dim3 grid = tiles_of(n, p.T);
        ST_TRY((stats_kernel<T><<<grid, kThreads, 0, st>>>(o, targets, it, first, p.V, part_max, part_sum, hit)));
        ST_TRY((join_kernel<T><<<(unsigned)((p.T + 63) / 64), 1024, 0, st>>>(part_max, part_sum, grid.x, p.T, i == 0, i + 1 == p.pieces, run_max,
                                                                            run_sum, hit, targets, it, p.V, static_cast<S*>(lse), losses)));
    }
    ST_TRY((reduce_kernel<S><<<1, 1024, 0, st>>>(losses, targets, it, p.T, p.V, reduction, static_cast<S*>(loss), rows)));
    return hipSuccess;
}

template <typename T>
hipError_t run_bwd(const EntropyPlan& p, const T* h, const T* w, const void* targets, const void* lse, const double* rows, const void* grad,
                   T* grad_h, T* grad_w, int reduction, int it, unsigned char* ws, hipStream_t st)
{
    using S = typename Types<T>::Sum;
    if (p.T == 0) {
        if (grad_w) ST_TRY((zero_kernel<T><<<blocks_for(p.V * p.D), 256, 0, st>>>(grad_w, p.V * p.D)));
        return hipSuccess;
    }
    S *up = reinterpret_cast<S*>(ws + p.off_up), *scaling = up + p.T, *dh = reinterpret_cast<S*>(ws + p.off_dh);
    T *ht = reinterpret_cast<T*>(ws + p.off_ht), *wt = reinterpret_cast<T*>(ws + p.off_wt);
    T *g = reinterpret_cast<T*>(ws + p.off_g), *gt = reinterpret_cast<T*>(ws + p.off_gt);
    ST_TRY((upstream_kernel<T><<<1, 1024, 0, st>>>(static_cast<const S*>(grad), targets, it, p.T, p.V, reduction, rows, up, scaling)));
    const T* hs;
    hipError_t e = in_steps(h, p.T, p.D, p.Dp, ws + p.off_h, &hs, st);
    if (e != hipSuccess) return e;
    auto turn = [&](const T* src, T* dst, int64_t r, int64_t pitch, const void* only) -> hipError_t {
        ST_TRY((transpose_kernel<T><<<dim3((unsigned)((pitch + 63) / 64), (unsigned)((p.D + 63) / 64)), 256, 0, st>>>(src, dst, r, p.D, pitch, only, it,
                                                                                                                  p.V)));
        return hipSuccess;
    };
    if (grad_w && (e = turn(h, ht, p.T, p.Tp, targets)) != hipSuccess) return e;
    for (int64_t i = 0; i < p.pieces; ++i) {
        const int64_t first = i * p.piece, n = p.V - first < p.piece ? p.V - first : p.piece;
        const int64_t per = kStepBytes / (int64_t)sizeof(T), np = (n + per - 1) / per * per;
        const T* wsrc;
        if ((e = in_steps(w + first * p.D, n, p.D, p.Dp, ws + p.off_w, &wsrc, st)) != hipSuccess) return e;
        const Operands logits = operands(wsrc, p.Dp, n, hs, p.Dp, p.T, p.Dp);
        ST_TRY((grads_kernel<T><<<tiles_of(n, p.T), kThreads, 0, st>>>(logits, targets, it, first, static_cast<const S*>(lse), up, g, np, gt, p.Tp)));
        if (grad_h) {
            if ((e = turn(w + first * p.D, wt, n, np, nullptr)) != hipSuccess) return e;
            const Operands o = operands(wt, np, p.D, g, np, p.T, np);
            ST_TRY((product_kernel<T><<<tiles_of(p.D, p.T), kThreads, 0, st>>>(o, dh, grad_h, p.D, i == 0, i + 1 == p.pieces, scaling)));
        }
        if (grad_w) {
            const Operands o = operands(ht, p.Tp, p.D, gt, p.Tp, n, p.Tp);
            ST_TRY((product_kernel<T><<<tiles_of(p.D, n), kThreads, 0, st>>>(o, nullptr, grad_w + first * p.D, p.D, true, true, scaling)));
        }
    }
    return hipSuccess;
}

template <typename F>
hipError_t by_type(int dt, F&& f)
{
    switch (dt) {
    case ST_F64: return f(double{});
    case ST_F32: return f(float{});
    case ST_BF16: return f(bf16{});
    default: return f(f16{});
    }
}

}  // namespace

EntropyPlan entropy_plan(bool backward, int64_t T, int64_t V, int64_t D, int dt, bool least, size_t ws_bytes)
{
    EntropyPlan p{};
    p.T = T;
    p.V = V;
    p.D = D;
    p.size = dtype_size(dt);
    p.sum_size = dt == ST_F64 ? 8 : 4;
    const int64_t per = kStepBytes / p.size;
    auto steps = [&](int64_t n) { return (n + per - 1) / per * per; };
    p.Dp = steps(D);
    p.Tp = steps(T);
    auto lay = [&](int64_t piece) {
        p.piece = piece;
        p.pieces = (V + piece - 1) / piece;
        size_t at = 0;
        auto take = [&](int64_t entries, int size) {
            const size_t here = at;
            at += round_up((size_t)entries * size, 256);
            return here;
        };
        p.off_h = take(T * p.Dp, p.size);
        p.off_w = take(piece * p.Dp, p.size);
        if (!backward) {
            p.off_max = take(T, p.sum_size);
            p.off_sum = take(T, p.sum_size);
            p.off_hit = take(T, p.sum_size);
            p.off_part = take(2 * T * (piece / kTile), p.sum_size);
        } else {
            p.off_up = take(T + 2, p.sum_size);
            p.off_ht = take(D * p.Tp, p.size);
            p.off_wt = take(D * piece, p.size);
            p.off_g = take(T * piece, p.size);
            p.off_gt = take(piece * p.Tp, p.size);
            p.off_dh = take(p.pieces > 1 ? T * D : 0, p.sum_size);
        }
        p.total = at;
    };
    const int64_t all = (V + kTile - 1) / kTile * kTile;
    if (least) {
        lay(kTile);
        return p;
    }
    // Pieces as large as 512 MiB of what a class takes: the fewer there are, the less often the sums of grad_h are read and written.
    const int64_t each = backward ? 2 * p.Tp * p.size + 2 * p.Dp * p.size : p.Dp * p.size + 2 * T * p.sum_size / kTile + 1;
    int64_t most = ((int64_t)512 << 20) / each / kTile * kTile;
    if (most < kTile) most = kTile;
    if (most > ((int64_t)1 << 22)) most = (int64_t)1 << 22;   // (tiles of a piece are a grid's second index)
    for (int64_t count = (all + most - 1) / most;; ++count) {
        const int64_t piece = ((all + count - 1) / count + kTile - 1) / kTile * kTile;
        lay(piece);
        if (ws_bytes == 0 || p.total <= ws_bytes || piece == kTile) return p;
    }
}

hipError_t entropy_fwd(const EntropyPlan& p, const void* h, const void* w, const void* targets, void* loss, void* lse, double* rows,
                       int reduction, int it, int dt, void* ws, hipStream_t st)
{
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        return run_fwd<T>(p, static_cast<const T*>(h), static_cast<const T*>(w), targets, loss, lse, rows, reduction, it,
                          static_cast<unsigned char*>(ws), st);
    });
}

hipError_t entropy_bwd(const EntropyPlan& p, const void* h, const void* w, const void* targets, const void* lse, const double* rows,
                       const void* grad, void* grad_h, void* grad_w, int reduction, int it, int dt, void* ws, hipStream_t st)
{
    return by_type(dt, [&](auto type) {
        using T = decltype(type);
        return run_bwd<T>(p, static_cast<const T*>(h), static_cast<const T*>(w), targets, lse, rows, grad, static_cast<T*>(grad_h),
                          static_cast<T*>(grad_w), reduction, it, static_cast<unsigned char*>(ws), st);
    });
}

}  // namespace st
