// Element types and loads shared by the kernels of sigtrain.h.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace st {

using bf16 = __bf16;
using f16 = _Float16;

// E elements that are moved as one access of up to 16 bytes.  Global memory takes such accesses at any element's alignment, so
// rows of odd lengths need no kernels of their own.
template <typename T, int E>
struct alignas(sizeof(T)) Vec {
    T v[E];
};
template <typename T>
constexpr int kPer16 = 16 / (int)sizeof(T);

template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_vec(const T* p)
{
    Vec<T, E> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <typename T, int E>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, E>& r)
{
    __builtin_memcpy(p, &r, sizeof(r));
}
// ... of a row's last few elements (n < E of them): the rest is 0, or not written
template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_some(const T* p, int n)
{
    Vec<T, E> r;
#pragma unroll
    for (int i = 0; i < E; ++i) r.v[i] = i < n ? p[i] : T(0);
    return r;
}
template <typename T, int E>
__device__ __forceinline__ void store_some(T* p, const Vec<T, E>& r, int n)
{
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < n) p[i] = r.v[i];
}

// Sums of values of a type: double where the values are float or double (the kernels that use it wait for memory).
template <typename T>
using sum_t = std::conditional_t<sizeof(T) == 2, float, double>;

// A symbol or target, ST_I32 or ST_I64.
__device__ __forceinline__ int64_t load_index(const void* p, int64_t i, int it)
{
    return it == 0 ? (int64_t) static_cast<const int32_t*>(p)[i] : static_cast<const int64_t*>(p)[i];
}

}  // namespace st
