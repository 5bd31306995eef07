// Rows of fp32, bf16 or f16 elements at any address, eight elements at a time, and sums over a workgroup.  Included by kernel sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace bmgd {
namespace {

typedef float float8v __attribute__((ext_vector_type(8)));

// Eight neighbouring elements at any multiple of an element's size: 16-bit ones are one instruction, 32-bit ones two.
template <typename T> struct Eight {
    typedef T vec __attribute__((ext_vector_type(8)));
    typedef T loose __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    static __device__ __forceinline__ vec load(const T* p) { return *reinterpret_cast<const loose*>(p); }
    static __device__ __forceinline__ void store(T* p, vec v) { *reinterpret_cast<loose*>(p) = v; }
    // the first `count` (1 to 7) of them; `fill` elsewhere
    static __device__ __forceinline__ vec load_part(const T* p, int count, T fill)
    {
        vec v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < count ? p[k] : fill;
        return v;
    }
    static __device__ __forceinline__ void store_part(T* p, vec v, int count)
    {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < count) p[k] = v[k];
    }
};

template <typename T> __device__ __forceinline__ float8v widen(typename Eight<T>::vec v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __builtin_convertvector(v, float8v);
}
template <typename T> __device__ __forceinline__ typename Eight<T>::vec narrow(float8v v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __builtin_convertvector(v, typename Eight<T>::vec);
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
template <typename V> __device__ __forceinline__ V wave_max(V v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const V o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}

}  // namespace
}  // namespace bmgd
