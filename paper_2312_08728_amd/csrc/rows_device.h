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

// The value of another lane of the same 16: lane ^ 1, lane ^ 2, 7 - lane of eight, 15 - lane.
enum { kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140 };
template <int WAY, typename V> __device__ __forceinline__ V from_lane(V v)
{
    if constexpr (sizeof(V) == 4)
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), WAY, 0xf, 0xf, true));
    else {
        typedef int int2v __attribute__((ext_vector_type(2)));
        int2v p = __builtin_bit_cast(int2v, v);
        p[0] = __builtin_amdgcn_update_dpp(0, p[0], WAY, 0xf, 0xf, true);
        p[1] = __builtin_amdgcn_update_dpp(0, p[1], WAY, 0xf, 0xf, true);
        return __builtin_bit_cast(V, p);
    }
}
template <typename V> __device__ __forceinline__ V of_lane(V v, int lane)
{
    if constexpr (sizeof(V) == 4)
        return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    else {
        typedef int int2v __attribute__((ext_vector_type(2)));
        int2v p = __builtin_bit_cast(int2v, v);
        p[0] = __builtin_amdgcn_readlane(p[0], lane);
        p[1] = __builtin_amdgcn_readlane(p[1], lane);
        return __builtin_bit_cast(V, p);
    }
}
// f over all 64 lanes, known to all: four steps in registers, then the four rows of 16.  (Steps through the shared memory's permutation take 6 x 0.05 us.)
template <typename V, typename F> __device__ __forceinline__ V over_wave(V v, F f)
{
    v = f(v, from_lane<kSwap1>(v));
    v = f(v, from_lane<kSwap2>(v));
    v = f(v, from_lane<kMirror8>(v));
    v = f(v, from_lane<kMirror16>(v));
    return f(f(of_lane(v, 0), of_lane(v, 16)), f(of_lane(v, 32), of_lane(v, 48)));
}
__device__ __forceinline__ float wave_sum(float v)
{
    return over_wave(v, [](float a, float b) { return a + b; });
}
template <typename V> __device__ __forceinline__ V wave_max(V v)
{
    return over_wave(v, [](V a, V b) { return b > a ? b : a; });
}

}  // namespace
}  // namespace bmgd
