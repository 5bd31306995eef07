// Rows of fp32, bf16 or f16 elements at any address, eight elements at a time, and sums over a workgroup.  Included by kernel sources only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace bmgd {
namespace {

// A piece: the neighbouring elements of 16 bytes, eight of 16 bits or four of 32.  At any multiple of an element's size one instruction (where it crosses a line of the
// cache it takes longer).
template <typename T> struct Piece {
    static constexpr int N = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(N)));
    typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    typedef float wide __attribute__((ext_vector_type(N)));
    static __device__ __forceinline__ vec load(const T* p) { return *reinterpret_cast<const loose*>(p); }
    static __device__ __forceinline__ void store(T* p, vec v) { *reinterpret_cast<loose*>(p) = v; }
    // those of elements j, j + 1, ... that are in [begin, end); `fill` elsewhere
    static __device__ __forceinline__ vec load_part(const T* p, int j, int begin, int end, T fill)
    {
        vec v;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = j + k >= begin && j + k < end ? p[j + k] : fill;
        return v;
    }
    static __device__ __forceinline__ void store_part(T* p, int j, int begin, int end, vec v)
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (j + k >= begin && j + k < end) p[j + k] = v[k];
    }
};

template <typename T> __device__ __forceinline__ typename Piece<T>::wide widen(typename Piece<T>::vec v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __builtin_convertvector(v, typename Piece<T>::wide);
}
template <typename T> __device__ __forceinline__ typename Piece<T>::vec narrow(typename Piece<T>::wide v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return __builtin_convertvector(v, typename Piece<T>::vec);
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
