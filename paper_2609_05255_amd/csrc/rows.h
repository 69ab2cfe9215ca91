// Vectors of rows whose length is no multiple of a vector, and exchanges between the lanes of a row.
#pragma once

#include "vec.h"

namespace gsr {

// A vector of a row of which `left` elements are the row's. What it reaches beyond the row's end is loaded with it as long
// as it lies before `end`, the matrix's own end: any value there. WHOLE: rows are whole vectors.
template <typename T, bool WHOLE>
__device__ __forceinline__ typename Vec<T>::Packed get_vec(const T* p, int64_t left, const T* end)
{
    if (WHOLE || p + Vec<T>::N <= end) return *reinterpret_cast<const typename Vec<T>::Any*>(p);
    return load_any(p, left);
}

// The first `left` elements, in at most three stores.
template <typename T, bool WHOLE>
__device__ __forceinline__ void put_vec(T* p, int64_t left, typename Vec<T>::Packed v)
{
    constexpr int N = Vec<T>::N;
    typedef T V4 __attribute__((ext_vector_type(4)));
    typedef T V2 __attribute__((ext_vector_type(2)));
    typedef V4 Any4 __attribute__((aligned(sizeof(T))));
    typedef V2 Any2 __attribute__((aligned(sizeof(T))));
    if (WHOLE || left >= N) {
        *reinterpret_cast<typename Vec<T>::Any*>(p) = v;
        return;
    }
    if constexpr (N == 8) {
        if (left & 4) *reinterpret_cast<Any4*>(p) = V4{v[0], v[1], v[2], v[3]};
        if (left & 2) *reinterpret_cast<Any2*>(p + (left & 4)) = left & 4 ? V2{v[4], v[5]} : V2{v[0], v[1]};
        if (left & 1) p[left & 6] = left & 4 ? (left & 2 ? v[6] : v[4]) : left & 2 ? v[2] : v[0];
    } else {
        if (left & 2) *reinterpret_cast<Any2*>(p) = V2{v[0], v[1]};
        if (left & 1) p[left & 2] = left & 2 ? v[2] : v[0];
    }
}

template <typename T, bool WHOLE>
__device__ __forceinline__ void put_floats(T* p, int64_t left, const float* in)
{
    typename Vec<T>::Packed v;
#pragma unroll
    for (int j = 0; j < Vec<T>::N; ++j) v[j] = (T)in[j];
    put_vec<T, WHOLE>(p, left, v);
}

// Value of another lane of the aligned group of 2, 4, 8 or 16 (a step of a reduction over the group, whose smaller groups
// have theirs already), then of the other half of 32 and 64 lanes.
template <int D>
__device__ __forceinline__ uint32_t lane_exchange(uint32_t v)
{
    if constexpr (D == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false);
    if constexpr (D == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false);
    if constexpr (D == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false);
    if constexpr (D == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false);
    return (uint32_t)__shfl_xor((int)v, D, 64);
}

// f over the G lanes of a group, left in all of them.
template <int G, typename F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, F f)
{
    if constexpr (G > 1) v = f(v, lane_exchange<1>(v));
    if constexpr (G > 2) v = f(v, lane_exchange<2>(v));
    if constexpr (G > 4) v = f(v, lane_exchange<4>(v));
    if constexpr (G > 8) v = f(v, lane_exchange<8>(v));
    if constexpr (G > 16) v = f(v, lane_exchange<16>(v));
    if constexpr (G > 32) v = f(v, lane_exchange<32>(v));
    return v;
}

template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t v)
{
    return group_reduce<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

template <int G>
__device__ __forceinline__ uint32_t group_min(uint32_t v)
{
    return group_reduce<G>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

template <int G>
__device__ __forceinline__ float group_sum(float v)
{
    return __uint_as_float(group_reduce<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

template <int G>
__device__ __forceinline__ float group_maxf(float v)
{
    return __uint_as_float(group_reduce<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}

}  // namespace gsr
