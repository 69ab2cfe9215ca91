// 16-byte vectors of the element types of the row operators (layer norm, linear,
// gradient clipping): loads at any element alignment, conversion to and from
// fp32 (to nearest even), and sums over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gsr {

typedef _Float16 f16;
typedef __bf16 bf16;

template <typename T>
struct Vec {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T Packed __attribute__((ext_vector_type(N)));
    // the same at any element's address: global memory is read and written at unaligned addresses
    typedef Packed Any __attribute__((aligned(sizeof(T))));
};

// N elements p[0, N) of which the first `left` exist (any value), as fp32; those beyond read as `pad`.
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, int64_t left, float* out, float pad = 0.f)
{
    constexpr int N = Vec<T>::N;
    if (left >= N) {
        const typename Vec<T>::Any v = *reinterpret_cast<const typename Vec<T>::Any*>(p);
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = (float)v[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = j < left ? (float)p[j] : pad;
    }
}

// The same as stored: elements beyond `left` read as 0.
template <typename T>
__device__ __forceinline__ typename Vec<T>::Packed load_any(const T* p, int64_t left)
{
    typename Vec<T>::Packed t = {};
    if (left >= Vec<T>::N) {
        t = *reinterpret_cast<const typename Vec<T>::Any*>(p);
    } else {
#pragma unroll
        for (int j = 0; j < Vec<T>::N; ++j)
            if (j < left) t[j] = p[j];
    }
    return t;
}

template <typename T>
__device__ __forceinline__ void store_vec(T* p, int64_t left, const float* in)
{
    constexpr int N = Vec<T>::N;
    if (left >= N) {
        typename Vec<T>::Any v;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (T)in[j];
        *reinterpret_cast<typename Vec<T>::Any*>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < left) p[j] = (T)in[j];
    }
}

// Sum over the aligned group of G lanes (a power of two, at most 64) that a lane belongs to.
template <int G>
__device__ __forceinline__ float lane_sum(float v)
{
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

__device__ __forceinline__ double lane_sum64(double v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

}  // namespace gsr
