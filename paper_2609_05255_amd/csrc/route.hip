// The router of a mixture: the experts of a row's largest logits and their weights, and the logits' gradient.
//
//   c_0 .. c_k-1: the experts of the k largest logits, the lower one of equals first; one of -infinity is never taken
//   normalise:  w_j = exp(l_c_j - m) / sum over j of exp(l_c_j - m),  dl_c_j = w_j (dw_j - sum of dw w), others 0
//   otherwise:  w_j = p_c_j, p = softmax of the row,                  dl_i = p_i ([i = c_j] dw_j - sum of dw w)
//
// Bound by HBM: a row of logits is read once and stays in the registers of a group of lanes. A choice is the maximum of
// integers that order as the logits do and hold the expert's number in their low bits, so that ties go to the lowest
// expert whatever the order of the exchanges between lanes; what is taken counts as nothing in the next round. 16-bit
// logits and numbers share 32 bits.
#include <type_traits>

#include "activation.h"
#include "gs_internal.h"
#include "vec.h"

namespace gsr {

namespace {

// A logit as an integer that orders as it does, above 0 for all but -infinity; undefined ones are the largest. With the
// number of its expert below: the lower one is larger.
template <typename T>
struct Choice {
    typedef uint32_t Key;   // 16 bits each
    static __device__ __forceinline__ uint16_t bits(T v) { return __builtin_bit_cast(uint16_t, v); }
    static __device__ __forceinline__ Key key(T v, int expert)
    {
        const float f = (float)v;
        uint32_t b = bits(v);
        if (f == 0.f) b = 0;   // the two zeros are equal
        b = b & 0x8000 ? b ^ 0xFFFF : b | 0x8000;
        if (f != f) b = 0xFFFF;
        return f == -__builtin_inff() ? 0 : b << 16 | (0xFFFF - expert);
    }
    static __device__ __forceinline__ int expert(Key k) { return 0xFFFF - (int)(k & 0xFFFF); }
    static __device__ __forceinline__ float value(Key k)
    {
        uint32_t b = k >> 16;
        b = b & 0x8000 ? b ^ 0x8000 : b ^ 0xFFFF;
        return (float)__builtin_bit_cast(T, (uint16_t)b);
    }
    static __device__ __forceinline__ Key exchange(Key k, int d) { return (Key)__shfl_xor((int)k, d, 64); }
};

template <>
struct Choice<float> {
    typedef uint64_t Key;
    static __device__ __forceinline__ Key key(float v, int expert)
    {
        uint32_t b = __float_as_uint(v);
        if (v == 0.f) b = 0;
        b = b >> 31 ? ~b : b | 0x80000000u;
        if (v != v) b = 0xFFFFFFFFu;
        return v == -__builtin_inff() ? 0 : (uint64_t)b << 32 | (0xFFFFFFFFu - (uint32_t)expert);
    }
    static __device__ __forceinline__ int expert(Key k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }
    static __device__ __forceinline__ float value(Key k)
    {
        const uint32_t b = (uint32_t)(k >> 32);
        return __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b);
    }
    static __device__ __forceinline__ Key exchange(Key k, int d)
    {
        return (uint64_t)(uint32_t)__shfl_xor((int)(k >> 32), d, 64) << 32 | (uint32_t)__shfl_xor((int)k, d, 64);
    }
};

struct RouteArgs {
    const void* logits;
    int64_t ldl, rows;
    int32_t experts, k, normalise;
    int32_t* expert;
    float* weight;
    const float* dweight;   // backward
    void* dlogits;
    int64_t ldd;
};

// G lanes share a row, with NV vectors each.
template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_route_fwd(RouteArgs a)
{
    constexpr int N = Vec<T>::N, kGroups = kBlock / G;
    constexpr int M = GS_MAX_CHOICES > G ? GS_MAX_CHOICES / G : 1;   // choices that a lane keeps
    typedef typename Choice<T>::Key Key;
    const int lane = threadIdx.x & (G - 1);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G; r < a.rows; r += step) {
        Key key[NV][N];
        float top = -__builtin_inff();
        typename Vec<T>::Packed raw[NV];
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (q * G + lane) * N;
            raw[q] = load_any((const T*)a.logits + r * a.ldl + c, a.experts - c);
        }
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int c = (q * G + lane) * N + e;
                key[q][e] = c < a.experts ? Choice<T>::key(raw[q][e], c) : 0;
            }
        float total = 0.f, mine[M];
        int32_t number[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            mine[m] = 0.f;
            number[m] = -1;
            for (int jj = 0; jj < G && m * G + jj < a.k; ++jj) {
                Key best = 0;
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < N; ++e) best = key[q][e] > best ? key[q][e] : best;
#pragma unroll
                for (int d = 1; d < G; d <<= 1) {
                    const Key other = Choice<T>::exchange(best, d);
                    best = other > best ? other : best;
                }
                if (best == 0) break;   // (in all lanes of the row)
                const float v = Choice<T>::value(best);
                if (m == 0 && jj == 0) top = v;
                const float p = exp_of(v - top);
                total += p;
                if (lane == jj) {
                    mine[m] = p;
                    number[m] = Choice<T>::expert(best);
                }
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < N; ++e) key[q][e] = key[q][e] == best ? 0 : key[q][e];
            }
        }
        if (!a.normalise) {
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int c = (q * G + lane) * N + e;
                    // (a masked one is 0 even where the largest is infinite, and undefined)
                    s += c < a.experts ? exp_of((float)raw[q][e] - top) : 0.f;
                }
            total = lane_sum<G>(s);
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int j = m * G + lane;
            if (j >= a.k) break;
            a.expert[r * a.k + j] = number[m];
            a.weight[r * a.k + j] = number[m] < 0 ? 0.f : mine[m] / total;
        }
    }
}

template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_route_bwd(RouteArgs a)
{
    constexpr int N = Vec<T>::N, kGroups = kBlock / G;
    const int lane = threadIdx.x & (G - 1);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G; r < a.rows; r += step) {
        float p[NV][N], d[NV][N];
        if (!a.normalise) {
            float top = -__builtin_inff(), s = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = (q * G + lane) * N;
                load_vec((const T*)a.logits + r * a.ldl + c, a.experts - c, p[q], -__builtin_inff());
#pragma unroll
                for (int e = 0; e < N; ++e) top = fmaxf(top, p[q][e]);
            }
#pragma unroll
            for (int x = 1; x < G; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    p[q][e] = top == -__builtin_inff() ? 0.f : exp_of(p[q][e] - top);
                    s += p[q][e];
                }
            s = lane_sum<G>(s);
            const float inv = s == 0.f ? 0.f : 1.f / s;   // (a row without experts)
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) p[q][e] *= inv;
        }
        float inner = 0.f;
        const int64_t at = r * a.k;
        for (int j = 0; j < a.k; ++j)
            if (a.expert[at + j] >= 0) inner = fmaf(a.dweight[at + j], a.weight[at + j], inner);
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < N; ++e) d[q][e] = a.normalise ? 0.f : -p[q][e] * inner;
        for (int j = 0; j < a.k; ++j) {
            const int32_t expert = a.expert[at + j];
            const float w = a.weight[at + j], dw = a.dweight[at + j];
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if ((q * G + lane) * N + e == expert) d[q][e] = a.normalise ? w * (dw - inner) : p[q][e] * (dw - inner);
        }
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (q * G + lane) * N;
            store_vec((T*)a.dlogits + r * a.ldd + c, a.experts - c, d[q]);
        }
    }
}

template <typename T>
hipError_t route(bool backward, const RouteArgs& a, hipStream_t s)
{
    const int64_t vecs = div_up(a.experts, Vec<T>::N);
    auto run = [&](auto lanes, auto count) {
        constexpr int G = decltype(lanes)::value, NV = decltype(count)::value;
        const dim3 grid((unsigned)std::min<int64_t>(div_up(a.rows, kBlock / G), 256 * 16));
        if (backward)
            hipLaunchKernelGGL((k_route_bwd<T, G, NV>), grid, dim3(kBlock), 0, s, a);
        else
            hipLaunchKernelGGL((k_route_fwd<T, G, NV>), grid, dim3(kBlock), 0, s, a);
        return hipGetLastError();
    };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    if (vecs <= 1) return run(one, one);
    if (vecs <= 2) return run(integral_constant<int, 2>(), one);
    if (vecs <= 4) return run(integral_constant<int, 4>(), one);
    if (vecs <= 8) return run(integral_constant<int, 8>(), one);
    if (vecs <= 16) return run(integral_constant<int, 16>(), one);
    if (vecs <= 32) return run(integral_constant<int, 32>(), one);
    if (vecs <= 64) return run(integral_constant<int, 64>(), one);
    if (vecs <= 128) return run(integral_constant<int, 64>(), integral_constant<int, 2>());
    return run(integral_constant<int, 64>(), integral_constant<int, 4>());
}

}  // namespace

static_assert(GS_MAX_EXPERTS <= 64 * 4 * 4, "a row of fp32 logits fits the registers of a wave");

hipError_t launch_route_fwd(int type, int64_t rows, int experts, int k, const void* logits, int64_t ldl, int normalise,
                            int32_t* expert, float* weight, hipStream_t s)
{
    const RouteArgs a = {logits, ldl, rows, experts, k, normalise, expert, weight, nullptr, nullptr, 0};
    if (type == GS_F16) return route<f16>(false, a, s);
    if (type == GS_BF16) return route<bf16>(false, a, s);
    return route<float>(false, a, s);
}

hipError_t launch_route_bwd(int type, int64_t rows, int experts, int k, const float* dweight, const void* logits,
                            int64_t ldl, const int32_t* expert, const float* weight, int normalise, void* dlogits,
                            int64_t ldd, hipStream_t s)
{
    const RouteArgs a = {logits, ldl, rows, experts, k, normalise, const_cast<int32_t*>(expert),
                         const_cast<float*>(weight), dweight, dlogits, ldd};
    if (type == GS_F16) return route<f16>(true, a, s);
    if (type == GS_BF16) return route<bf16>(true, a, s);
    return route<float>(true, a, s);
}

}  // namespace gsr
