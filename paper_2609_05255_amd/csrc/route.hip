// The router of a mixture: the experts of a row's largest logits and their weights, and the logits' gradient.
//
//   c_0 .. c_k-1: the experts of the k largest logits, the lower one of equals first; one of -infinity is never taken
//   normalise:  w_j = exp(l_c_j - m) / sum over j of exp(l_c_j - m),  dl_c_j = w_j (dw_j - sum of dw w), others 0
//   otherwise:  w_j = p_c_j, p = softmax of the row,                  dl_i = p_i ([i = c_j] dw_j - sum of dw w)
//
// Bound by HBM, and nearly so by the instructions that the choices take: a row of logits is read once and stays in the
// registers of a group of lanes. A choice is a maximum of integers that order as the logits do, with ties to the lowest
// expert whatever the order of the exchanges between lanes (DPP up to 16 lanes).
//
// Measured: 1,000,000 x 64 in binary16, top 2, normalised 29 us, 4.9 TB/s (47 before one word held a logit's order
// and its expert, and lanes exchanged by DPP); the backward of 100,003 x 37 in bfloat16, top 3, out of the softmax over all
// 9.1 us, 1.9 TB/s, of which a launch is 4.
#include <type_traits>

#include "activation.h"
#include "gs_internal.h"
#include "rows.h"

namespace gsr {

namespace {

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

// A logit as an integer that orders as it does: its bits as a number with a sign (the two zeros are equal), moved up by
// half the range. Undefined ones are the largest; -infinity is kNone, with nothing but them below it.
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v), m = (uint32_t)((int32_t)b >> 31);
    const uint32_t o = ((b ^ (m & 0x7FFFFFFFu)) - m) ^ 0x80000000u;
    return v != v ? 0xFFFFFFFFu : o;
}
constexpr uint32_t kNone = 0x80000000u - 0x7F800000u;
__device__ __forceinline__ float order_value(uint32_t o)
{
    o ^= 0x80000000u;
    return __uint_as_float(o >> 31 ? 0x80000000u - o : o);
}

// The same for a pair of 16-bit logits at once, in the halves of a word; undefined ones apart (they are looked for before).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t Words __attribute__((ext_vector_type(4)));
template <typename T>
struct Order16 {
    static constexpr uint32_t kInf = __is_same(T, f16) ? 0x7C00 : 0x7F80;
    static constexpr uint32_t kNone = 0x8000 - kInf;
    static constexpr uint32_t kMasked = (kInf | 0x8000) * 0x10001u;   // a pair of -infinity
    static __device__ __forceinline__ uint32_t of(uint32_t pair)
    {
        const u16x2 x = __builtin_bit_cast(u16x2, pair);
        const u16x2 m = __builtin_bit_cast(u16x2, __builtin_bit_cast(i16x2, x) >> 15);
        const u16x2 s = (x ^ (m & (uint16_t)0x7FFF)) - m;
        return __builtin_bit_cast(uint32_t, s) ^ 0x80008000u;
    }
    static __device__ __forceinline__ float value(uint32_t o)
    {
        o ^= 0x8000;
        o = o & 0x8000 ? 0x8000 - o : o;   // (in 16 bits)
        return (float)__builtin_bit_cast(T, (uint16_t)o);
    }
};

// The middle one of three, where a >= b: a word inserted between two places of a falling list.
__device__ __forceinline__ uint32_t middle(uint32_t a, uint32_t b, uint32_t v)
{
    uint32_t o;
    asm("v_med3_u32 %0, %1, %2, %3" : "=v"(o) : "v"(a), "v"(b), "v"(v));
    return o;
}

// The K largest of a lane's words, in falling order.
template <int K>
__device__ __forceinline__ void insert(uint32_t (&top)[K], uint32_t v)
{
#pragma unroll
    for (int k = K - 1; k > 0; --k) top[k] = middle(top[k - 1], top[k], v);
    top[0] = v > top[0] ? v : top[0];
}

// G lanes share a row, with NV vectors each; K: choices, at most (as many as a lane has to know of its own logits).
// WHOLE: rows are whole vectors.
//
// 16-bit logits: a choice is the maximum of words that hold the logit's order above the expert's number (falling, so that
// the lower one is larger), of which each lane keeps its K largest. fp32: the maximum of the orders, then the lowest
// expert that has it.
template <typename T, int G, int NV, int K, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_route_fwd(RouteArgs a)
{
    constexpr int N = Vec<T>::N, kGroups = kBlock / G;
    constexpr bool HALF = sizeof(T) == 2;
    constexpr int kOwn = K < N * NV ? K : N * NV;          // of a lane's own logits that can be chosen
    constexpr int M = K > G ? K / G : 1;                    // choices that a lane writes
    typedef typename Vec<T>::Packed Packed;
    const int lane = threadIdx.x & (G - 1);
    const T* end = (const T*)a.logits + (a.rows - 1) * a.ldl + a.experts;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    Packed next[NV];
    auto fetch = [&](int64_t r) {
        const T* row = (const T*)a.logits + r * a.ldl;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (q * G + lane) * N;
            const bool in = c < a.experts;   // (other lanes load the row's first vector)
            next[q] = get_vec<T, WHOLE>(row + (in ? c : 0), in ? a.experts - c : a.experts, end);
        }
    };
    uint32_t numbers[HALF ? NV : 1][HALF ? N : 1];   // of the lane's experts, in the low bits of their words
    if constexpr (HALF)
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int e = 0; e < N; ++e) numbers[q][e] = 0xFFFF - ((q * G + lane) * N + e);
    const int64_t first = (int64_t)blockIdx.x * kGroups + threadIdx.x / G;
    if (first < a.rows) fetch(first);
    for (int64_t r = first; r < a.rows; r += step) {
        Packed raw[NV];
#pragma unroll
        for (int q = 0; q < NV; ++q) raw[q] = next[q];
        if (r + step < a.rows) fetch(r + step);
        uint32_t own[kOwn] = {}, key[HALF ? 1 : NV][HALF ? 1 : N];
        if constexpr (HALF) {
            // what lies beyond the row is masked
            u16x2 sizes = {0, 0};
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                Words w = __builtin_bit_cast(Words, raw[q]);
                const int left = a.experts - (q * G + lane) * N;
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    uint32_t pair = w[e / 2];
                    if (WHOLE) {
                        pair = left > 0 ? pair : Order16<T>::kMasked;
                    } else {
                        pair = left > e + 1 ? pair : left > e ? (pair & 0xFFFF) | (Order16<T>::kMasked & 0xFFFF0000u)
                                                              : Order16<T>::kMasked;
                    }
                    w[e / 2] = pair;
                    sizes = __builtin_elementwise_max(sizes, __builtin_bit_cast(u16x2, pair & 0x7FFF7FFFu));
                }
                raw[q] = __builtin_bit_cast(Packed, w);
            }
            // undefined values: one at a time
            const bool odd = sizes[0] > Order16<T>::kInf || sizes[1] > Order16<T>::kInf;
            if (__builtin_expect(__ballot(odd) != 0, 0)) {
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const uint32_t pair = __builtin_bit_cast(Words, raw[q])[e / 2], o = Order16<T>::of(pair);
                        const bool undefined = (float)raw[q][e] != (float)raw[q][e];
                        insert<kOwn>(own, (undefined ? 0xFFFF0000u : e & 1 ? o & 0xFFFF0000u : o << 16) | numbers[q][e]);
                    }
            } else {
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < N; e += 2) {
                        const uint32_t pair = __builtin_bit_cast(Words, raw[q])[e / 2], o = Order16<T>::of(pair);
                        insert<kOwn>(own, o << 16 | numbers[q][e]);
                        insert<kOwn>(own, (o & 0xFFFF0000u) | numbers[q][e + 1]);
                    }
            }
        } else {
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    key[q][e] = (q * G + lane) * N + e < a.experts ? order_of((float)raw[q][e]) : 0;
        }
        float top = 0.f, total = 0.f, mine[M];
        int32_t number[M];
        bool left = true;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            mine[m] = 0.f;
            number[m] = -1;
#pragma unroll
            for (int jj = 0; jj < G && m * G + jj < K; ++jj) {
                if (m * G + jj >= a.k) break;
                float v;
                int32_t chosen;
                if constexpr (HALF) {
                    const uint32_t best = group_max<G>(own[0]);
                    left = left && best >> 16 > Order16<T>::kNone;
                    v = Order16<T>::value(best >> 16);
                    chosen = 0xFFFF - (int)(best & 0xFFFF);
                    const bool taken = own[0] == best;
#pragma unroll
                    for (int k = 0; k + 1 < kOwn; ++k) own[k] = taken ? own[k + 1] : own[k];
                    own[kOwn - 1] = taken ? 0 : own[kOwn - 1];
                } else {
                    uint32_t best = 0, at = 0x7FFFFFFF;
#pragma unroll
                    for (int q = 0; q < NV; ++q)
#pragma unroll
                        for (int e = 0; e < N; ++e) best = key[q][e] > best ? key[q][e] : best;
                    best = group_max<G>(best);
                    left = left && best > kNone;
                    v = order_value(best);
#pragma unroll
                    for (int q = NV - 1; q >= 0; --q)
#pragma unroll
                        for (int e = N - 1; e >= 0; --e) at = key[q][e] == best ? (q * G + lane) * N + e : at;
                    at = group_min<G>(at);
                    chosen = (int32_t)at;
#pragma unroll
                    for (int q = 0; q < NV; ++q)
#pragma unroll
                        for (int e = 0; e < N; ++e) key[q][e] = (q * G + lane) * N + e == (int)at ? 0 : key[q][e];
                }
                if (m == 0 && jj == 0) top = v;
                const float p = left ? exp_of(v - top) : 0.f;
                total += p;
                if (lane == jj) {
                    mine[m] = p;
                    number[m] = left ? chosen : -1;
                }
            }
        }
        if (!a.normalise) {
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    s += HALF || (q * G + lane) * N + e < a.experts ? exp_of((float)raw[q][e] - top) : 0.f;
            total = group_sum<G>(s);
        }
        const float inv = __builtin_amdgcn_rcpf(total);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int j = m * G + lane;
            if (j >= a.k) break;
            a.expert[r * a.k + j] = number[m];
            a.weight[r * a.k + j] = number[m] < 0 ? 0.f : mine[m] * inv;
        }
    }
}

constexpr int kRouteChoices = 4;   // of a row under way together

template <typename T, int G, int NV>
__global__ __launch_bounds__(kBlock) void k_route_bwd(RouteArgs a)
{
    constexpr int N = Vec<T>::N, kGroups = kBlock / G, U = kRouteChoices;
    typedef typename Vec<T>::Packed Packed;
    const int lane = threadIdx.x & (G - 1);
    const T* end = (const T*)a.logits + (a.rows - 1) * a.ldl + a.experts;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G; r < a.rows; r += step) {
        const int64_t at = r * a.k;
        float p[NV][N], d[NV][N];
        Packed raw[NV];
        int32_t expert[U];
        float w[U], dw[U];
        auto choices = [&](int j0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = j0 + u < a.k;
                expert[u] = in ? a.expert[at + j0 + u] : -1;
                w[u] = in ? a.weight[at + j0 + u] : 0.f;
                dw[u] = in ? a.dweight[at + j0 + u] : 0.f;
            }
        };
        if (!a.normalise)
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                const int c = (q * G + lane) * N;
                if (c < a.experts) raw[q] = get_vec<T, false>((const T*)a.logits + r * a.ldl + c, a.experts - c, end);
            }
        float inner = 0.f;
        for (int j0 = 0; j0 < a.k; j0 += U) {
            choices(j0);
#pragma unroll
            for (int u = 0; u < U; ++u) inner = expert[u] >= 0 ? fmaf(dw[u], w[u], inner) : inner;
        }
        if (!a.normalise) {
            float top = -__builtin_inff(), s = 0.f;
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    p[q][e] = (q * G + lane) * N + e < a.experts ? (float)raw[q][e] : -__builtin_inff();
                    top = fmaxf(top, p[q][e]);
                }
            top = group_maxf<G>(top);
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    p[q][e] = top == -__builtin_inff() ? 0.f : exp_of(p[q][e] - top);
                    s += p[q][e];
                }
            s = group_sum<G>(s);
            const float inv = s == 0.f ? 0.f : 1.f / s;   // (a row without experts)
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    p[q][e] *= inv;
                    d[q][e] = -p[q][e] * inner;
                }
        } else {
#pragma unroll
            for (int q = 0; q < NV; ++q)
#pragma unroll
                for (int e = 0; e < N; ++e) d[q][e] = 0.f;
        }
        for (int j0 = 0; j0 < a.k; j0 += U) {
            if (a.k > U) choices(j0);   // (else they are still here)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float t = dw[u] - inner;
#pragma unroll
                for (int q = 0; q < NV; ++q)
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if ((q * G + lane) * N + e == expert[u]) d[q][e] = (a.normalise ? w[u] : p[q][e]) * t;
            }
        }
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            const int c = (q * G + lane) * N;
            if (c < a.experts) put_floats<T, false>((T*)a.dlogits + r * a.ldd + c, a.experts - c, d[q]);
        }
    }
}

template <typename T, int G, int NV, bool WHOLE>
void route_fwd(const RouteArgs& a, dim3 grid, hipStream_t s)
{
    if (a.k <= 2)
        hipLaunchKernelGGL((k_route_fwd<T, G, NV, 2, WHOLE>), grid, dim3(kBlock), 0, s, a);
    else if (a.k <= 4)
        hipLaunchKernelGGL((k_route_fwd<T, G, NV, 4, WHOLE>), grid, dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL((k_route_fwd<T, G, NV, GS_MAX_CHOICES, WHOLE>), grid, dim3(kBlock), 0, s, a);
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
        else if (a.experts % Vec<T>::N == 0)
            route_fwd<T, G, NV, true>(a, grid, s);
        else
            route_fwd<T, G, NV, false>(a, grid, s);
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
