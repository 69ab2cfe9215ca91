// Rows of several experts one after the other, cut into units of rows of one expert.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gsr {

// Expert e's rows are offsets[e] .. offsets[e + 1] of `rows`.
struct Mix {
    const int32_t* offsets;        // device, [experts + 1]; NULL: no mixture
    int32_t experts;
    int32_t size;                  // rows of a unit, where the kernel does not say
    int64_t rows;                  // of the matrices; those from offsets[experts] on belong to nobody
    int64_t w_stride, dw_stride;   // elements between the experts' weights, and their gradients
    int64_t limit;                 // parts that the workspace holds (more than offsets in order can need)
};

// A unit: its expert, the expert's rows, and which of the expert's units it is.
struct MixUnit {
    int expert;                    // -1: there is no such unit
    int32_t first, rows;           // the expert's
    int64_t unit, units;           // of the expert
    int64_t before;                // units of the experts before
};

__device__ __forceinline__ int32_t mix_offset(const Mix& m, int e)
{
    const int64_t o = m.offsets[e];
    return (int32_t)(o < 0 ? 0 : o < m.rows ? o : m.rows);   // (never beyond the matrices, whatever the array holds)
}

// Units of `size` rows (the last of an expert: fewer), `least` at least for each expert. A wave looks at 64 experts at a
// time; every wave of a workgroup does, so that nothing has to meet. All results are the same in every lane.
struct MixScan {
    int32_t first, rows;
    int64_t units, upto;           // a lane's expert's, and with those of the lanes before
    int64_t total;                 // of the 64

    __device__ __forceinline__ MixScan(const Mix& m, int e0, int size, int least)
    {
        const int lane = threadIdx.x & 63, e = e0 + lane;
        first = rows = 0;
        units = 0;
        if (e < m.experts) {
            first = mix_offset(m, e);
            const int32_t end = mix_offset(m, e + 1);
            rows = end > first ? end - first : 0;
            units = ((int64_t)rows + size - 1) / size;
            units = units < least ? least : units;
        }
        upto = units;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t before = __shfl_up(upto, d, 64);
            if (lane >= d) upto += before;
        }
        total = __shfl(upto, 63, 64);
    }
    __device__ __forceinline__ int64_t before() const { return upto - units; }
};

__device__ __forceinline__ int64_t mix_total(const Mix& m, int size, int least)
{
    int64_t total = 0;
    for (int e0 = 0; e0 < m.experts; e0 += 64) total += MixScan(m, e0, size, least).total;
    return total;
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// The unit number `at` of all.
__device__ __forceinline__ MixUnit mix_unit(const Mix& m, int size, int least, int64_t at)
{
    MixUnit u = {-1, 0, 0, 0, 0, 0};
    int64_t before = 0;
    for (int e0 = 0; e0 < m.experts; e0 += 64) {
        const MixScan s(m, e0, size, least);
        const uint64_t hit = __ballot(at >= before + s.before() && at < before + s.upto);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            u.expert = uniform(e0 + l);
            u.first = uniform(__shfl(s.first, l, 64));
            u.rows = uniform(__shfl(s.rows, l, 64));
            u.units = uniform(__shfl(s.units, l, 64));
            u.before = uniform(before + __shfl(s.before(), l, 64));
            u.unit = uniform(at - u.before);
            return u;
        }
        before += s.total;
    }
    return u;
}

// The units of expert e.
__device__ __forceinline__ MixUnit mix_expert(const Mix& m, int size, int least, int e)
{
    MixUnit u = {e, 0, 0, 0, 0, 0};
    int64_t before = 0;
    for (int e0 = 0; e0 < m.experts; e0 += 64) {
        const MixScan s(m, e0, size, least);
        if (e < e0 + 64) {
            const int l = e - e0;
            u.first = uniform(__shfl(s.first, l, 64));
            u.rows = uniform(__shfl(s.rows, l, 64));
            u.units = uniform(__shfl(s.units, l, 64));
            u.before = uniform(before + __shfl(s.before(), l, 64));
            break;
        }
        before += s.total;
    }
    return u;
}

// The units of the experts before e that have several.
__device__ __forceinline__ int64_t mix_parts_before(const Mix& m, int size, int e)
{
    int64_t sum = 0;
    for (int e0 = 0; e0 < e; e0 += 64) {
        const MixScan s(m, e0, size, 0);
        int64_t v = e0 + (int)(threadIdx.x & 63) < e && s.units > 1 ? s.units : 0;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
        sum += v;
    }
    return uniform(sum);
}

}  // namespace gsr
