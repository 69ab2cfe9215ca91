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
    int32_t unit, units;           // of the expert
    int32_t before;                // units of the experts before
};

__device__ __forceinline__ int32_t mix_offset(const Mix& m, int e)
{
    const int64_t o = m.offsets[e];
    return (int32_t)(o < 0 ? 0 : o < m.rows ? o : m.rows);   // (never beyond the matrices, whatever the array holds)
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Sum over the lanes up to this one: within rows of 16 lanes, then from row to row.
__device__ __forceinline__ int32_t sum_upto(int32_t v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // 1, 2, 4 and 8 lanes before
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // lane 15 of the row before, rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // lane 31, rows 2 and 3
    return v;
}

// Units of `size` rows (the last of an expert: fewer), `least` at least for each expert. A wave looks at 64 experts at a
// time; every wave of a workgroup does, with all its lanes, so that nothing has to meet. Units are counted in 31 bits.
struct MixScan {
    int32_t first, rows;           // a lane's expert's
    int32_t units, upto;           // and with those of the lanes before

    __device__ __forceinline__ MixScan(const Mix& m, int e0, int size, int least)
    {
        const int lane = threadIdx.x & 63, e = e0 + lane;
        first = rows = units = 0;
        if (e < m.experts) {
            first = mix_offset(m, e);
            const int32_t end = mix_offset(m, e + 1);
            rows = end > first ? end - first : 0;
            units = (int32_t)(((uint32_t)rows + (uint32_t)size - 1) / (uint32_t)size);
            units = units < least ? least : units;
        }
        upto = sum_upto(units);
    }
    __device__ __forceinline__ int32_t total() const { return __builtin_amdgcn_readlane(upto, 63); }
    __device__ __forceinline__ int32_t before() const { return upto - units; }
    // lane l's, after `past` units of the experts before the 64
    __device__ __forceinline__ MixUnit unit(int e0, int l, int32_t past) const
    {
        const int32_t n = __builtin_amdgcn_readlane(units, l);
        return {e0 + l, __builtin_amdgcn_readlane(first, l), __builtin_amdgcn_readlane(rows, l), 0, n,
                past + __builtin_amdgcn_readlane(upto, l) - n};
    }
};

__device__ __forceinline__ int32_t mix_total(const Mix& m, int size, int least)
{
    int32_t total = 0;
    for (int e0 = 0; e0 < m.experts; e0 += 64) total += MixScan(m, e0, size, least).total();
    return total;
}

// The unit number `at` of all.
__device__ __forceinline__ MixUnit mix_unit(const Mix& m, int size, int least, int32_t at)
{
    int32_t past = 0;
    for (int e0 = 0; e0 < m.experts; e0 += 64) {
        const MixScan s(m, e0, size, least);
        const uint64_t hit = __ballot(at >= past + s.before() && at < past + s.upto);
        if (hit) {
            MixUnit u = s.unit(e0, __builtin_ctzll(hit), past);
            u.unit = at - u.before;
            return u;
        }
        past += s.total();
    }
    return {-1, 0, 0, 0, 0, 0};
}

// The units of expert e.
__device__ __forceinline__ MixUnit mix_expert(const Mix& m, int size, int least, int e)
{
    int32_t past = 0;
    for (int e0 = 0; e0 < m.experts; e0 += 64) {
        const MixScan s(m, e0, size, least);
        if (e < e0 + 64) return s.unit(e0, e - e0, past);
        past += s.total();
    }
    return {-1, 0, 0, 0, 0, 0};
}

// The units of the experts before e that have several.
__device__ __forceinline__ int64_t mix_parts_before(const Mix& m, int size, int e)
{
    int32_t sum = 0;
    for (int e0 = 0; e0 < e; e0 += 64) {
        const MixScan s(m, e0, size, 0);
        const int32_t v = e0 + (int)(threadIdx.x & 63) < e && s.units > 1 ? s.units : 0;
        sum += __builtin_amdgcn_readlane(sum_upto(v), 63);
    }
    return sum;
}

}  // namespace gsr
