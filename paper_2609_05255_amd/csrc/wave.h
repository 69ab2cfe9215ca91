// Ranking keys within a wave: shared by the radix sorts of sort.hip and sort_rows.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gsr {

__device__ __forceinline__ uint64_t lanemask_lt() { return (1ull << __lane_id()) - 1ull; }

// Lanes of this wave holding the same kBits-bit digit (restricted to valid lanes).
template <int kBits>
__device__ __forceinline__ uint64_t match_digit(uint32_t d, bool valid)
{
    const uint64_t v = __ballot(valid);
    uint32_t lo = (uint32_t)v, hi = (uint32_t)(v >> 32);
#pragma unroll
    for (int b = 0; b < kBits; ++b) {
        const uint32_t bit = (d >> b) & 1u;
        const uint64_t bm = __ballot(bit);
        const uint32_t s = 0u - bit;   // all ones where this lane's bit is set
        // keep the lanes whose bit equals ours: bm where set, ~bm where clear
        lo &= ~((uint32_t)bm ^ s);
        hi &= ~((uint32_t)(bm >> 32) ^ s);
    }
    return ((uint64_t)hi << 32) | lo;
}

}  // namespace gsr
