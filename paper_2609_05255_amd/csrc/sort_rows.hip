// Rows sorted by a key, stably: the order in which an embedding's gradient is summed and in which experts take their
// rows.
//
//   order: positions in order of (key, position), those without a group behind the others
//   sorted[p] = the key of order[p], place[order[p]] = p (-1: no group),
//   offsets[g] = number of positions with a key below g
//
// A least-significant-digit radix sort of up to 8 bits a pass over keys in [0, groups] (groups: none). One pass is
// k_keys_count (digit counts of each workgroup's keys, and their sums over groups of workgroups) and k_keys_move (each
// workgroup adds up the counts before its own, ranks its keys by ballots, reorders them by digit in LDS and writes each
// digit's run). Where one pass is enough the offsets are its digits' totals; otherwise k_offsets searches the sorted
// keys. Up to kSmallCount keys one workgroup sorts in LDS, in one launch.
#include "gs_internal.h"
#include "wave.h"

namespace gsr {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigits = 256;
constexpr int kItems = 4, kKeysTile = kThreads * kItems;   // keys of a workgroup
constexpr int kSmallCount = 8192;
constexpr int kSmallGroups = 16384;      // whose offsets the one workgroup writes as well

__device__ __forceinline__ uint32_t key_of(const int32_t* group_of, int64_t i, uint32_t groups)
{
    const uint32_t k = (uint32_t)group_of[i];
    return k < groups ? k : groups;   // (negative ones are large)
}

// Exclusive scan of one value per thread over the workgroup.
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) before += w < wave ? lds[w] : 0;
    __syncthreads();
    return before + x - v;
}

struct KeysPass {
    const int32_t* group_of;     // the first pass, else NULL
    const uint32_t* keys_in;     // the others
    const uint32_t* vals_in;
    int64_t count;
    uint32_t groups;
    int32_t shift;
    uint32_t* hist;              // [workgroups][kDigits]
    uint32_t* sup;               // [workgroups / group][kDigits], cleared beforehand
    int32_t group;
    uint32_t* keys_out;          // or NULL
    uint32_t* vals_out;
    int32_t* place;              // the last pass, or NULL
    int32_t* offsets;            // the only pass, or NULL
};

__device__ __forceinline__ uint32_t pass_key(const KeysPass& a, int64_t i)
{
    return a.group_of ? key_of(a.group_of, i, a.groups) : a.keys_in[i];
}

__global__ __launch_bounds__(kThreads) void k_keys_count(KeysPass a)
{
    // 16 copies of the counts, so that few lanes of an instruction meet on the counter of a frequent digit
    __shared__ uint32_t h[16][kDigits];
    for (int k = threadIdx.x; k < 16 * kDigits; k += kThreads) (&h[0][0])[k] = 0;
    __syncthreads();
    const int copy = ((threadIdx.x >> 6) & 3) * 4 + (threadIdx.x & 3);
    const int64_t base = (int64_t)blockIdx.x * kKeysTile;
    uint32_t k[kItems];
#pragma unroll
    for (int r = 0; r < kItems; ++r) {
        const int64_t i = base + r * kThreads + threadIdx.x;
        k[r] = i < a.count ? pass_key(a, i) : 0;
    }
#pragma unroll
    for (int r = 0; r < kItems; ++r)
        if (base + r * kThreads + threadIdx.x < a.count) atomicAdd(&h[copy][(k[r] >> a.shift) & (kDigits - 1)], 1u);
    __syncthreads();
    if (threadIdx.x >= kDigits) return;
    uint32_t c = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) c += h[w][threadIdx.x];
    a.hist[(int64_t)blockIdx.x * kDigits + threadIdx.x] = c;
    if (c) atomicAdd(&a.sup[(int64_t)(blockIdx.x / a.group) * kDigits + threadIdx.x], c);
}

// Ranks a wave's slice of ITEMS * 64 keys by digit: rank[k] = keys of the same digit before the lane's k-th one in the
// slice; counts[digit] of the wave (cleared beforehand) ends up as their number.
template <int ITEMS>
__device__ __forceinline__ void rank_slice(const uint32_t (&digit)[ITEMS], const bool (&valid)[ITEMS],
                                           uint32_t* counts, uint32_t (&rank)[ITEMS])
{
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const uint64_t same = match_digit<8>(digit[k], valid[k]);
        const uint32_t below = __popcll(same & lanemask_lt());
        uint32_t base = 0;
        if (valid[k]) base = counts[digit[k]];
        rank[k] = base + below;
        // (LDS keeps a wave's order: all its lanes have read before the first lane of each digit writes)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (valid[k] && below == 0) counts[digit[k]] = base + (uint32_t)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

__global__ __launch_bounds__(kThreads) void k_keys_move(KeysPass a)
{
    __shared__ uint32_t counts[kWaves][kDigits];   // of each wave, then the first place of its keys of each digit
    __shared__ uint32_t start[kDigits];            // global place of a digit's first key, less its place in the workgroup
    __shared__ uint32_t buf_k[kKeysTile], buf_v[kKeysTile];
    __shared__ uint32_t sums[2][4][kDigits], lds[kWaves];
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
    const int64_t base = (int64_t)blockIdx.x * kKeysTile;
    const int n = (int)(a.count - base < kKeysTile ? a.count - base : kKeysTile);
    const int at0 = wave * kItems * 64 + lane;
    uint32_t key[kItems], digit[kItems], val[kItems], rank[kItems];
    bool valid[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = at0 + k * 64;
        valid[k] = i < n;
        key[k] = valid[k] ? pass_key(a, base + i) : 0;
        val[k] = a.vals_in && valid[k] ? a.vals_in[base + i] : (uint32_t)(base + i);
        digit[k] = (key[k] >> a.shift) & (kDigits - 1);
    }
    for (int k = t; k < kWaves * kDigits; k += kThreads) (&counts[0][0])[k] = 0;
    {   // the digits' totals, and those before this workgroup: four threads a digit
        const int d = t & (kDigits - 1), q = t >> 8;
        const int64_t mine = blockIdx.x / a.group, groups = (gridDim.x + a.group - 1) / a.group;
        uint32_t total = 0, before = 0;
        for (int64_t g = q; g < groups; g += 4) {
            const uint32_t v = a.sup[g * kDigits + d];
            total += v;
            before += g < mine ? v : 0;
        }
        for (int64_t b = mine * a.group + q; b < blockIdx.x; b += 4) before += a.hist[b * kDigits + d];
        sums[0][q][d] = total;
        sums[1][q][d] = before;
    }
    __syncthreads();
    rank_slice<kItems>(digit, valid, counts[wave], rank);
    uint32_t total = 0, before = 0, here = 0;
    __syncthreads();
    if (t < kDigits) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            total += sums[0][q][t];
            before += sums[1][q][t];
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) here += counts[w][t];
    }
    const uint32_t first = scan_before(total, lds);   // global place of the digit's first key
    const uint32_t local = scan_before(here, lds);    // place in the workgroup
    if (t < kDigits) {
        start[t] = first + before - local;
        uint32_t c = local;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t mine = counts[w][t];
            counts[w][t] = c;
            c += mine;
        }
        if (a.offsets && blockIdx.x == 0 && t <= (int)a.groups) a.offsets[t] = (int32_t)first;
    }
    // (groups = 256: the keys of no group would be a 257th digit, and the pass is not the only one)
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        if (!valid[k]) continue;
        const uint32_t at = counts[wave][digit[k]] + rank[k];
        buf_k[at] = key[k];
        buf_v[at] = val[k];
        if (a.place) a.place[val[k]] = key[k] < a.groups ? (int32_t)(start[digit[k]] + at) : -1;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int at = k * kThreads + t;
        if (at >= n) continue;
        const uint32_t q = buf_k[at];
        const int64_t to = (int64_t)start[(q >> a.shift) & (kDigits - 1)] + at;
        if (a.keys_out) a.keys_out[to] = q;
        a.vals_out[to] = buf_v[at];
    }
}

// First of sorted[0, count) that is not below `key`.
__device__ __forceinline__ uint32_t first_at(const uint32_t* sorted, uint32_t count, uint32_t key)
{
    uint32_t lo = 0, hi = count;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (sorted[mid] < key)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kBlock) void k_offsets(const uint32_t* __restrict__ sorted, uint32_t count,
                                                    uint32_t groups, int32_t* __restrict__ offsets)
{
    const int64_t g = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (g <= groups) offsets[g] = (int32_t)first_at(sorted, count, (uint32_t)g);
}

// All passes over a few keys by one workgroup.
__global__ __launch_bounds__(kThreads) void k_keys_small(const int32_t* __restrict__ group_of, int count,
                                                         uint32_t groups, int bits, int32_t* __restrict__ order,
                                                         int32_t* __restrict__ sorted, int32_t* __restrict__ place,
                                                         int32_t* __restrict__ offsets)
{
    constexpr int kI = kSmallCount / kThreads;
    __shared__ uint32_t counts[kWaves][kDigits];
    __shared__ uint32_t buf_k[kSmallCount], lds[kWaves];
    __shared__ uint16_t buf_v[kSmallCount];
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
    const int at0 = wave * kI * 64 + lane;
    uint32_t key[kI], val[kI], digit[kI], rank[kI];
    bool valid[kI];
#pragma unroll
    for (int k = 0; k < kI; ++k) {
        const int i = at0 + k * 64;
        valid[k] = i < count;
        key[k] = valid[k] ? key_of(group_of, i, groups) : 0;
        val[k] = i;
    }
    for (int shift = 0;; shift += 8) {
#pragma unroll
        for (int k = 0; k < kI; ++k) digit[k] = (key[k] >> shift) & (kDigits - 1);
        for (int k = t; k < kWaves * kDigits; k += kThreads) (&counts[0][0])[k] = 0;
        __syncthreads();
        rank_slice<kI>(digit, valid, counts[wave], rank);
        __syncthreads();
        uint32_t here = 0;
        if (t < kDigits)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) here += counts[w][t];
        uint32_t c = scan_before(here, lds);
        if (t < kDigits)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t mine = counts[w][t];
                counts[w][t] = c;
                c += mine;
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kI; ++k) {
            if (!valid[k]) continue;
            const uint32_t at = counts[wave][digit[k]] + rank[k];
            buf_k[at] = key[k];
            buf_v[at] = (uint16_t)val[k];
        }
        __syncthreads();
        if (shift + 8 >= bits) break;
#pragma unroll
        for (int k = 0; k < kI; ++k)
            if (valid[k]) {
                key[k] = buf_k[at0 + k * 64];
                val[k] = buf_v[at0 + k * 64];
            }
    }
    for (int p = t; p < count; p += kThreads) {
        const uint32_t k = buf_k[p], i = buf_v[p];
        order[p] = (int32_t)i;
        if (sorted) sorted[p] = (int32_t)k;
        if (place) place[i] = k < groups ? p : -1;
    }
    if (offsets)
        for (uint32_t g = t; g <= groups; g += kThreads) offsets[g] = (int32_t)first_at(buf_k, (uint32_t)count, g);
}

int bits_of(int64_t groups)   // of keys up to `groups`
{
    int b = 1;
    while (groups >> b) ++b;
    return b;
}

int passes_of(int64_t groups) { return (int)div_up(bits_of(groups), 8); }

struct SortSpace {
    uint32_t *hist, *sup, *keys[2], *vals[2];
    int64_t blocks, group, groups;   // workgroups, of them in a group, and groups
    size_t bytes;
};

SortSpace sort_space(void* base, int64_t count, int64_t groups)
{
    SortSpace w = {};
    size_t at = 0;
    auto take = [&](int64_t values) {
        uint32_t* p = base ? (uint32_t*)((char*)base + at) : nullptr;
        at += align_up((size_t)values * 4, 256);
        return p;
    };
    const int passes = passes_of(groups);
    if (count > kSmallCount) {
        w.blocks = div_up(count, kKeysTile);
        w.group = 1;
        while (w.group * w.group < w.blocks) ++w.group;
        w.groups = div_up(w.blocks, w.group);
        w.hist = take(w.blocks * kDigits);
        w.sup = take(passes * w.groups * kDigits);
        // the last pass writes the caller's arrays, or keys that only the offsets are read from
        for (int k = 0; k < 2; ++k) {
            if (passes > 1) w.keys[k] = take(count);
            if (passes > k + 1) w.vals[k] = take(count);
        }
    } else if (groups > kSmallGroups) {
        w.keys[0] = take(count);
    }
    w.bytes = at;
    return w;
}

}  // namespace

size_t sort_rows_workspace(int64_t count, int64_t groups) { return sort_space(nullptr, count, groups).bytes; }

hipError_t launch_sort_rows(const int32_t* group_of, const gs_row_order& o, void* ws, hipStream_t s)
{
    const SortSpace w = sort_space(ws, o.count, o.groups);
    const int passes = passes_of(o.groups);
    auto find_offsets = [&](const uint32_t* sorted) {
        hipLaunchKernelGGL(k_offsets, dim3((unsigned)div_up(o.groups + 1, kBlock)), dim3(kBlock), 0, s, sorted,
                           (uint32_t)o.count, (uint32_t)o.groups, o.offsets);
        return hipGetLastError();
    };
    if (o.count <= kSmallCount) {
        const bool few = o.groups <= kSmallGroups;
        int32_t* sorted = o.sorted || few ? o.sorted : (int32_t*)w.keys[0];
        hipLaunchKernelGGL(k_keys_small, dim3(1), dim3(kThreads), 0, s, group_of, (int)o.count, (uint32_t)o.groups,
                           bits_of(o.groups), o.order, sorted, o.place, few ? o.offsets : nullptr);
        const hipError_t e = hipGetLastError();
        return e != hipSuccess || few ? e : find_offsets((const uint32_t*)sorted);
    }
    hipError_t e = launch_fill_u32(w.sup, passes * w.groups * kDigits, 0u, s);
    KeysPass a = {};
    a.count = o.count;
    a.groups = (uint32_t)o.groups;
    a.group = (int32_t)w.group;
    a.hist = w.hist;
    for (int p = 0; p < passes && e == hipSuccess; ++p) {
        const bool last = p + 1 == passes;
        a.group_of = p == 0 ? group_of : nullptr;
        a.keys_in = p == 0 ? nullptr : w.keys[(p - 1) & 1];
        a.vals_in = p == 0 ? nullptr : w.vals[(p - 1) & 1];
        a.shift = 8 * p;
        a.sup = w.sup + p * w.groups * kDigits;
        a.keys_out = last && (o.sorted || passes == 1) ? (uint32_t*)o.sorted : w.keys[p & 1];
        a.vals_out = last ? (uint32_t*)o.order : w.vals[p & 1];
        a.place = last ? o.place : nullptr;
        a.offsets = passes == 1 ? o.offsets : nullptr;
        hipLaunchKernelGGL(k_keys_count, dim3((unsigned)w.blocks), dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(k_keys_move, dim3((unsigned)w.blocks), dim3(kThreads), 0, s, a);
        e = hipGetLastError();
    }
    return e != hipSuccess || passes == 1 ? e : find_offsets(a.keys_out);
}

}  // namespace gsr
