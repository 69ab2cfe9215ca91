// Rows sorted by a key, stably: the order in which an embedding's gradient is summed and in which experts take their
// rows.
//
//   order: positions in order of (key, position), those without a group behind the others
//   sorted[p] = the key of order[p], place[order[p]] = p (-1: no group),
//   offsets[g] = number of positions with a key below g
//
// A least-significant-digit radix sort of up to 9 bits a pass over keys in [0, groups] (groups: none). One pass is
// k_keys_count (digit counts of each workgroup's keys, and with many workgroups their sums over groups of these) and
// k_keys_move (each workgroup adds up the counts before its own, ranks its keys by ballots, reorders them by digit in LDS
// and writes each digit's run). Where one pass is enough the offsets are its digits' totals; otherwise k_offsets searches
// the sorted keys. Up to kSmallCount keys one workgroup sorts in LDS, in one launch; with more than kSmallGroups groups
// k_offsets is a second one, which reads the keys back.
//
// Bound by the chain of steps in a workgroup: of the 10 us that one of 4,096 keys took (2,000,000 keys, all workgroups at
// the same time) 3 were reading the counts, 2 adding them up in LDS, where a few digits' now meet, and 0.7 ranking; keys
// and results are 24 MB, 5 us at the rate of a copy. Measured (us a call): 8 keys 5.4, 8,192 keys 10.7, 100,000 by 256
// groups 12.3, 2,000,000 by 16 20, 3,000,000 by 65,536 60 (in two passes; with places, which are written one by one, 91),
// by 1,000,000 82.
#include <type_traits>

#include "gs_internal.h"
#include "wave.h"

namespace gsr {

namespace {

constexpr int kThreads = 1024;           // of a workgroup, or with few keys kFewThreads
constexpr int kFewThreads = 256;
constexpr int kMostBits = 9;             // of a digit
constexpr int kSmallBits = 9;            // of a digit in LDS
constexpr int kSmallCount = 8192;
constexpr int kSmallGroups = 16384;      // whose offsets the one workgroup writes as well
constexpr int kFewBlocks = 64;           // workgroups whose counts the others add up one by one
constexpr int64_t kFewKeys = kFewBlocks * kFewThreads * 4;
// Keys of a thread: 4, or 6 where that many workgroups are more than the compute units hold at once (two each).
constexpr int64_t kFewItems = 512 * kThreads * 4;

__device__ __forceinline__ uint32_t key_of(const int32_t* group_of, int64_t i, uint32_t groups)
{
    const uint32_t k = (uint32_t)group_of[i];
    return k < groups ? k : groups;   // (negative ones are large)
}

// Exclusive scan of one value per thread over the workgroup.
template <int THREADS>
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* lds)
{
    constexpr int kWaves = THREADS / 64;
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
    uint32_t* hist;              // [workgroups][digits]
    uint32_t* sup;               // [workgroups / group][digits], cleared beforehand; NULL: few workgroups
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

template <int BITS, int ITEMS, int THREADS>
__global__ __launch_bounds__(THREADS) void k_keys_count(KeysPass a)
{
    constexpr int R = 1 << BITS;
    // 16 copies of the counts, so that few lanes of an instruction meet on the counter of a frequent digit
    __shared__ uint32_t h[16][R + 1];   // (the copies of a digit in different banks)
    for (int k = threadIdx.x; k < 16 * (R + 1); k += THREADS) (&h[0][0])[k] = 0;
    const int copy = ((threadIdx.x >> 6) & 3) * 4 + (threadIdx.x & 3);
    const int64_t base = (int64_t)blockIdx.x * (THREADS * ITEMS);
    uint32_t k[ITEMS];
#pragma unroll
    for (int r = 0; r < ITEMS; ++r) {
        const int64_t i = base + r * THREADS + threadIdx.x;
        k[r] = i < a.count ? pass_key(a, i) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ITEMS; ++r)
        if (base + r * THREADS + threadIdx.x < a.count) atomicAdd(&h[copy][(k[r] >> a.shift) & (R - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < R; d += THREADS) {
        uint32_t c = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) c += h[w][d];
        a.hist[(int64_t)blockIdx.x * R + d] = c;
        if (a.sup && c) atomicAdd(&a.sup[(int64_t)(blockIdx.x / a.group) * R + d], c);
    }
}

// Ranks a wave's slice of ITEMS * 64 keys by digit: rank[k] = keys of the same digit before the lane's k-th one in the
// slice, the lane's k-th being key 64 k of which `left` there are; counts[digit] of the wave (cleared beforehand) ends up
// as their number.
template <int BITS, int ITEMS>
__device__ __forceinline__ void rank_slice(const uint32_t (&key)[ITEMS], int shift, int left, uint16_t* counts,
                                           uint32_t (&rank)[ITEMS])
{
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const bool valid = k * 64 < left;
        const uint32_t digit = (key[k] >> shift) & ((1 << BITS) - 1);
        const uint64_t same = match_digit<BITS>(digit, valid);
        const uint32_t below = __popcll(same & lanemask_lt());
        uint32_t base = 0;
        if (valid) base = counts[digit];
        rank[k] = base + below;
        // (LDS keeps a wave's order: all its lanes have read before the first lane of each digit writes)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (valid && below == 0) counts[digit] = (uint16_t)(base + (uint32_t)__popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Sums over rows [0, rows) of R digits, of all and of those before `mine`: four digits of a thread and every slice-th row.
// total (or NULL), before: [THREADS * 4 / R slices][R] each.
template <int R, int THREADS>
__device__ __forceinline__ void sum_rows(const uint32_t* table, int64_t rows, int64_t mine, uint32_t* total,
                                         uint32_t* before)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int kQuads = R / 4, kSlices = THREADS / kQuads;
    static_assert(kQuads >= 64, "a wave's digits are of one slice");
    constexpr int kFly = THREADS == kThreads ? 4 : 16;   // (fewer threads have more rows each, and more registers)
    const int quad = threadIdx.x % kQuads, slice = threadIdx.x / kQuads;
    u32x4 t = {0, 0, 0, 0}, b = {0, 0, 0, 0};
    for (int64_t r = slice; r < rows; r += kSlices * kFly) {
        u32x4 v[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int64_t at = r + u * kSlices;
            v[u] = at < rows ? *reinterpret_cast<const u32x4*>(table + at * R + quad * 4) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            t += v[u];
            if (r + u * kSlices < mine) b += v[u];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (total) total[slice * R + quad * 4 + e] = t[e];
        before[slice * R + quad * 4 + e] = b[e];
    }
}

// A digit's keys in all workgroups, and in those before `block`, added to total[R] and before[R] (cleared beforehand): the
// counts of groups of workgroups and then those of the workgroup's own group, or with few workgroups all of them. Four
// digits of a thread and every slice-th row; the rows of both kinds are under way together.
template <int R, int THREADS>
__device__ __forceinline__ void add_rows(const KeysPass& a, uint32_t* total, uint32_t* before)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int kQuads = R / 4, kSlices = THREADS / kQuads, kFly = 4;
    static_assert(kQuads < 64, "a wave has several slices");
    const int quad = threadIdx.x % kQuads, slice = threadIdx.x / kQuads;
    const int64_t mine = a.sup ? blockIdx.x / a.group : blockIdx.x, first = a.sup ? mine * a.group : 0;
    const uint32_t* sums = (a.sup ? a.sup : a.hist) + quad * 4;
    const uint32_t* own = a.hist + first * R + quad * 4;
    const int64_t rows = a.sup ? (gridDim.x + a.group - 1) / a.group : gridDim.x, left = a.sup ? blockIdx.x - first : 0;
    u32x4 t = {0, 0, 0, 0}, b = {0, 0, 0, 0};
    for (int64_t r0 = slice; r0 < rows || r0 < left; r0 += kSlices * kFly) {
        u32x4 v[kFly], w[kFly];
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            const int64_t r = r0 + u * kSlices;
            v[u] = r < rows ? *reinterpret_cast<const u32x4*>(sums + r * R) : u32x4{0, 0, 0, 0};
            w[u] = r < left ? *reinterpret_cast<const u32x4*>(own + r * R) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < kFly; ++u) {
            t += v[u];
            b += w[u];
            if (r0 + u * kSlices < mine) b += v[u];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int d = kQuads; d < 64; d <<= 1) {
            t[e] += (uint32_t)__shfl_xor((int)t[e], d, 64);
            b[e] += (uint32_t)__shfl_xor((int)b[e], d, 64);
        }
        if ((threadIdx.x & 63) < kQuads) {
            atomicAdd(&total[quad * 4 + e], t[e]);
            atomicAdd(&before[quad * 4 + e], b[e]);
        }
    }
}

// (two workgroups on a compute unit: 64 registers)
template <int BITS, int ITEMS, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == kThreads ? 8 : 4) void k_keys_move(KeysPass a)
{
    constexpr int R = 1 << BITS, kTile = THREADS * ITEMS;
    // Many digits: the rows' sums are tables of each slice of threads, up to three (meeting on counters in LDS, and with the
    // registers for all rows at once, a sort of 3,000,000 keys takes 74 us instead of 61). Few: they meet in LDS.
    constexpr bool kTables = R >= 256;
    constexpr int kSlices = kTables ? THREADS * 4 / R : 1, kSums = kSlices * R;
    constexpr int kWaves = THREADS / 64, kEach = R > THREADS ? R / THREADS : 1;   // digits of a thread, neighbours
    static_assert(ITEMS * 64 < 65536 && kTile < 65536, "counts of 16 bits");
    __shared__ uint16_t counts[kWaves][R];         // of each wave, then the first place of its keys of each digit
    __shared__ uint32_t start[R];                  // global place of a digit's first key, less its place in the workgroup
    // keys of a digit: all, and those of the workgroups before; then the workgroup's keys in their order, then the values
    constexpr int kLds = kTables ? 3 * kSums : 2 * kSums + kTile;
    __shared__ __attribute__((aligned(16))) uint32_t buf_sums[kLds > kTile ? kLds : kTile];
    uint32_t *totals = buf_sums, *before0 = buf_sums + kSums, *before1 = before0 + kSums;
    uint32_t* buf = kTables ? buf_sums : buf_sums + 2 * kSums;
    __shared__ uint32_t lds[kWaves];
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
    const int64_t base = (int64_t)blockIdx.x * kTile;
    const int n = (int)(a.count - base < kTile ? a.count - base : kTile);
    const int at0 = wave * ITEMS * 64 + lane;
    uint32_t key[ITEMS], rank[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) key[k] = at0 + k * 64 < n ? pass_key(a, base + at0 + k * 64) : 0;
    for (int k = t; k < kWaves * R; k += THREADS) (&counts[0][0])[k] = 0;
    if constexpr (kTables) {
        if (a.sup) {
            const int64_t mine = blockIdx.x / a.group, left = blockIdx.x - mine * a.group;
            sum_rows<R, THREADS>(a.sup, (gridDim.x + a.group - 1) / a.group, mine, totals, before0);
            sum_rows<R, THREADS>(a.hist + mine * a.group * R, left, left, nullptr, before1);
        } else {
            sum_rows<R, THREADS>(a.hist, gridDim.x, blockIdx.x, totals, before0);
        }
        __syncthreads();
    } else {
        for (int k = t; k < 2 * R; k += THREADS) totals[k] = 0;
        __syncthreads();
        add_rows<R, THREADS>(a, totals, before0);
    }
    rank_slice<BITS, ITEMS>(key, a.shift, n - at0, counts[wave], rank);
    uint32_t here[kEach] = {}, total[kEach] = {}, before[kEach] = {}, all = 0, all_here = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int d = t * kEach + k;
        if (d >= R) break;
#pragma unroll
        for (int q = 0; q < kSlices; ++q) {
            total[k] += totals[q * R + d];
            before[k] += before0[q * R + d];
            if (kTables && a.sup) before[k] += before1[q * R + d];
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) here[k] += counts[w][d];
        all += total[k];
        all_here += here[k];
    }
    uint32_t first = scan_before<THREADS>(all, lds);      // global place of the digit's first key
    uint32_t local = scan_before<THREADS>(all_here, lds);   // place in the workgroup
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int d = t * kEach + k;
        if (d >= R) break;
        start[d] = first + before[k] - local;
        uint32_t c = local;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t mine = counts[w][d];
            counts[w][d] = (uint16_t)c;
            c += mine;
        }
        if (a.offsets && blockIdx.x == 0 && d <= (int)a.groups) a.offsets[d] = (int32_t)first;
        first += total[k];
        local += here[k];
    }
    __syncthreads();
    uint32_t val[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int i = at0 + k * 64;
        if (i >= n) continue;
        const uint32_t digit = (key[k] >> a.shift) & (R - 1);
        val[k] = a.vals_in ? a.vals_in[base + i] : (uint32_t)(base + i);
        rank[k] += counts[wave][digit];
        buf[rank[k]] = key[k];
        if (a.place) a.place[val[k]] = key[k] < a.groups ? (int32_t)(start[digit] + rank[k]) : -1;
    }
    __syncthreads();
    uint32_t to[ITEMS];   // where the workgroup's places t, t + THREADS, ... go
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int at = k * THREADS + t;
        if (at >= n) continue;
        const uint32_t q = buf[at];
        to[k] = start[(q >> a.shift) & (R - 1)] + at;
        if (a.keys_out) a.keys_out[to[k]] = q;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (at0 + k * 64 < n) buf[rank[k]] = val[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int at = k * THREADS + t;
        if (at < n) a.vals_out[to[k]] = buf[at];
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

// (Starting each search in 1,024 keys that the workgroup has read at once takes 7.0 us instead of 7.9 for 65,537 offsets of
// 3,000,000 keys, but 99 instead of 90 for the whole sort with 1,000,001.)
__global__ __launch_bounds__(kBlock) void k_offsets(const uint32_t* __restrict__ sorted, uint32_t count,
                                                    uint32_t groups, int32_t* __restrict__ offsets)
{
    const int64_t g = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (g <= groups) offsets[g] = (int32_t)first_at(sorted, count, (uint32_t)g);
}

// All passes over a few keys by one workgroup, 8 of a thread.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_keys_small(const int32_t* __restrict__ group_of, int count,
                                                         uint32_t groups, int bits, int32_t* __restrict__ order,
                                                         int32_t* __restrict__ sorted, int32_t* __restrict__ place,
                                                         int32_t* __restrict__ offsets)
{
    constexpr int kI = 8, kKeys = THREADS * kI, kDigits = 1 << kSmallBits, kWaves = THREADS / 64;
    constexpr int kEach = kDigits > THREADS ? kDigits / THREADS : 1;
    __shared__ uint16_t counts[kWaves][kDigits];
    __shared__ uint32_t buf_k[kKeys], lds[kWaves];
    __shared__ uint16_t buf_v[kKeys];
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
    const int at0 = wave * kI * 64 + lane;
    uint32_t key[kI], val[kI], rank[kI];
#pragma unroll
    for (int k = 0; k < kI; ++k) {
        const int i = at0 + k * 64;
        key[k] = i < count ? key_of(group_of, i, groups) : 0;
        val[k] = i;
    }
    for (int shift = 0;; shift += kSmallBits) {
        for (int k = t; k < kWaves * kDigits; k += THREADS) (&counts[0][0])[k] = 0;
        __syncthreads();
        rank_slice<kSmallBits, kI>(key, shift, count - at0, counts[wave], rank);
        __syncthreads();
        uint32_t here = 0;
        if (t * kEach < kDigits)
#pragma unroll
            for (int k = 0; k < kEach; ++k)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) here += counts[w][t * kEach + k];
        uint32_t c = scan_before<THREADS>(here, lds);
        if (t * kEach < kDigits)
#pragma unroll
            for (int k = 0; k < kEach; ++k)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const uint32_t mine = counts[w][t * kEach + k];
                    counts[w][t * kEach + k] = (uint16_t)c;
                    c += mine;
                }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kI; ++k) {
            if (at0 + k * 64 >= count) continue;
            const uint32_t at = counts[wave][(key[k] >> shift) & (kDigits - 1)] + rank[k];
            buf_k[at] = key[k];
            buf_v[at] = (uint16_t)val[k];
        }
        __syncthreads();
        if (shift + kSmallBits >= bits) break;
#pragma unroll
        for (int k = 0; k < kI; ++k)
            if (at0 + k * 64 < count) {
                key[k] = buf_k[at0 + k * 64];
                val[k] = buf_v[at0 + k * 64];
            }
    }
    for (int p = t; p < count; p += THREADS) {
        const uint32_t k = buf_k[p], i = buf_v[p];
        order[p] = (int32_t)i;
        if (sorted) sorted[p] = (int32_t)k;
        if (place) place[i] = k < groups ? p : -1;
    }
    if (offsets)
        for (uint32_t g = t; g <= groups; g += THREADS) offsets[g] = (int32_t)first_at(buf_k, (uint32_t)count, g);
}

int bits_of(int64_t groups)   // of keys up to `groups`
{
    int b = 1;
    while (groups >> b) ++b;
    return b;
}

int passes_of(int64_t groups) { return (int)div_up(bits_of(groups), kMostBits); }

// Bits of a pass's digits that the kernels are built for: 5, 7 or 9.
int digit_bits(int64_t groups)
{
    const int64_t each = div_up(bits_of(groups), passes_of(groups));
    return each <= 5 ? 5 : each <= 7 ? 7 : 9;
}

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
    const int passes = passes_of(groups), digits = 1 << digit_bits(groups);
    if (count > kSmallCount) {
        w.blocks = div_up(count, count <= kFewKeys ? kFewThreads * 4 : kThreads * (count <= kFewItems ? 4 : 6));
        w.hist = take(w.blocks * digits);
        w.group = 1;
        if (w.blocks > kFewBlocks) {
            while (w.group * w.group < w.blocks) ++w.group;
            w.groups = div_up(w.blocks, w.group);
            w.sup = take(passes * w.groups * digits);
        }
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

template <int BITS>
hipError_t sort_pass(const KeysPass& a, int64_t blocks, hipStream_t s)
{
    auto run = [&](auto items, auto threads) {
        constexpr int ITEMS = decltype(items)::value, THREADS = decltype(threads)::value;
        hipLaunchKernelGGL((k_keys_count<BITS, ITEMS, THREADS>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
        hipLaunchKernelGGL((k_keys_move<BITS, ITEMS, THREADS>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
    };
    using std::integral_constant;
    if (a.count <= kFewKeys)
        run(integral_constant<int, 4>(), integral_constant<int, kFewThreads>());
    else if (a.count <= kFewItems)
        run(integral_constant<int, 4>(), integral_constant<int, kThreads>());
    else
        run(integral_constant<int, 6>(), integral_constant<int, kThreads>());
    return hipGetLastError();
}

}  // namespace

size_t sort_rows_workspace(int64_t count, int64_t groups) { return sort_space(nullptr, count, groups).bytes; }

hipError_t launch_sort_rows(const int32_t* group_of, const gs_row_order& o, void* ws, hipStream_t s)
{
    const SortSpace w = sort_space(ws, o.count, o.groups);
    const int passes = passes_of(o.groups), bits = digit_bits(o.groups);
    auto find_offsets = [&](const uint32_t* sorted) {
        hipLaunchKernelGGL(k_offsets, dim3((unsigned)div_up(o.groups + 1, kBlock)), dim3(kBlock), 0, s, sorted,
                           (uint32_t)o.count, (uint32_t)o.groups, o.offsets);
        return hipGetLastError();
    };
    if (o.count <= kSmallCount) {
        const bool few = o.groups <= kSmallGroups;
        int32_t* sorted = o.sorted || few ? o.sorted : (int32_t*)w.keys[0];
        auto run = [&](auto threads) {
            constexpr int THREADS = decltype(threads)::value;
            hipLaunchKernelGGL((k_keys_small<THREADS>), dim3(1), dim3(THREADS), 0, s, group_of, (int)o.count,
                               (uint32_t)o.groups, bits_of(o.groups), o.order, sorted, o.place, few ? o.offsets : nullptr);
        };
        if (o.count <= kFewThreads * 8)
            run(std::integral_constant<int, kFewThreads>());
        else
            run(std::integral_constant<int, kThreads>());
        const hipError_t e = hipGetLastError();
        return e != hipSuccess || few ? e : find_offsets((const uint32_t*)sorted);
    }
    const int64_t sup = w.groups << bits;   // values of a pass
    hipError_t e = w.sup ? launch_fill_u32(w.sup, passes * sup, 0u, s) : hipSuccess;
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
        a.shift = bits * p;
        a.sup = w.sup ? w.sup + p * sup : nullptr;
        a.keys_out = last && (o.sorted || passes == 1) ? (uint32_t*)o.sorted : w.keys[p & 1];
        a.vals_out = last ? (uint32_t*)o.order : w.vals[p & 1];
        a.place = last ? o.place : nullptr;
        a.offsets = passes == 1 ? o.offsets : nullptr;
        e = bits == 5 ? sort_pass<5>(a, w.blocks, s) : bits == 7 ? sort_pass<7>(a, w.blocks, s) : sort_pass<9>(a, w.blocks, s);
    }
    return e != hipSuccess || passes == 1 ? e : find_offsets(a.keys_out);
}

}  // namespace gsr
