// Rows copied to where an index says and added up on their way back: embedding lookup, rows moved to experts and their
// results combined, and the gradients of these.
//
//   lookup   y[i] = s table[index[i]], zero without an entry;  dtable[v] = s sum of dy[i] over index[i] = v
//   dispatch xs[p] = x[order[p] / k];                          dx[i] = sum over j of dxs[place[i k + j]] [+ add]
//   combine  y[i] = sum over j of w[i k + j] ys[place[i k + j]] [+ residual]
//            dys[p] = w[order[p]] dy[order[p] / k],            dw[i k + j] = <dy[i], ys[place[i k + j]]>
//
// All are bound by HBM: every row is read once and written once, in vectors of 16 bytes at any alignment, a group of
// lanes for each row, several rows of a group under way together. Sums are fp32 and have a fixed order: no atomics, the
// same call gives the same bits. Results are rounded to the element type once, as they are stored.
//
// Measured (us, and TB/s of what has to be moved): dispatch of 1,000,000 x 128 in binary16 to two of 16 experts 146 (5.3),
// with the sort 169; combination of 20,003 x 333 in fp32, three choices and a residual 29 (4.2, rows at odd multiples of 4
// bytes); its backward for 8,192 x 4,096 in bfloat16, two choices 75 (4.5); the gradient of 3,000,000 x 64 in binary16 into
// 65,536 entries 98 and 8 for the entries that workgroups share (3.9), with the sort 168 (without it 92 for even shares, 110
// where one entry has all the rows; of 190,000 x 1,024 in bfloat16 133 and 203, as the workgroups that add up an entry's parts
// are as few as its columns in 256s); of 50,001 x 333 in bfloat16 into
// 150,007 entries 20, and 21 for the empty ones' zeros, with the sort 78. A row alone takes 6.6 a call.
#include <type_traits>

#include "gs_internal.h"
#include "rows.h"

namespace gsr {

namespace {

// Lanes that share a row of `vecs` vectors: a power of two up to a wave, from 16 on the one whose last turn leaves the
// fewest idle (84 vectors: three turns of 32 lanes rather than two of 64).
int row_lanes(int64_t vecs)
{
    if (vecs <= 16) return vecs > 8 ? 16 : vecs > 4 ? 8 : vecs > 2 ? 4 : (int)vecs;
    int best = 64;
    for (int g = 32; g >= 16; g >>= 1)
        if (div_up(vecs, g) * g < div_up(vecs, best) * best) best = g;
    return best;
}

template <typename F>
void with_lanes(int g, F f)
{
    switch (g) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    case 16: f(std::integral_constant<int, 16>()); break;
    case 32: f(std::integral_constant<int, 32>()); break;
    default: f(std::integral_constant<int, 64>());
    }
}

constexpr int64_t kMoveBlocks = 256 * 64;   // workgroups at most; they take rows in turn

int64_t move_blocks(int64_t rows, int g, int fly)
{
    return std::max<int64_t>(1, std::min<int64_t>(div_up(rows, (int64_t)kBlock / g * fly), kMoveBlocks));
}

// Behind the last row's end.
template <typename T>
__device__ __forceinline__ const T* end_of(const void* p, int64_t ld, int64_t rows, int64_t dim)
{
    return (const T*)p + (rows - 1) * ld + dim;
}

// ---- one row to one row -----------------------------------------------------

struct GatherArgs {
    const void* src;
    void* dst;
    int64_t lds, ldd, rows, dim;
    const int32_t* index;
    const int32_t* used;   // dispatch: how many rows there are
    int64_t entries;       // lookup: rows of src
    int32_t k;             // dispatch: choices of a row
    float scale;
};

constexpr int kGatherRows = 4;   // neighbours, of a group under way together

// LOOKUP: an index outside [0, entries) gives a row of zeros. Otherwise index[p] / k is the row, below *used. Where there
// is no row to read, the first one is, and left out.
template <typename T, int G, bool LOOKUP, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_gather(GatherArgs a)
{
    constexpr int N = Vec<T>::N, U = kGatherRows, kGroups = kBlock / G;
    constexpr int kIndexed = G < U ? G : U;   // rows that the lanes of a group look up together
    typedef typename Vec<T>::Packed Packed;
    const int lane = threadIdx.x & (G - 1);
    const int64_t rows = LOOKUP ? a.rows : min((int64_t)*a.used, a.rows);
    const T* end = end_of<T>(a.src, a.lds, LOOKUP ? a.entries : a.rows / a.k, a.dim);
    const int64_t step = (int64_t)gridDim.x * kGroups * U;
    for (int64_t r0 = ((int64_t)blockIdx.x * kGroups + threadIdx.x / G) * U; r0 < rows; r0 += step) {
        const T* from[U];
        bool in[U];
#pragma unroll
        for (int q = 0; q < U; q += kIndexed) {
            const int64_t r = r0 + q + (lane & (kIndexed - 1));
            int32_t i = r < rows ? a.index[r] : -1;
            if (LOOKUP)
                i = i >= 0 && i < a.entries ? i : -1;
            else
                i = i >= 0 && i < a.rows ? (int32_t)((uint32_t)i / (uint32_t)a.k) : -1;
#pragma unroll
            for (int u = 0; u < kIndexed; ++u) {
                const int32_t iu = G == 1 ? i : __shfl(i, u, kIndexed);
                in[q + u] = iu >= 0;
                from[q + u] = (const T*)a.src + (int64_t)(iu >= 0 ? iu : 0) * a.lds;
            }
        }
        for (int64_t c = (int64_t)lane * N; c < a.dim; c += G * N) {
            const int64_t left = a.dim - c;
            Packed v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = get_vec<T, WHOLE>(from[u] + c, left, end);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r0 + u >= rows) break;
                T* to = (T*)a.dst + (r0 + u) * a.ldd + c;
                if (LOOKUP) {
                    float f[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = in[u] ? (float)v[u][e] * a.scale : 0.f;
                    put_floats<T, WHOLE>(to, left, f);
                } else if (in[u]) {
                    put_vec<T, WHOLE>(to, left, v[u]);
                }
            }
        }
    }
}

// ---- one row to several -----------------------------------------------------

struct ScatterArgs {
    const void* src;
    void* dst;
    int64_t lds, ldd, rows, dim;
    const int32_t* place;
    const int32_t* used;
    int32_t k;
};

// Rows copied to the places of their choices: x is read once, in order, where the gather reads it once for each choice
// (1,000,000 x 128 in binary16, two of 16 experts: 146 us for 194). An order without places is left to the gather.
template <typename T, int G, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_scatter(ScatterArgs a)
{
    constexpr int N = Vec<T>::N, U = kGatherRows, kGroups = kBlock / G;
    typedef typename Vec<T>::Packed Packed;
    const int lane = threadIdx.x & (G - 1);
    const int64_t used = min((int64_t)*a.used, a.rows * a.k);
    const T* end = end_of<T>(a.src, a.lds, a.rows, a.dim);
    const int64_t step = (int64_t)gridDim.x * kGroups * U;
    for (int64_t r0 = ((int64_t)blockIdx.x * kGroups + threadIdx.x / G) * U; r0 < a.rows; r0 += step)
        for (int64_t c = (int64_t)lane * N; c < a.dim; c += G * N) {
            const int64_t left = a.dim - c;
            Packed v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t r = r0 + u < a.rows ? r0 + u : a.rows - 1;
                v[u] = get_vec<T, WHOLE>((const T*)a.src + r * a.lds + c, left, end);
            }
            for (int j = 0; j < a.k; ++j)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int32_t p = r0 + u < a.rows ? a.place[(r0 + u) * a.k + j] : -1;
                    if (p >= 0 && p < used) put_vec<T, WHOLE>((T*)a.dst + p * a.ldd + c, left, v[u]);
                }
        }
}

// ---- the choices of a row added up ------------------------------------------

struct SumArgs {
    const void* src;       // [sorted rows][dim]
    const void* add;       // [rows][dim] or NULL
    void* dst;
    const float* weight;   // [rows][k], or NULL: 1
    const int32_t* place;
    const int32_t* used;
    int64_t lds, ldadd, ldd, rows, dim;
    int32_t k;
};

constexpr int kSumChoices = 4;   // under way together

// (a choice of no expert loads the first row, which is left out)
template <typename T, int G, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_sum_choices(SumArgs a)
{
    constexpr int N = Vec<T>::N, U = kSumChoices, kGroups = kBlock / G;
    typedef typename Vec<T>::Packed Packed;
    const int lane = threadIdx.x & (G - 1);
    const int64_t used = min((int64_t)*a.used, a.rows * a.k);
    const T *end = end_of<T>(a.src, a.lds, a.rows * a.k, a.dim), *add_end = end_of<T>(a.add, a.ldadd, a.rows, a.dim);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G; r < a.rows; r += step) {
        const int64_t at = r * a.k;
        for (int64_t c = (int64_t)lane * N; c < a.dim; c += G * N) {
            const int64_t left = a.dim - c;
            float sum[N] = {};
            Packed add = {};
            if (a.add) add = get_vec<T, WHOLE>((const T*)a.add + r * a.ldadd + c, left, add_end);
            for (int j0 = 0; j0 < a.k; j0 += U) {
                Packed v[U];
                float w[U];
                bool in[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (j0 + u < a.k) {
                        const int32_t p = a.place[at + j0 + u];
                        w[u] = a.weight ? a.weight[at + j0 + u] : 1.f;
                        in[u] = p >= 0 && p < used;
                        v[u] = get_vec<T, WHOLE>((const T*)a.src + (in[u] ? p : 0) * a.lds + c, left, end);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (j0 + u < a.k && in[u])
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[e] = fmaf(w[u], (float)v[u][e], sum[e]);
            }
            if (a.add)
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += (float)add[e];
            put_floats<T, WHOLE>((T*)a.dst + r * a.ldd + c, left, sum);
        }
    }
}

// ---- the gradients of a combination -----------------------------------------

struct CombineBwdArgs {
    const void *dy, *ys;
    void* dys;
    const float* weight;
    float* dweight;
    const int32_t* place;
    const int32_t* used;
    int64_t lddy, ldys, lddys, rows, dim;
    int32_t k;
};

template <typename T, int G, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_combine_bwd(CombineBwdArgs a)
{
    constexpr int N = Vec<T>::N, U = kSumChoices, kGroups = kBlock / G;
    typedef typename Vec<T>::Packed Packed;
    const int lane = threadIdx.x & (G - 1);
    const int64_t used = min((int64_t)*a.used, a.rows * a.k);
    const T *end = end_of<T>(a.ys, a.ldys, a.rows * a.k, a.dim), *dy_end = end_of<T>(a.dy, a.lddy, a.rows, a.dim);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    for (int64_t r = (int64_t)blockIdx.x * kGroups + threadIdx.x / G; r < a.rows; r += step) {
        const int64_t at = r * a.k;
        for (int j0 = 0; j0 < a.k; j0 += U) {
            int64_t p[U];
            float w[U], dot[U] = {};
            bool in[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j0 + u < a.k) {
                    const int32_t to = a.place[at + j0 + u];
                    w[u] = a.weight[at + j0 + u];
                    in[u] = to >= 0 && to < used;
                    p[u] = in[u] ? to : 0;
                }
            for (int64_t c = (int64_t)lane * N; c < a.dim; c += G * N) {
                const int64_t left = a.dim - c;
                const Packed g = get_vec<T, WHOLE>((const T*)a.dy + r * a.lddy + c, left, dy_end);
                Packed v[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (j0 + u < a.k) v[u] = get_vec<T, WHOLE>((const T*)a.ys + p[u] * a.ldys + c, left, end);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (j0 + u >= a.k || !in[u]) continue;
                    float o[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        if (WHOLE || e < left) dot[u] = fmaf((float)g[e], (float)v[u][e], dot[u]);
                        o[e] = (float)g[e] * w[u];
                    }
                    put_floats<T, WHOLE>((T*)a.dys + p[u] * a.lddys + c, left, o);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (j0 + u >= a.k) continue;
                const float d = group_sum<G>(dot[u]);
                if (lane == 0) a.dweight[at + j0 + u] = d;
            }
        }
    }
}

// ---- the gradient of a lookup -----------------------------------------------
//
// The sorted positions are cut into equal parts, whatever the entries' shares are: a group of lanes sums a part of its
// workgroup's, a row after the other, and writes the entries that begin and end in it. What an entry has in several
// groups meets in LDS, and what it has in several workgroups in k_join_entries, both in the sorted order. Columns beyond
// 64 vectors are other workgroups'.

struct EntriesArgs {
    const void* dy;
    void* dtable;
    int64_t lddy, lddt, dim, entries, count;
    const int32_t *order, *sorted, *offsets;
    float scale;
    float* part;           // [workgroups][2][dim]: sums of the first entry, if it began before, and of the last, if it
                           // began here and does not end here
    int32_t per;           // positions of a group of lanes
    int32_t out_f32;
};

// Rows of a group under way together (4: 3,000,000 x 64 in binary16 106 us for 99, 50,001 x 333 in bfloat16 54 for 49).
constexpr int kEntryRows = 8;

template <typename T>
__device__ __forceinline__ void store_entry(const EntriesArgs& a, int64_t v, int64_t c, float value)
{
    if (a.out_f32)
        ((float*)a.dtable)[v * a.lddt + c] = value * a.scale;
    else
        ((T*)a.dtable)[v * a.lddt + c] = (T)(value * a.scale);
}

// N values, of which the first `left` are the row's.
template <typename T, int N>
__device__ __forceinline__ void store_entries(const EntriesArgs& a, int64_t v, int64_t c, int64_t left, const float* values)
{
    float o[N];
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = values[e] * a.scale;
    if (a.out_f32) {
        float* to = (float*)a.dtable + v * a.lddt + c;
#pragma unroll
        for (int e = 0; e < N; e += 4)
            if (left > e) put_floats<float, false>(to + e, left - e, o + e);
    } else {
        put_floats<T, false>((T*)a.dtable + v * a.lddt + c, left, o);
    }
}

// WHOLE: rows are whole vectors. Lanes behind a row's end load its first vector and store nothing.
template <typename T, int G, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_sum_entries(EntriesArgs a)
{
    constexpr int N = Vec<T>::N, U = kEntryRows, kGroups = kBlock / G, kCols = G * N;
    constexpr int kIndexed = G < U ? G : U;   // positions that the lanes of a group look up together
    typedef typename Vec<T>::Packed Packed;
    // a group's sums of its first entry, and of its last where that is another one
    __shared__ float sums[kGroups][2][kCols];
    __shared__ int32_t keys[kGroups][2];
    const int lane = threadIdx.x & (G - 1), group = threadIdx.x / G;
    const int64_t c = (int64_t)blockIdx.y * kCols + lane * N, left = a.dim - c;
    const int64_t w0 = (int64_t)blockIdx.x * kGroups * a.per;
    const int64_t w1 = w0 + kGroups * a.per < a.count ? w0 + kGroups * a.per : a.count;
    const int32_t key_before = w0 > 0 ? a.sorted[w0 - 1] : -1, key_behind = w1 < a.count ? a.sorted[w1] : -1;
    const int64_t p0 = w0 + (int64_t)group * a.per, p1 = p0 + a.per < w1 ? p0 + a.per : w1;
    const T *dy = (const T*)a.dy + (left > 0 ? c : 0), *end = end_of<T>(a.dy, a.lddy, a.count, a.dim);
    int32_t first = -1, key = -1;
    float sum[N] = {};
    constexpr int kLooks = U / kIndexed;
    uint32_t row_next[kLooks];
    int32_t key_next[kLooks];
    // (positions behind the last one: its row again, and no entry)
    auto look = [&](int64_t p) {
#pragma unroll
        for (int q = 0; q < kLooks; ++q) {
            const int64_t at = p + q * kIndexed + (lane & (kIndexed - 1)), in = at < p1 ? at : p1 - 1;
            const uint32_t i = (uint32_t)a.order[in];
            const int32_t e = a.sorted[in];
            key_next[q] = at >= p1 || i >= a.count || (uint32_t)e >= a.entries ? -1 : e;
            row_next[q] = i < a.count ? i : 0;
        }
    };
    if (p0 < p1) look(p0);
    for (int64_t p = p0; p < p1; p += U) {
        Packed v[U];
        int32_t k[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = u / kIndexed;
            const uint32_t i = G == 1 ? row_next[q] : (uint32_t)__shfl((int)row_next[q], u % kIndexed, kIndexed);
            k[u] = G == 1 ? key_next[q] : __shfl(key_next[q], u % kIndexed, kIndexed);
            v[u] = get_vec<T, WHOLE>(dy + (int64_t)i * a.lddy, left > 0 ? left : a.dim, end);
        }
        if (p + U < p1) look(p + U);   // under the rows' loads
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k[u] < 0) continue;
            if (k[u] != key) {
                if (key == first) {   // (nothing yet, or the first entry)
                    if (key < 0)
                        first = k[u];
                    else
#pragma unroll
                        for (int e = 0; e < N; ++e) sums[group][0][lane * N + e] = sum[e];
                } else if (left > 0) {
                    store_entries<T, N>(a, key, c, left, sum);
                }
                key = k[u];
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += (float)v[u][e];
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sums[group][key == first ? 0 : 1][lane * N + e] = sum[e];
    if (lane == 0) {
        keys[group][0] = first;
        keys[group][1] = key;
    }
    __syncthreads();
    const int32_t w_first = keys[0][0];
    if (w_first < 0) return;   // (rows without an entry are the last ones)
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.dim;
    for (int col = threadIdx.x; col < kCols; col += kBlock) {
        const int64_t cc = (int64_t)blockIdx.y * kCols + col;
        if (cc >= a.dim) break;
        int32_t at = w_first;
        float t = 0.f;
        auto finish = [&](bool last) {
            if (at == w_first && at == key_before)
                part[cc] = t;
            else if (last && at == key_behind)
                part[a.dim + cc] = t;
            else
                store_entry<T>(a, at, cc, t);
        };
        constexpr int kFly = kGroups < 8 ? kGroups : 8;   // groups whose sums are read together
        for (int g0 = 0; g0 < kGroups; g0 += kFly) {
            int32_t k0[kFly], k1[kFly];
            float head[kFly], tail[kFly];
#pragma unroll
            for (int u = 0; u < kFly; ++u) {
                k0[u] = keys[g0 + u][0];
                k1[u] = keys[g0 + u][1];
                head[u] = sums[g0 + u][0][col];
                tail[u] = sums[g0 + u][1][col];
            }
            if (k0[0] < 0) break;
#pragma unroll
            for (int u = 0; u < kFly; ++u) {
                if (k0[u] < 0) continue;
                if (k0[u] != at) {
                    finish(false);
                    at = k0[u];
                    t = 0.f;
                }
                t += head[u];
                if (k1[u] != k0[u]) {
                    finish(false);
                    at = k1[u];
                    t = tail[u];
                }
            }
        }
        finish(true);
    }
}

// Entries that workgroups of k_sum_entries share, a workgroup for each that such an entry begins in, and 16 columns; and
// zeros for the entries that have no rows (the other workgroups).
constexpr int kJoinCols = 16, kJoinSlices = kBlock / kJoinCols;
constexpr int64_t kZeroBlocks = 4096;

template <typename T>
__global__ __launch_bounds__(kBlock) void k_join_entries(EntriesArgs a, int64_t parts, int64_t span, int lanes)
{
    const int64_t first_col = (int64_t)blockIdx.y * kJoinCols * 16;
    const int64_t end_col = min(a.dim, first_col + kJoinCols * 16);
    if (blockIdx.x >= parts) {
        // a wave looks at 64 entries, and each group of a row's lanes clears the empty ones among its share of them
        if (blockIdx.y > 0) return;
        a.scale = 1.f;
        constexpr int N = Vec<T>::N;
        const int lane = threadIdx.x & 63, groups = 64 / lanes, group = lane / lanes, part = lane % lanes;
        const float zero[N] = {};
        const int64_t step = (gridDim.x - parts) * kBlock;
        for (int64_t v0 = (blockIdx.x - parts) * kBlock + (threadIdx.x & ~63); v0 < a.entries; v0 += step) {
            const int64_t v = v0 + lane;
            const uint64_t empty = __ballot(v < a.entries && a.offsets[v] == a.offsets[v + 1]);
            for (int k = group; k < 64; k += groups)
                if (empty >> k & 1)
                    for (int64_t c = (int64_t)part * N; c < a.dim; c += lanes * N)
                        store_entries<T, N>(a, v0 + k, c, a.dim - c, zero);
        }
        return;
    }
    __shared__ float s[kJoinSlices][kJoinCols];
    const int64_t w0 = (int64_t)blockIdx.x * span, w1 = w0 + span;
    if (w1 >= a.count) return;
    const int32_t key = a.sorted[w1 - 1], behind = a.sorted[w1], first = a.sorted[w0];
    const int32_t before = w0 > 0 ? a.sorted[w0 - 1] : -1;
    if (key != behind || key < 0 || key >= a.entries) return;   // it ends here, or is none
    if (first == key && before == key) return;                  // it began before
    const int64_t last = min((int64_t)a.offsets[key + 1] - 1, a.count - 1) / span;
    const int col = threadIdx.x % kJoinCols, slice = threadIdx.x / kJoinCols;
    for (int64_t c0 = first_col; c0 < end_col; c0 += kJoinCols) {
        const int64_t c = c0 + col;
        float t = 0.f;
        if (c < a.dim) {
            if (slice == 0) t = a.part[((int64_t)blockIdx.x * 2 + 1) * a.dim + c];
#pragma unroll 4
            for (int64_t b = blockIdx.x + 1 + slice; b <= last; b += kJoinSlices) t += a.part[b * 2 * a.dim + c];
        }
        s[slice][col] = t;
        __syncthreads();
        if (slice == 0 && c < a.dim) {
#pragma unroll
            for (int k = 1; k < kJoinSlices; ++k) t += s[k][col];
            store_entry<T>(a, key, c, t);
        }
        __syncthreads();
    }
}

// Workgroups of k_sum_entries, about; four times as many of rows of up to 4 vectors, whose lanes then look up positions
// that lie closer together (us with 2,048 and 8,192: 10,000,000 x 8 in binary16 424 and 253, 3,000,000 x 16 119 and 113,
// but 3,000,000 x 64 103 and 105, 1,000,000 x 128 in fp32 112 and 132).
constexpr int64_t kEntryBlocks = 256 * 8;

struct EntriesPlan {
    int lanes;
    int64_t per, span, parts;   // positions of a group and of a workgroup, workgroups
};

EntriesPlan entries_plan(int type, int64_t count, int64_t dim)
{
    EntriesPlan p;
    p.lanes = row_lanes(div_up(dim, type == GS_F32 ? 4 : 8));
    const int64_t groups = kBlock / p.lanes, all = kEntryBlocks * (p.lanes < 8 ? 4 : 1) * groups;
    p.per = std::max<int64_t>(kEntryRows, div_up(div_up(count, all), kEntryRows) * kEntryRows);
    p.span = p.per * groups;
    p.parts = std::max<int64_t>(1, div_up(count, p.span));
    return p;
}

// Calls f with the lanes of a row and whether it ends with a whole vector.
template <typename T, typename F>
hipError_t with_row(int64_t dim, F f)
{
    const int g = row_lanes(div_up(dim, Vec<T>::N));
    with_lanes(g, [&](auto lanes) {
        if (dim % Vec<T>::N == 0)
            f(lanes, std::true_type());
        else
            f(lanes, std::false_type());
    });
    return hipGetLastError();
}

template <typename T>
hipError_t lookup(const GatherArgs& a, hipStream_t s)
{
    return with_row<T>(a.dim, [&](auto lanes, auto whole) {
        constexpr int G = decltype(lanes)::value;
        hipLaunchKernelGGL((k_gather<T, G, true, decltype(whole)::value>),
                           dim3((unsigned)move_blocks(a.rows, G, kGatherRows)), dim3(kBlock), 0, s, a);
    });
}

template <typename T>
hipError_t dispatch(const GatherArgs& a, const int32_t* place, hipStream_t s)
{
    return with_row<T>(a.dim, [&](auto lanes, auto whole) {
        constexpr int G = decltype(lanes)::value;
        constexpr bool WHOLE = decltype(whole)::value;
        if (place) {
            const ScatterArgs b = {a.src, a.dst, a.lds, a.ldd, a.rows / a.k, a.dim, place, a.used, a.k};
            hipLaunchKernelGGL((k_scatter<T, G, WHOLE>), dim3((unsigned)move_blocks(b.rows, G, kGatherRows)), dim3(kBlock),
                               0, s, b);
        } else {
            hipLaunchKernelGGL((k_gather<T, G, false, WHOLE>), dim3((unsigned)move_blocks(a.rows, G, kGatherRows)),
                               dim3(kBlock), 0, s, a);
        }
    });
}

template <typename T>
hipError_t sum_choices(const SumArgs& a, hipStream_t s)
{
    return with_row<T>(a.dim, [&](auto lanes, auto whole) {
        constexpr int G = decltype(lanes)::value;
        hipLaunchKernelGGL((k_sum_choices<T, G, decltype(whole)::value>), dim3((unsigned)move_blocks(a.rows, G, 1)),
                           dim3(kBlock), 0, s, a);
    });
}

template <typename T>
hipError_t combine_bwd(const CombineBwdArgs& a, hipStream_t s)
{
    return with_row<T>(a.dim, [&](auto lanes, auto whole) {
        constexpr int G = decltype(lanes)::value;
        hipLaunchKernelGGL((k_combine_bwd<T, G, decltype(whole)::value>), dim3((unsigned)move_blocks(a.rows, G, 1)),
                           dim3(kBlock), 0, s, a);
    });
}

template <typename T>
hipError_t embedding_bwd(int type, const EntriesArgs& args, hipStream_t s)
{
    EntriesArgs a = args;
    const EntriesPlan p = entries_plan(type, a.count, a.dim);
    a.per = (int32_t)p.per;
    hipError_t e = hipSuccess;
    if (a.count > 0) {
        with_lanes(p.lanes, [&](auto lanes) {
            constexpr int G = decltype(lanes)::value;
            const dim3 grid((unsigned)p.parts, (unsigned)div_up(a.dim, G * Vec<T>::N));
            if (a.dim % Vec<T>::N == 0)
                hipLaunchKernelGGL((k_sum_entries<T, G, true>), grid, dim3(kBlock), 0, s, a);
            else
                hipLaunchKernelGGL((k_sum_entries<T, G, false>), grid, dim3(kBlock), 0, s, a);
        });
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    const int64_t parts = a.count > 0 ? p.parts : 0;
    hipLaunchKernelGGL((k_join_entries<T>), dim3((unsigned)(parts + std::min(div_up(a.entries, kBlock), kZeroBlocks)),
                                                 (unsigned)div_up(a.dim, kJoinCols * 16)),
                       dim3(kBlock), 0, s, a, parts, p.span, p.lanes);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_fwd(int type, const void* table, int64_t ldt, int64_t entries, const int32_t* index,
                                float scale, int64_t rows, int64_t dim, void* y, int64_t ldy, hipStream_t s)
{
    const GatherArgs a = {table, y, ldt, ldy, rows, dim, index, nullptr, entries, 1, scale};
    if (type == GS_F16) return lookup<f16>(a, s);
    if (type == GS_BF16) return lookup<bf16>(a, s);
    return lookup<float>(a, s);
}

hipError_t launch_dispatch_fwd(int type, const void* x, int64_t ldx, const gs_row_order& o, int k, int64_t dim, void* xs,
                               int64_t ldxs, hipStream_t s)
{
    const GatherArgs a = {x, xs, ldx, ldxs, o.count, dim, o.order, o.offsets + o.groups, 0, k, 1.f};
    if (type == GS_F16) return dispatch<f16>(a, o.place, s);
    if (type == GS_BF16) return dispatch<bf16>(a, o.place, s);
    return dispatch<float>(a, o.place, s);
}

hipError_t launch_sum_choices(int type, const void* src, int64_t lds, const gs_row_order& o, const float* weight,
                              const void* add, int64_t ldadd, int64_t rows, int64_t dim, void* dst, int64_t ldd,
                              hipStream_t s)
{
    const SumArgs a = {src,   add, dst,  weight, o.place, o.offsets + o.groups, lds,
                       ldadd, ldd, rows, dim,    (int32_t)(o.count / rows)};
    if (type == GS_F16) return sum_choices<f16>(a, s);
    if (type == GS_BF16) return sum_choices<bf16>(a, s);
    return sum_choices<float>(a, s);
}

hipError_t launch_combine_bwd(int type, const void* dy, int64_t lddy, const void* ys, int64_t ldys, const gs_row_order& o,
                              const float* weight, int64_t rows, int64_t dim, void* dys, int64_t lddys, float* dweight,
                              hipStream_t s)
{
    const CombineBwdArgs a = {dy,    ys,   dys,  weight, dweight, o.place, o.offsets + o.groups, lddy, ldys,
                              lddys, rows, dim, (int32_t)(o.count / rows)};
    if (type == GS_F16) return combine_bwd<f16>(a, s);
    if (type == GS_BF16) return combine_bwd<bf16>(a, s);
    return combine_bwd<float>(a, s);
}

size_t embedding_workspace(int type, int64_t count, int64_t dim)
{
    return count > 0 ? (size_t)entries_plan(type, count, dim).parts * 2 * (size_t)dim * sizeof(float) : 0;
}

hipError_t launch_embedding_bwd(int type, const void* dy, int64_t lddy, const gs_row_order& o, float scale, int64_t dim,
                                void* dtable, int64_t lddt, int out_f32, float* part, hipStream_t s)
{
    const EntriesArgs a = {dy,       dtable,   lddy,      lddt,  dim,  o.groups, o.count,
                           o.order, o.sorted, o.offsets, scale, part, 0,        out_f32};
    if (type == GS_F16) return embedding_bwd<f16>(type, a, s);
    if (type == GS_BF16) return embedding_bwd<bf16>(type, a, s);
    return embedding_bwd<float>(type, a, s);
}

}  // namespace gsr
