// Layer norm over the rows of a matrix, forward and backward.
//
//   mu = sum x / d, var = sum (x - mu)^2 / d, rstd = 1 / sqrt(var + eps),
//   xh = (x - mu) rstd, y = xh w + b
//   g = dy w, dx = rstd (g - mean(g) - xh mean(g xh)) [+ add],
//   dw = sum over rows of dy xh, db = sum over rows of dy
//
// Bound by HBM: a row is read once and stays in registers, spread over a group
// of G lanes of which each holds NV vectors of 16 bytes; the variance is taken
// around the mean from those registers, so an offset of x does not cancel.
// Groups take rows in turn, so that the weights, and in the backward each lane's
// sums for dw and db, stay in registers over all rows of a workgroup; a
// workgroup adds up its sums in LDS and writes one partial row, and
// k_column_sum adds the partial rows in a fixed order (no atomics: the same
// call gives the same bits). All arithmetic is fp32; results are rounded to the
// element type once, as they are stored.
//
// Measured: forward of 30,000 x 1,024 in binary16 21 us, 5.9 TB/s of what it has
// to move (it partly stays in the last-level cache); backward of 16,384 x 4,096
// in bfloat16 with the skip connection's gradient 106 us and 7 for the partial
// sums, of 100,003 x 333 in fp32 79 and 5: both 5.2 TB/s in counted bytes, the
// rate of a large copy. One row is the latency of a launch, 7 us a call.
// Rows longer than a workgroup's registers are read two or three times: forward of
// 2,000 x 16,384 in fp32 106 us, backward of 2,000 x 8,192 in fp32 84, of 2,000 x
// 16,384 in bfloat16 167 (52 and 39 at the rate of a copy).
#include "gs_internal.h"
#include "vec.h"

namespace gsr {

namespace {

constexpr int kNormWaves = 4;            // waves of a workgroup whose rows lie within one wave
constexpr int kSumCols = 16;             // columns per workgroup of k_column_sum
constexpr int kSumSlices = 64;           // row slices of k_column_sum

// Parameters [c, c + N) of a row of dim; `otherwise` where there are none.
template <int N>
__device__ __forceinline__ void load_parameters(const float* p, int c, int dim, float otherwise, float* out)
{
    if (p) {
#pragma unroll
        for (int e = 0; e < N; e += 4) load_vec(p + c + e, dim - c - e, out + e);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = otherwise;
    }
}

// Sum of v over the G lanes of a row, left in all of them. G > 64: the row is the workgroup's; `slot` is LDS
// of G / 64 floats that the previous call did not use.
template <int G>
__device__ __forceinline__ float row_sum(float v, float* slot)
{
    v = lane_sum<(G < 64 ? G : 64)>(v);
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int k = 0; k < G / 64; ++k) v += slot[k];
    }
    return v;
}

template <typename T, int G, int NV>
__global__ __launch_bounds__(G > 64 ? G : kNormWaves * 64) void k_norm_fwd(
    const T* __restrict__ x, int64_t ldx, const float* __restrict__ w, const float* __restrict__ b, int64_t rows,
    int dim, float eps, T* __restrict__ y, int64_t ldy, float* __restrict__ mean, float* __restrict__ rstd)
{
    constexpr int N = Vec<T>::N;
    constexpr int kThreads = G > 64 ? G : kNormWaves * 64;
    __shared__ float slots[2][kThreads / 64];
    const int lane = threadIdx.x & (G - 1);
    const float inv = 1.f / (float)dim;
    float wv[NV][N], bv[NV][N];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_parameters<N>(w, (k * G + lane) * N, dim, 1.f, wv[k]);
        load_parameters<N>(b, (k * G + lane) * N, dim, 0.f, bv[k]);
    }
    // a row's vectors are fetched while the row before it is worked on
    const int64_t step = (int64_t)gridDim.x * (kThreads / G);
    typename Vec<T>::Packed next[NV];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + lane) * N;
            next[k] = load_any(x + r * ldx + c, dim - c);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
    if (first < rows) fetch(first);
    for (int64_t r = first; r < rows; r += step) {
        float v[NV][N];
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[k][j] = (float)next[k][j];   // 0 beyond the row
                s += v[k][j];
            }
        if (r + step < rows) fetch(r + step);
        const float mu = row_sum<G>(s, slots[0]) * inv;
        float q = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = (k * G + lane) * N + j < dim ? v[k][j] - mu : 0.f;
                v[k][j] = t;
                q += t * t;
            }
        const float rs = 1.f / sqrtf(row_sum<G>(q, slots[1]) * inv + eps);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + lane) * N;
            float o[N];
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = v[k][j] * rs * wv[k][j] + bv[k][j];
            store_vec(y + r * ldy + c, dim - c, o);
        }
        if (lane == 0) {
            if (mean) mean[r] = mu;
            if (rstd) rstd[r] = rs;
        }
    }
}

// A row longer than the registers of a workgroup: read three times, from the caches after the first.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_fwd_long(const T* __restrict__ x, int64_t ldx,
                                                        const float* __restrict__ w, const float* __restrict__ b,
                                                        int64_t rows, int dim, float eps, T* __restrict__ y,
                                                        int64_t ldy, float* __restrict__ mean,
                                                        float* __restrict__ rstd)
{
    constexpr int N = Vec<T>::N;
    __shared__ float slots[2][16];
    const float inv = 1.f / (float)dim;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* xr = x + r * ldx;
        float s = 0.f, v[N];
        for (int64_t c = (int64_t)threadIdx.x * N; c < dim; c += 1024 * N) {
            load_vec(xr + c, dim - c, v);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) t += v[j];
            s += t;
        }
        const float mu = row_sum<1024>(s, slots[0]) * inv;
        float q = 0.f;
        for (int64_t c = (int64_t)threadIdx.x * N; c < dim; c += 1024 * N) {
            load_vec(xr + c, dim - c, v, mu);
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) t += (v[j] - mu) * (v[j] - mu);
            q += t;
        }
        const float rs = 1.f / sqrtf(row_sum<1024>(q, slots[1]) * inv + eps);
        for (int64_t c = (int64_t)threadIdx.x * N; c < dim; c += 1024 * N) {
            load_vec(xr + c, dim - c, v);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool in = c + j < dim;
                v[j] = (v[j] - mu) * rs * (w && in ? w[c + j] : 1.f) + (b && in ? b[c + j] : 0.f);
            }
            store_vec(y + r * ldy + c, dim - c, v);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[r] = mu;
            if (rstd) rstd[r] = rs;
        }
    }
}

// part: [gridDim.x][2][dim] partial sums for dw, db; NULL: a single workgroup writes dw and db themselves
template <typename T, int G, int NV>
__global__ __launch_bounds__(G > 64 ? G : kNormWaves * 64) void k_norm_bwd(
    const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const float* __restrict__ w,
    const float* __restrict__ mean, const float* __restrict__ rstd, const T* __restrict__ add, int64_t ldadd,
    int64_t rows, int dim, T* __restrict__ dx, int64_t lddx, float* __restrict__ dw, float* __restrict__ db,
    float* __restrict__ part)
{
    constexpr int N = Vec<T>::N;
    constexpr int kThreads = G > 64 ? G : kNormWaves * 64;
    constexpr int kW = kThreads / 64;
    __shared__ float slots[4][kW];
    __shared__ float sums[G > 64 ? 1 : kW][G > 64 ? 1 : G * NV * N];
    const int lane = threadIdx.x & (G - 1);
    const float inv = 1.f / (float)dim;
    float wv[NV][N], sw[NV][N], sb[NV][N];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        load_parameters<N>(w, (k * G + lane) * N, dim, 1.f, wv[k]);
#pragma unroll
        for (int j = 0; j < N; ++j) sw[k][j] = sb[k][j] = 0.f;
    }
    // a row's vectors are fetched while the row before it is worked on
    const int64_t step = (int64_t)gridDim.x * (kThreads / G);
    typename Vec<T>::Packed nx[NV], ng[NV], na[NV];
    float nmu = 0.f, nrs = 0.f;
    auto fetch = [&](int64_t r) {
        nmu = mean[r];
        nrs = rstd[r];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + lane) * N;
            nx[k] = load_any(x + r * ldx + c, dim - c);
            ng[k] = load_any(dy + r * lddy + c, dim - c);
            if (add) na[k] = load_any(add + r * ldadd + c, dim - c);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
    if (first < rows) fetch(first);
    for (int64_t r = first; r < rows; r += step) {
        const float mu = nmu, rs = nrs;
        float xh[NV][N], g[NV][N];
        typename Vec<T>::Packed ar[NV];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            ar[k] = na[k];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                xh[k][j] = (float)nx[k][j];
                g[k][j] = (float)ng[k][j];   // 0 beyond the row, and with it what such a place adds
            }
        }
        if (r + step < rows) fetch(r + step);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                // (beyond the row 0 as well: the mean times rstd can be infinite where no x of the row is far from it)
                xh[k][j] = (k * G + lane) * N + j < dim ? (xh[k][j] - mu) * rs : 0.f;
                sb[k][j] += g[k][j];
                sw[k][j] += g[k][j] * xh[k][j];
                g[k][j] *= wv[k][j];
                s1 += g[k][j];
                s2 += g[k][j] * xh[k][j];
            }
        if constexpr (G > 64) {
            s1 = lane_sum<64>(s1);
            s2 = lane_sum<64>(s2);
            // two pairs of slots in turn: a wave may be a row ahead of one that still reads the last row's
            const int turn = (int)((r / gridDim.x) & 1) * 2;
            if ((threadIdx.x & 63) == 0) {
                slots[turn][threadIdx.x >> 6] = s1;
                slots[turn + 1][threadIdx.x >> 6] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int k = 0; k < kW; ++k) {
                s1 += slots[turn][k];
                s2 += slots[turn + 1][k];
            }
        } else {
            s1 = lane_sum<G>(s1);
            s2 = lane_sum<G>(s2);
        }
        s1 *= inv;
        s2 *= inv;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * G + lane) * N;
            float o[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = rs * (g[k][j] - s1 - xh[k][j] * s2);
                o[j] = add ? t + (float)ar[k][j] : t;
            }
            store_vec(dx + r * lddx + c, dim - c, o);
        }
    }
    if (!dw && !db) return;
    float* ow = part ? part + (int64_t)blockIdx.x * 2 * dim : dw;
    float* ob = part ? part + (int64_t)blockIdx.x * 2 * dim + dim : db;
    if constexpr (G > 64) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int c = (k * G + lane) * N + j;
                if (c < dim) {
                    if (ow) ow[c] = sw[k][j];
                    if (ob) ob[c] = sb[k][j];
                }
            }
    } else {
        // the groups' sums within a wave by lane exchanges, the waves' in LDS
        auto finish = [&](const float(&sum)[NV][N], float* o) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    float t = sum[k][j];
#pragma unroll
                    for (int d = G; d < 64; d <<= 1) t += __shfl_xor(t, d, 64);
                    if ((threadIdx.x & 63) < G) sums[threadIdx.x >> 6][(k * G + lane) * N + j] = t;
                }
            __syncthreads();
            if (o)
                for (int c = threadIdx.x; c < dim; c += kThreads) {
                    float t = 0.f;
#pragma unroll
                    for (int k = 0; k < kW; ++k) t += sums[k][c];
                    o[c] = t;
                }
        };
        finish(sw, ow);
        __syncthreads();   // the first sums are read
        finish(sb, ob);
    }
}

// dx of rows longer than a workgroup's registers.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_bwd_long(const T* __restrict__ dy, int64_t lddy,
                                                        const T* __restrict__ x, int64_t ldx,
                                                        const float* __restrict__ w, const float* __restrict__ mean,
                                                        const float* __restrict__ rstd, const T* __restrict__ add,
                                                        int64_t ldadd, int64_t rows, int dim, T* __restrict__ dx,
                                                        int64_t lddx)
{
    constexpr int N = Vec<T>::N;
    __shared__ float slots[2][16];
    const float inv = 1.f / (float)dim;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.f, s2 = 0.f, g[N], v[N], o[N];
        for (int64_t c = (int64_t)threadIdx.x * N; c < dim; c += 1024 * N) {
            load_vec(dy + r * lddy + c, dim - c, g);
            load_vec(x + r * ldx + c, dim - c, v, mu);
            float t1 = 0.f, t2 = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float gj = g[j] * (w && c + j < dim ? w[c + j] : 1.f);
                t1 += gj;
                t2 += gj * ((v[j] - mu) * rs);
            }
            s1 += t1;
            s2 += t2;
        }
        // both sums through one barrier each, in slots of their own
        s1 = row_sum<1024>(s1, slots[0]) * inv;
        s2 = row_sum<1024>(s2, slots[1]) * inv;
        for (int64_t c = (int64_t)threadIdx.x * N; c < dim; c += 1024 * N) {
            load_vec(dy + r * lddy + c, dim - c, g);
            load_vec(x + r * ldx + c, dim - c, v, mu);
            if (add) load_vec(add + r * ldadd + c, dim - c, o);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float gj = g[j] * (w && c + j < dim ? w[c + j] : 1.f);
                const float t = rs * (gj - s1 - (v[j] - mu) * rs * s2);
                o[j] = add ? t + o[j] : t;
            }
            store_vec(dx + r * lddx + c, dim - c, o);
        }
    }
}

// dw and db of such rows: a thread per column, workgroup (x, y) sums every gridDim.y-th row.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_norm_bwd_long_sums(const T* __restrict__ dy, int64_t lddy,
                                                               const T* __restrict__ x, int64_t ldx,
                                                               const float* __restrict__ mean,
                                                               const float* __restrict__ rstd, int64_t rows, int dim,
                                                               float* __restrict__ part)
{
    const int c = blockIdx.x * kBlock + threadIdx.x;
    if (c >= dim) return;
    float sw = 0.f, sb = 0.f;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const float g = (float)dy[r * lddy + c];
        sb += g;
        sw += g * (((float)x[r * ldx + c] - mean[r]) * rstd[r]);
    }
    part[(int64_t)blockIdx.y * 2 * dim + c] = sw;
    part[(int64_t)blockIdx.y * 2 * dim + dim + c] = sb;
}

// out[c] = sum over k of part[k][c], c in [0, cols): [0, split) to out0, the rest to out1 (either may be NULL).
__global__ __launch_bounds__(kSumCols* kSumSlices) void k_column_sum(const float* __restrict__ part, int count,
                                                                     int64_t cols, int64_t split,
                                                                     float* __restrict__ out0,
                                                                     float* __restrict__ out1)
{
    __shared__ float s[kSumSlices][kSumCols];
    const int col = threadIdx.x % kSumCols, slice = threadIdx.x / kSumCols;
    const int64_t c = (int64_t)blockIdx.x * kSumCols + col;
    float t = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int k = slice; k < count; k += kSumSlices) t += part[(int64_t)k * cols + c];
    s[slice][col] = t;
    __syncthreads();
    if (slice != 0 || c >= cols) return;
    t = 0.f;
#pragma unroll
    for (int k = 0; k < kSumSlices; ++k) t += s[k][col];
    float* o = c < split ? out0 : out1;
    if (o) o[c < split ? c : c - split] = t;
}

// Lanes and vectors of a row: the fewest lanes (a power of two up to a wave, then 4 or 16 waves) that hold it
// with as few vectors each as possible. A wave holds 2 or 3 vectors a lane before a row goes to a workgroup: its sums
// then need no barrier, and fewer lanes are idle. Against workgroups of one vector a lane from 65 vectors on: forward of
// 30,000 x 1,024 in binary16 21 us for 31, of 100,003 x 333 in fp32 56 for 89; backward 47 for 58 and 85 for 133, of
// 20,000 x 1,500 in bfloat16 61 for 87 (of 20,003 x 700 in fp32 42 for 37).
struct RowShape {
    int g, nv;   // g = 0: longer than a workgroup holds
};

RowShape row_shape(int type, int64_t dim, bool backward)
{
    const int64_t n = type == GS_F32 ? 4 : 8;
    const int64_t vecs = div_up(dim, n);
    for (int g = 1; g <= 64; g <<= 1)
        if (vecs <= g) return {g, 1};
    if (vecs <= 128) return {64, 2};
    for (int g = 64; g <= 512; g <<= 1) {
        if (vecs <= 3 * g && g <= 256) return {g, 3};
        if (vecs <= 4 * g && g <= 256) return {4 * g, 1};
    }
    // (the backward of 16-bit rows that long would need more than a 1,024-thread workgroup's 128 registers)
    if (vecs <= 2048 && !backward) return {1024, 2};
    return {0, 0};
}

// Partial rows of the backward's sums: up to 4 workgroups of 256 threads per compute unit (one of 1,024), fewer
// where the partial rows' bytes would be more than about a sixteenth of the matrices'.
constexpr int kNormParts = 1024;

int norm_bwd_blocks(int type, int64_t rows, int64_t dim)
{
    const RowShape sh = row_shape(type, dim, true);
    if (sh.g == 0) return (int)std::min<int64_t>(std::max<int64_t>(rows / 64, 1), 64);
    const int64_t per = sh.g > 64 ? 1 : kNormWaves * 64 / sh.g;
    const int64_t most = sh.g > 256 ? 256 * 1024 / sh.g : kNormParts;
    return (int)std::max<int64_t>(1, std::min(most, div_up(rows, per * 4)));
}

template <typename T, int G, int NV>
void norm_fwd(const void* x, int64_t ldx, const float* w, const float* b, int64_t rows, int dim, float eps, void* y,
              int64_t ldy, float* mean, float* rstd, hipStream_t s)
{
    constexpr int kThreads = G > 64 ? G : kNormWaves * 64;
    // (every group takes a few rows where there are enough: its parameters are loaded once)
    const int64_t blocks = std::min<int64_t>(div_up(rows, kThreads / G), 256 * (NV == 1 ? 2048 : 1024) / kThreads);
    hipLaunchKernelGGL((k_norm_fwd<T, G, NV>), dim3((unsigned)blocks), dim3(kThreads), 0, s, (const T*)x, ldx, w, b,
                       rows, dim, eps, (T*)y, ldy, mean, rstd);
}

template <typename T, int G, int NV>
void norm_bwd(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* w, const float* mean,
              const float* rstd, const void* add, int64_t ldadd, int64_t rows, int dim, void* dx, int64_t lddx,
              float* dw, float* db, float* part, int blocks, hipStream_t s)
{
    constexpr int kThreads = G > 64 ? G : kNormWaves * 64;
    hipLaunchKernelGGL((k_norm_bwd<T, G, NV>), dim3((unsigned)blocks), dim3(kThreads), 0, s, (const T*)dy, lddy,
                       (const T*)x, ldx, w, mean, rstd, (const T*)add, ldadd, rows, dim, (T*)dx, lddx, dw, db, part);
}

#define GS_NORM_SHAPES(call)                        \
    switch (sh.g * 8 + sh.nv) {                     \
    case 1 * 8 + 1: call(1, 1); break;              \
    case 2 * 8 + 1: call(2, 1); break;              \
    case 4 * 8 + 1: call(4, 1); break;              \
    case 8 * 8 + 1: call(8, 1); break;              \
    case 16 * 8 + 1: call(16, 1); break;            \
    case 32 * 8 + 1: call(32, 1); break;            \
    case 64 * 8 + 1: call(64, 1); break;            \
    case 64 * 8 + 2: call(64, 2); break;            \
    case 64 * 8 + 3: call(64, 3); break;            \
    case 128 * 8 + 3: call(128, 3); break;          \
    case 256 * 8 + 3: call(256, 3); break;          \
    case 256 * 8 + 1: call(256, 1); break;          \
    case 512 * 8 + 1: call(512, 1); break;          \
    case 1024 * 8 + 1: call(1024, 1); break;

template <typename T>
hipError_t norm_fwd_type(int type, const void* x, int64_t ldx, const float* w, const float* b, int64_t rows, int dim,
                         float eps, void* y, int64_t ldy, float* mean, float* rstd, hipStream_t s)
{
    const RowShape sh = row_shape(type, dim, false);
#define CALL(G, NV) norm_fwd<T, G, NV>(x, ldx, w, b, rows, dim, eps, y, ldy, mean, rstd, s)
    GS_NORM_SHAPES(CALL)
    case 1024 * 8 + 2: CALL(1024, 2); break;
    default:
        hipLaunchKernelGGL((k_norm_fwd_long<T>), dim3((unsigned)std::min<int64_t>(rows, 512)), dim3(1024), 0, s,
                           (const T*)x, ldx, w, b, rows, dim, eps, (T*)y, ldy, mean, rstd);
    }
#undef CALL
    return hipGetLastError();
}

template <typename T>
hipError_t norm_bwd_type(int type, const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* w,
                         const float* mean, const float* rstd, const void* add, int64_t ldadd, int64_t rows, int dim,
                         void* dx, int64_t lddx, float* dw, float* db, float* part, hipStream_t s)
{
    const RowShape sh = row_shape(type, dim, true);
    const int blocks = norm_bwd_blocks(type, rows, dim);
    float* p = blocks == 1 && sh.g ? nullptr : part;
#define CALL(G, NV) \
    norm_bwd<T, G, NV>(dy, lddy, x, ldx, w, mean, rstd, add, ldadd, rows, dim, dx, lddx, dw, db, p, blocks, s)
    GS_NORM_SHAPES(CALL)
    default:
        if (rows > 0)
            hipLaunchKernelGGL((k_norm_bwd_long<T>), dim3((unsigned)std::min<int64_t>(rows, 512)), dim3(1024), 0, s,
                               (const T*)dy, lddy, (const T*)x, ldx, w, mean, rstd, (const T*)add, ldadd, rows, dim,
                               (T*)dx, lddx);
        if (dw || db)
            hipLaunchKernelGGL((k_norm_bwd_long_sums<T>), dim3((unsigned)div_up(dim, kBlock), (unsigned)blocks),
                               dim3(kBlock), 0, s, (const T*)dy, lddy, (const T*)x, ldx, mean, rstd, rows, dim, p);
    }
#undef CALL
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p || !(dw || db)) return e;
    return launch_column_sum(p, blocks, 2 * (int64_t)dim, dim, dw, db, s);
}

}  // namespace

hipError_t launch_column_sum(const float* part, int count, int64_t cols, int64_t split, float* out0, float* out1,
                             hipStream_t s)
{
    hipLaunchKernelGGL(k_column_sum, dim3((unsigned)div_up(cols, kSumCols)), dim3(kSumCols * kSumSlices), 0, s, part,
                       count, cols, split, out0, out1);
    return hipGetLastError();
}

size_t layer_norm_workspace(int type, int64_t rows, int64_t dim)
{
    return (size_t)norm_bwd_blocks(type, rows, dim) * 2 * (size_t)dim * sizeof(float);
}

hipError_t launch_layer_norm_fwd(int type, const void* x, int64_t ldx, const float* w, const float* b, int64_t rows,
                                 int dim, float eps, void* y, int64_t ldy, float* mean, float* rstd, hipStream_t s)
{
    if (type == GS_F16) return norm_fwd_type<f16>(type, x, ldx, w, b, rows, dim, eps, y, ldy, mean, rstd, s);
    if (type == GS_BF16) return norm_fwd_type<bf16>(type, x, ldx, w, b, rows, dim, eps, y, ldy, mean, rstd, s);
    return norm_fwd_type<float>(type, x, ldx, w, b, rows, dim, eps, y, ldy, mean, rstd, s);
}

hipError_t launch_layer_norm_bwd(int type, const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* w,
                                 const float* mean, const float* rstd, const void* add, int64_t ldadd, int64_t rows,
                                 int dim, void* dx, int64_t lddx, float* dw, float* db, float* part, hipStream_t s)
{
#define CALL(T) norm_bwd_type<T>(type, dy, lddy, x, ldx, w, mean, rstd, add, ldadd, rows, dim, dx, lddx, dw, db, part, s)
    if (type == GS_F16) return CALL(f16);
    if (type == GS_BF16) return CALL(bf16);
    return CALL(float);
#undef CALL
}

}  // namespace gsr
