// Matrix product on the matrix cores with the linear operators' epilogue, one
// template for binary16, bfloat16 (16x16x32 MFMA) and fp32 (16x16x4 MFMA).
//
// A workgroup computes a BI x BJ tile of C with WI x WJ waves; the operands'
// tiles (128 bytes along the sum: 64 16-bit or 32 fp32 values) go from memory to
// LDS with buffer loads that write LDS directly, double-buffered, one barrier
// per step: the next tile's loads run under the current one's MFMAs. Out of
// range rows come out of the buffer descriptor's range check as zeros.
//
// LDS slots are 16 bytes. Reading a fragment takes one slot from each of 16
// rows (NT), or four 4-value pieces of rows through the transposing LDS read
// (TT, 16-bit); slots are XOR-ed with a hash of the row so that the rows fall in
// different banks. As LDS is written in slot order, the permutation is applied
// to the addresses that the lanes load from.
//
// In NT a fragment's 16 columns j are not neighbours: the columns of fragments
// f, f + 1 interleave in fours, so that a lane ends up with 8 neighbouring
// columns of one row and the epilogue moves whole 16-byte vectors.
#pragma once

#include "activation.h"
#include "linear.h"

namespace gsr {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr uint32_t kOutOfRange = 0x80000000u;   // beyond any descriptor's range (at most 2^31 - 1 bytes)

template <typename T>
struct Mma {
    typedef T Frag __attribute__((ext_vector_type(8)));   // 16-bit: 8 values along the sum
    static constexpr int kBK = 64;                        // values along the sum per tile
    static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c)
    {
        if constexpr (__is_same(T, f16))
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

template <>
struct Mma<float> {
    typedef float Frag __attribute__((ext_vector_type(4)));
    static constexpr int kBK = 32;
    static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// ---- operand tiles ----------------------------------------------------------

// NT: X rows of 8 slots along the sum. Fragment rows are base + l%16 (A) or the interleaved columns (B).
__device__ __forceinline__ int nt_hash_a(int row) { return row & 7; }
__device__ __forceinline__ int nt_hash_b(int row) { return (row & 3) | ((row >> 1) & 4); }

// TT: kBK rows c of X * sizeof(T) / 16 slots.
template <typename T, int X>
__device__ __forceinline__ int tt_hash(int c)
{
    constexpr int kSlots = X * (int)sizeof(T) / 16;
    if constexpr (sizeof(T) == 2) {
        // the 32 lanes of half a wave read 32 bytes of each of 8 rows
        const int h = (c & 3) | ((c >> 1) & 4);
        return (h << 1) & (kSlots - 1);
    } else {
        return ((c & 3) << 2) & (kSlots - 1);   // 64 bytes of each of 4 rows
    }
}

// Geometry of one operand's tile: which slot of which row a thread fills, and from which vector of that row.
template <typename T, int X, bool TT, bool IS_B, int THREADS>
struct Tile {
    static constexpr int kBK = Mma<T>::kBK;
    static constexpr int kVec = 16 / (int)sizeof(T);
    static constexpr int kRowSlots = TT ? X / kVec : 8;
    static constexpr int kSlotsTotal = X * 8;             // X * 128 bytes
    static constexpr int kPasses = kSlotsTotal / THREADS;
    static constexpr int kBytes = X * 128;
    static_assert(kSlotsTotal % THREADS == 0, "whole passes");

    static __device__ __forceinline__ int row(int q) { return q / kRowSlots; }
    static __device__ __forceinline__ int vec(int q)
    {
        const int r = row(q), s = q % kRowSlots;
        return TT ? s ^ tt_hash<T, X>(r) : s ^ (IS_B ? nt_hash_b(r) : nt_hash_a(r));
    }

    // LDS <- memory. p: the operand, stored rows of ld values; x0: first row (NT) or column (TT) of the tile;
    // c0: position along the sum; c_end, x_end: where both end.
    static __device__ __forceinline__ void load_async(char* lds, const T* p, int64_t ld, int64_t stored, int64_t x0,
                                                      int64_t x_end, int64_t c0, int64_t c_end)
    {
        const int64_t r0 = TT ? c0 : x0;
        const int64_t rows_end = TT ? c_end : x_end;
        const int64_t first = r0 * ld;
        // bytes from the tile's first row to the end of its last valid one
        const int64_t bytes = ((rows_end < stored ? rows_end : stored) - r0) * ld * (int64_t)sizeof(T);
        const int range = bytes > 0x7FFFFFF0 ? 0x7FFFFFF0 : (int)bytes;
        __amdgpu_buffer_rsrc_t rsrc =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p + first), 0, range, 0x00027000);
        const int64_t v0 = TT ? x0 : c0, v_end = TT ? x_end : c_end;
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int q = k * THREADS + threadIdx.x;
            const int64_t v = v0 + (int64_t)vec(q) * kVec;
            // (vectors are whole in this form: v < v_end covers all of one)
            uint32_t off = (uint32_t)row(q) * (uint32_t)(ld * (int64_t)sizeof(T)) + (uint32_t)(v * (int64_t)sizeof(T));
            if (v >= v_end) off = kOutOfRange;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(lds + (k * (THREADS / 64) + wave) * 1024), 16,
                                                     off, 0, 0, 0);
        }
    }

    // registers <- memory at any alignment, masked value by value at the ends
    typedef typename Vec<T>::Packed Packed;
    static __device__ __forceinline__ void load_regs(Packed (&r)[kPasses], const T* p, int64_t ld, int64_t x0,
                                                     int64_t x_end, int64_t c0, int64_t c_end)
    {
        const int64_t r0 = TT ? c0 : x0, rows_end = TT ? c_end : x_end;
        const int64_t v0 = TT ? x0 : c0, v_end = TT ? x_end : c_end;
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int q = k * THREADS + threadIdx.x;
            const int64_t rr = r0 + row(q), v = v0 + (int64_t)vec(q) * kVec;
            Packed t = {};
            if (rr < rows_end) {
                const T* src = p + rr * ld + v;
                if (v + kVec <= v_end)
                    t = *reinterpret_cast<const typename Vec<T>::Any*>(src);
                else
#pragma unroll
                    for (int j = 0; j < kVec; ++j)
                        if (v + j < v_end) t[j] = src[j];
            }
            r[k] = t;
        }
    }
    static __device__ __forceinline__ void store_regs(char* lds, const Packed (&r)[kPasses])
    {
#pragma unroll
        for (int k = 0; k < kPasses; ++k) *reinterpret_cast<Packed*>(lds + (k * THREADS + threadIdx.x) * 16) = r[k];
    }

    // Fragment for values [32 s, 32 s + 32) (16-bit) or [16 s, ...) (fp32) of the sum. f: fragment of the wave's
    // `wx` first row or column.
    static __device__ __forceinline__ typename Mma<T>::Frag frag(const char* lds, int wx, int f, int s)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
        if constexpr (!TT) {
            const int r = IS_B ? wx + 32 * (f >> 1) + 4 * (f & 1) + 8 * (i >> 2) + (i & 3) : wx + 16 * f + i;
            const int slot = (4 * s + g) ^ (IS_B ? nt_hash_b(r) : nt_hash_a(r));
            return *reinterpret_cast<const typename Mma<T>::Frag*>(lds + r * 128 + slot * 16);
        } else if constexpr (sizeof(T) == 2) {
            typename Mma<T>::Frag out;
            s16x4 h[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int c = 32 * s + 8 * g + 4 * t + (i >> 2);
                const int col = wx + 16 * f + 4 * (i & 3);
                const int slot = (col / 8) ^ tt_hash<T, X>(c);
                h[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4*)(lds + c * (X * 2) + slot * 16 + (col & 7) * 2));
            }
            __builtin_memcpy(&out, h, 16);
            return out;
        } else {
            typename Mma<T>::Frag out;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = 16 * s + 4 * e + g;
                const int col = wx + 16 * f + i;
                const int slot = (col / 4) ^ tt_hash<T, X>(c);
                out[e] = *reinterpret_cast<const float*>(lds + c * (X * 4) + slot * 16 + (col & 3) * 4);
            }
            return out;
        }
    }
};

// Tiles in an order in which neighbours in time on one XCD (workgroups b, b + 8, ...) share operand rows: each
// XCD takes a contiguous range of tiles, columns fastest within panels of kPanel tile rows.
__device__ __forceinline__ void tile_of(int64_t b, int64_t tiles_i, int64_t tiles_j, int64_t* ti, int64_t* tj)
{
    const int64_t total = tiles_i * tiles_j;
    const int64_t per = total >> 3, rest = total & 7, xcd = b & 7, k = b >> 3;
    int64_t t = xcd * per + (xcd < rest ? xcd : rest) + k;
    constexpr int64_t kPanel = 8;
    const int64_t panel = t / (kPanel * tiles_j), in = t - panel * kPanel * tiles_j;
    const int64_t left = tiles_i - panel * kPanel, h = left < kPanel ? left : kPanel;
    *ti = panel * kPanel + in % h;
    *tj = in / h;
}

// 8 neighbouring values of row i, columns [j, j + 8) of which `left` exist.
template <typename T>
__device__ __forceinline__ void epilogue8(const GemmArgs& g, int64_t i, int64_t j, int64_t left, float* v,
                                          const float* bias)
{
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += bias[e];
    if (g.z) {
        T* z = (T*)g.z + i * g.ldz + j;
#pragma unroll
        for (int e = 0; e < 8; e += N) store_vec(z + e, left - e, v + e);
    }
    activate<8>(g.act, v);
    if (g.residual) {
        const T* r = (const T*)g.residual + i * g.ldr + j;
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; e += N) load_vec(r + e, left - e, t + e);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += t[e];
    }
    if (g.out_f32) {
        float* o = (float*)g.out + i * g.ldo + j;
        store_vec(o, left, v);
        store_vec(o + 4, left - 4, v + 4);
    } else {
        T* o = (T*)g.out + i * g.ldo + j;
#pragma unroll
        for (int e = 0; e < 8; e += N) store_vec(o + e, left - e, v + e);
    }
}

// FAST: the operand that may be the caller's (A in NT, B in TT) is loaded asynchronously as well; the other
// always is.
template <typename T, bool TT, int BI, int BJ, int WI, int WJ, bool FAST>
__global__ __launch_bounds__(WI* WJ * 64) void k_gemm(GemmArgs g)
{
    constexpr int THREADS = WI * WJ * 64;
    constexpr int FI = BI / WI / 16, FJ = BJ / WJ / 16;
    constexpr int kBK = Mma<T>::kBK;
    using TA = Tile<T, BI, TT, false, THREADS>;
    using TB = Tile<T, BJ, TT, true, THREADS>;
    constexpr bool kAsyncA = FAST || TT, kAsyncB = FAST || !TT;
    static_assert(TT || FJ % 2 == 0, "columns interleave between pairs of fragments");
    __shared__ __attribute__((aligned(1024))) char lds[2][TA::kBytes + TB::kBytes];

    const int64_t tiles_i = (g.rows + BI - 1) / BI, tiles_j = (g.cols + BJ - 1) / BJ;
    int64_t ti, tj;
    tile_of(blockIdx.x, tiles_i, tiles_j, &ti, &tj);
    const int64_t i0 = ti * BI, j0 = tj * BJ;
    const int part = blockIdx.y, plane = part / g.splits, split = part - plane * g.splits;
    const int64_t c_begin = split * g.split_len;
    const int64_t c_end = c_begin + g.split_len < g.len ? c_begin + g.split_len : g.len;
    const T* a = (const T*)g.a + plane * g.plane_stride;
    const T* b = (const T*)g.b;
    const int wave = threadIdx.x >> 6, wi = (wave / WJ) * (BI / WI), wj = (wave % WJ) * (BJ / WJ);
    const int lane = threadIdx.x & 63, lg = lane >> 4, li = lane & 15;

    f32x4 acc[FI][FJ] = {};
    typename TA::Packed ra[kAsyncA ? 1 : TA::kPasses];
    typename TB::Packed rb[kAsyncB ? 1 : TB::kPasses];
    auto fetch = [&](char* to, int64_t c0) {
        if constexpr (kAsyncA)
            TA::load_async(to, a, g.lda, g.a_rows, i0, g.rows, c0, c_end);
        else
            TA::load_regs(ra, a, g.lda, i0, g.rows, c0, c_end);
        if constexpr (kAsyncB)
            TB::load_async(to + TA::kBytes, b, g.ldb, g.b_rows, j0, g.cols, c0, c_end);
        else
            TB::load_regs(rb, b, g.ldb, j0, g.cols, c0, c_end);
    };
    auto settle = [&](char* to) {
        if constexpr (!kAsyncA) TA::store_regs(to, ra);
        if constexpr (!kAsyncB) TB::store_regs(to + TA::kBytes, rb);
    };
    const int steps = c_end > c_begin ? (int)((c_end - c_begin + kBK - 1) / kBK) : 0;
    if (steps > 0) {
        fetch(lds[0], c_begin);
        settle(lds[0]);
    }
    for (int t = 0; t < steps; ++t) {
        char* cur = lds[t & 1];
        char* nxt = lds[(t + 1) & 1];
        __syncthreads();   // cur has arrived, and nxt is no longer read
        if (t + 1 < steps) fetch(nxt, c_begin + (int64_t)(t + 1) * kBK);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            typename Mma<T>::Frag fa[FI], fb[FJ];
#pragma unroll
            for (int f = 0; f < FI; ++f) fa[f] = TA::frag(cur, wi, f, s);
#pragma unroll
            for (int f = 0; f < FJ; ++f) fb[f] = TB::frag(cur + TA::kBytes, wj, f, s);
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int q = 0; q < FJ; ++q) acc[p][q] = Mma<T>::mma(fb[q], fa[p], acc[p][q]);
        }
        if (t + 1 < steps) settle(nxt);
    }

    // acc[p][q][r] is row i0 + wi + 16 p + li, column (TT) wj + 16 q + 4 lg + r or (NT) the interleaved one
    if constexpr (TT) {
        float* out = g.part ? g.part + (int64_t)part * g.rows * g.cols : nullptr;
#pragma unroll
        for (int p = 0; p < FI; ++p)
#pragma unroll
            for (int q = 0; q < FJ; ++q) {
                const int64_t i = i0 + wi + 16 * p + li, j = j0 + wj + 16 * q + 4 * lg;
                if (i >= g.rows || j >= g.cols) continue;
                float v[4] = {acc[p][q][0], acc[p][q][1], acc[p][q][2], acc[p][q][3]};
                if (out || g.out_f32) {
                    float* o = out ? out + i * g.cols + j : (float*)g.out + i * g.ldo + j;
                    store_vec(o, g.cols - j, v);
                } else {
                    T* o = (T*)g.out + i * g.ldo + j;
                    if (sizeof(T) == 2 && j + 4 <= g.cols) {
                        typedef T V4 __attribute__((ext_vector_type(4)));
                        typedef V4 V4any __attribute__((aligned(sizeof(T))));
                        V4 t;
#pragma unroll
                        for (int r = 0; r < 4; ++r) t[r] = (T)v[r];
                        *reinterpret_cast<V4any*>(o) = t;
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (j + r < g.cols) o[r] = (T)v[r];
                    }
                }
            }
    } else {
#pragma unroll
        for (int q = 0; q < FJ; q += 2) {
            const int64_t j = j0 + wj + 16 * q + 8 * lg;
            if (j >= g.cols) continue;
            float bias[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) bias[e] = g.bias && !g.part && j + e < g.cols ? g.bias[j + e] : 0.f;
#pragma unroll
            for (int p = 0; p < FI; ++p) {
                const int64_t i = i0 + wi + 16 * p + li;
                if (i >= g.rows) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = acc[p][q][e];
                    v[4 + e] = acc[p][q + 1][e];
                }
                if (g.part) {
                    float* o = g.part + ((int64_t)part * g.rows + i) * g.cols + j;
                    store_vec(o, g.cols - j, v);
                    store_vec(o + 4, g.cols - j - 4, v + 4);
                } else {
                    epilogue8<T>(g, i, j, g.cols - j, v, bias);
                }
            }
        }
    }
}

// Few rows (NT, rows <= 16 MF): a workgroup takes 16 columns j and its waves share the sum; the weights go from
// memory to registers once, 16 bytes per lane and load, and the waves' sums meet in LDS. Bound by reading the
// weights.
constexpr int kSkinnyWaves = 8;

template <typename T, int MF>
__global__ __launch_bounds__(kSkinnyWaves * 64) void k_skinny(GemmArgs g)
{
    constexpr int N = Vec<T>::N;
    constexpr int kStep = 4 * N;                     // values of the sum per MFMA step
    constexpr int kUnroll = 4;
    __shared__ float sums[kSkinnyWaves][MF][16][17];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lg = lane >> 4, li = lane & 15;
    const int64_t j0 = (int64_t)blockIdx.x * 16, i0 = (int64_t)blockIdx.y * (16 * MF);
    const T* w = (const T*)g.b + (j0 + li < g.cols ? j0 + li : g.cols - 1) * g.ldb;
    const T* x[MF];
#pragma unroll
    for (int m = 0; m < MF; ++m) {
        const int64_t i = i0 + 16 * m + li;
        x[m] = (const T*)g.a + (i < g.rows ? i : g.rows - 1) * g.lda;
    }
    f32x4 acc[MF] = {};
    const int64_t steps = (g.len + kStep - 1) / kStep;
    const int64_t per = (steps + kSkinnyWaves - 1) / kSkinnyWaves;
    const int64_t s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    for (int64_t s = s0; s < s1; s += kUnroll) {
        typename Vec<T>::Packed wv[kUnroll], xv[kUnroll][MF];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = (s + u) * kStep + lg * N;
            const int64_t left = s + u < s1 ? g.len - c : 0;
            wv[u] = load_any(w + c, left);
#pragma unroll
            for (int m = 0; m < MF; ++m) xv[u][m] = load_any(x[m] + c, left);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int m = 0; m < MF; ++m) acc[m] = Mma<T>::mma(wv[u], xv[u][m], acc[m]);
    }
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][m][li][4 * lg + r] = acc[m][r];
    __syncthreads();
    for (int k = threadIdx.x; k < MF * 256; k += kSkinnyWaves * 64) {
        const int m = k >> 8, ii = (k >> 4) & 15, jj = k & 15;
        const int64_t i = i0 + 16 * m + ii, j = j0 + jj;
        if (i >= g.rows || j >= g.cols) continue;
        float v = g.bias ? g.bias[j] : 0.f;
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < kSkinnyWaves; ++q) t += sums[q][m][ii][jj];
        v += t;
        if (g.z) ((T*)g.z)[i * g.ldz + j] = (T)v;
        activate<1>(g.act, &v);
        if (g.residual) v += (float)((const T*)g.residual)[i * g.ldr + j];
        ((T*)g.out)[i * g.ldo + j] = (T)v;
    }
}

// Adds up the parts of a split product in a fixed order and applies the epilogue. A workgroup takes 4 values each of
// kBlock / slices places; `slices` threads share a place's parts and meet in LDS.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join(GemmArgs g, float plane_scale, int slices)
{
    __shared__ f32x4 sums[kBlock];
    const int64_t quads = (g.cols + 3) / 4, total = g.rows * quads;
    const int64_t size = g.rows * g.cols;
    const int places = kBlock / slices, place = threadIdx.x % places, slice = threadIdx.x / places;
    const int64_t k = (int64_t)blockIdx.x * places + place;
    const int64_t i = k / quads, j = (k - i * quads) * 4, left = g.cols - j;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (k < total)
        for (int p = g.planes - 1; p >= 0; --p) {
            const float* part = g.part + (int64_t)p * g.splits * size + i * g.cols + j;
            f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (int s = slice; s < g.splits; s += slices) {
                float u[4];
                load_vec(part + (int64_t)s * size, left, u);
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] += u[e];
            }
            v = v * plane_scale + t;
        }
    if (slices > 1) {
        sums[threadIdx.x] = v;
        __syncthreads();
        if (slice == 0)
            for (int q = 1; q < slices; ++q) v += sums[q * places + place];
    }
    if (slice != 0 || k >= total) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= left) break;
        float t = v[e] + (g.bias ? g.bias[j + e] : 0.f);
        if (g.z) ((T*)g.z)[i * g.ldz + j + e] = (T)t;
        activate<1>(g.act, &t);
        if (g.residual) t += (float)((const T*)g.residual)[i * g.ldr + j + e];
        if (g.out_f32)
            ((float*)g.out)[i * g.ldo + j + e] = t;
        else
            ((T*)g.out)[i * g.ldo + j + e] = (T)t;
    }
}

// A thread takes a vector of columns and every gridDim.y * rows-per-workgroup'th row.
constexpr float kBf16Plane = 1.f / 256.f, kF16Plane = 1.f / 2048.f;

template <typename T>
__global__ __launch_bounds__(kBlock) void k_slope(SlopeArgs p, int lanes)
{
    constexpr int N = Vec<T>::N;
    __shared__ float s[kBlock][N + 1];
    const int lane = threadIdx.x % lanes, slice = threadIdx.x / lanes, slices = kBlock / lanes;
    const int64_t c = ((int64_t)blockIdx.x * lanes + lane) * N;
    const int64_t left = p.cols - c;
    float sum[N] = {};
    if (c < p.ldo || left > 0)
        for (int64_t r = (int64_t)blockIdx.y * slices + slice; r < p.rows; r += (int64_t)gridDim.y * slices) {
            float v[N], z[N];
            load_vec((const T*)p.dy + r * p.lddy + c, left, v);
            if (p.act != GS_ACT_NONE) {
                load_vec((const T*)p.z + r * p.ldz + c, left, z);
                times_slope<N>(p.act, v, z);
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = j < left ? v[j] : 0.f;
            }
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += v[j];
            if (p.out && c < p.ldo) {
                T* o = (T*)p.out + r * p.ldo + c;
                for (int k = 0; k < p.planes; ++k) {
                    store_vec(o + k * p.plane_stride, N, v);
                    if constexpr (sizeof(T) == 2) {
                        constexpr float kUp = __is_same(T, f16) ? 1.f / kF16Plane : 1.f / kBf16Plane;
#pragma unroll
                        for (int j = 0; j < N; ++j) {
                            // what the plane leaves; an infinite or undefined value is the first plane's alone
                            const float left_over = v[j] - (float)(T)v[j];
                            v[j] = fabsf(left_over) < __builtin_inff() ? left_over * kUp : 0.f;
                        }
                    }
                }
            }
        }
    if (!p.sums) return;
#pragma unroll
    for (int j = 0; j < N; ++j) s[threadIdx.x][j] = sum[j];
    __syncthreads();
    for (int k = threadIdx.x; k < lanes * N; k += kBlock) {
        const int64_t col = (int64_t)blockIdx.x * lanes * N + k;
        if (col >= p.cols) continue;
        float t = 0.f;
        for (int q = 0; q < slices; ++q) t += s[q * lanes + k / N][k % N];
        p.sums[(int64_t)blockIdx.y * p.cols + col] = t;
    }
}

// 64 x 64 tiles through LDS, whole 16-byte vectors in and out. dst: aligned rows of ldd values, a multiple of a
// vector, all written (padding: zero).
constexpr int kLayoutTile = 64;

template <typename T>
__global__ __launch_bounds__(kBlock) void k_layout(const T* __restrict__ src, int64_t lds, int64_t rows, int64_t cols,
                                                   int transpose, T* __restrict__ dst, int64_t ldd)
{
    constexpr int N = Vec<T>::N, kRowVecs = kLayoutTile / N;
    __shared__ T t[kLayoutTile][kLayoutTile + 4 / sizeof(T)];
    const int64_t r0 = (int64_t)blockIdx.y * kLayoutTile, c0 = (int64_t)blockIdx.x * kLayoutTile;
#pragma unroll
    for (int q = threadIdx.x; q < kLayoutTile * kRowVecs; q += kBlock) {
        const int r = q / kRowVecs, c = q % kRowVecs * N;
        const typename Vec<T>::Packed v = load_any(src + (r0 + r) * lds + c0 + c, r0 + r < rows ? cols - c0 - c : 0);
        if (!transpose) {
            if (r0 + r < rows && c0 + c < ldd)
                *reinterpret_cast<typename Vec<T>::Packed*>(dst + (r0 + r) * ldd + c0 + c) = v;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) t[r][c + e] = v[e];
        }
    }
    if (!transpose) return;
    __syncthreads();
#pragma unroll
    for (int q = threadIdx.x; q < kLayoutTile * kRowVecs; q += kBlock) {
        // neighbouring lanes take neighbouring columns of the tile: LDS reads without conflicts
        const int r = q % kLayoutTile, c = q / kLayoutTile * N;
        if (c0 + r >= cols || r0 + c >= ldd) continue;
        typename Vec<T>::Packed v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = t[c + e][r];
        *reinterpret_cast<typename Vec<T>::Packed*>(dst + (c0 + r) * ldd + r0 + c) = v;
    }
}

template <typename T, bool TT, int BI, int BJ, int WI, int WJ, bool FAST>
hipError_t run_gemm(const GemmArgs& g, hipStream_t s)
{
    const int64_t tiles = div_up(g.rows, BI) * div_up(g.cols, BJ);
    hipLaunchKernelGGL((k_gemm<T, TT, BI, BJ, WI, WJ, FAST>), dim3((unsigned)tiles, (unsigned)(g.planes * g.splits)),
                       dim3(WI * WJ * 64), 0, s, g);
    return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t LinearOps<T>::gemm_nt(int tile, bool fast_a, const GemmArgs& g, hipStream_t s)
{
    if (tile == kTile256) return run_gemm<T, false, 256, 256, 2, 4, true>(g, s);   // fast_a only
    if (tile == kTile128)
        return fast_a ? run_gemm<T, false, 128, 128, 2, 2, true>(g, s) : run_gemm<T, false, 128, 128, 2, 2, false>(g, s);
    if (tile == kTile128x32)
        return fast_a ? run_gemm<T, false, 128, 32, 4, 1, true>(g, s) : run_gemm<T, false, 128, 32, 4, 1, false>(g, s);
    return fast_a ? run_gemm<T, false, 64, 64, 2, 2, true>(g, s) : run_gemm<T, false, 64, 64, 2, 2, false>(g, s);
}

template <typename T>
hipError_t LinearOps<T>::gemm_tt(int tile, bool fast_b, const GemmArgs& g, hipStream_t s)
{
    if (tile == kTile256) return run_gemm<T, true, 256, 256, 2, 4, true>(g, s);   // fast_b only
    if (tile == kTile128)
        return fast_b ? run_gemm<T, true, 128, 128, 2, 2, true>(g, s) : run_gemm<T, true, 128, 128, 2, 2, false>(g, s);
    return fast_b ? run_gemm<T, true, 64, 64, 2, 2, true>(g, s) : run_gemm<T, true, 64, 64, 2, 2, false>(g, s);
}

template <typename T>
hipError_t LinearOps<T>::skinny(const GemmArgs& g, hipStream_t s)
{
    const unsigned x = (unsigned)div_up(g.cols, 16);
    if (g.rows <= 16)
        hipLaunchKernelGGL((k_skinny<T, 1>), dim3(x, 1), dim3(kSkinnyWaves * 64), 0, s, g);
    else if (g.rows <= 32)
        hipLaunchKernelGGL((k_skinny<T, 2>), dim3(x, 1), dim3(kSkinnyWaves * 64), 0, s, g);
    else
        hipLaunchKernelGGL((k_skinny<T, 4>), dim3(x, (unsigned)div_up(g.rows, 64)), dim3(kSkinnyWaves * 64), 0, s, g);
    return hipGetLastError();
}

template <typename T>
hipError_t LinearOps<T>::slope(const SlopeArgs& p, hipStream_t s)
{
    const int64_t vecs = div_up(p.ldo > p.cols ? p.ldo : p.cols, Vec<T>::N);
    int lanes = 1;
    while (lanes < 64 && lanes < vecs) lanes <<= 1;
    hipLaunchKernelGGL((k_slope<T>), dim3((unsigned)div_up(vecs, lanes), (unsigned)p.row_blocks), dim3(kBlock), 0, s, p,
                       lanes);
    return hipGetLastError();
}

template <typename T>
hipError_t LinearOps<T>::join(const GemmArgs& g, float plane_scale, hipStream_t s)
{
    // enough workgroups to fill the compute units, at least 4 parts a thread
    const int64_t places = g.rows * div_up(g.cols, 4);
    int slices = 1;
    while (slices < 32 && places * slices < 1024 * kBlock && g.splits >= 8 * slices) slices *= 2;
    hipLaunchKernelGGL((k_join<T>), dim3((unsigned)div_up(places, kBlock / slices)), dim3(kBlock), 0, s, g, plane_scale,
                       slices);
    return hipGetLastError();
}

template <typename T>
hipError_t LinearOps<T>::layout(const void* src, int64_t lds, int64_t rows, int64_t cols, bool transpose, void* dst,
                                int64_t ldd, hipStream_t s)
{
    const int64_t w = transpose ? cols : std::max(cols, ldd), h = transpose ? std::max(rows, ldd) : rows;
    hipLaunchKernelGGL((k_layout<T>), dim3((unsigned)div_up(w, kLayoutTile), (unsigned)div_up(h, kLayoutTile)),
                       dim3(kBlock), 0, s, (const T*)src, lds, rows, cols, transpose ? 1 : 0, (T*)dst, ldd);
    return hipGetLastError();
}

}  // namespace gsr
