// A linear layer of up to 128 inputs and outputs in one pass over the rows (16-bit types): its backward, and below it
// its forward.
//
//   dz = dy act'(z), dx = dz W, dW = dz^T x, db = column sums of dz
//
// Bound by HBM: dy, z and x are read once and dx is written once, where separate products would write dz and read it
// twice. W and some rows of dz and x are in LDS; a workgroup takes 32 to 128 rows at a time and keeps its dW and db in
// registers over all of them, so that both products come from the same tile: dx sums over dz's columns, dW over its
// rows. The next rows are fetched into registers under the products. Each workgroup writes its dW and db once;
// k_narrow_join adds them up in a fixed order. Measured: 1,000,000 x 128 x 128 in binary16 with relu 196 and 8 us, 5.0
// TB/s of what it has to move (separate products: 392); with gelu and an fp32 dW, in planes, 256 and 8 (bfloat16 270).
//
// LDS layout of each matrix: blocks of 64 columns, rows of 128 bytes, 16-byte slots XOR-ed with a hash of the row, so
// that the transposing reads (dW's operands, W) and the row reads (dz in dx) are free of bank conflicts. A fragment's
// value 4 t + e of lane group g is row (dW) or column (dx) 16 t + 4 g + e of its 32.
//
// P planes of dz: dz rounded to T (all that dx takes, as it is rounded to T itself), then what that leaves, so that an
// fp32 dW keeps 22 bits or more. In binary16 the second plane is scaled by 2^11 against underflow (below |dz| = 2^-14 dz
// is kept to within 2^-36, which is fewer bits); its products of 32 rows are summed apart and join dW's sums times 2^-11
// in fp32 (scaling x instead would round every x below 2^-3).
// An infinite or undefined x counts as 0 beside the lower planes, whose zeros and signs say nothing about its product
// with dz; a lane looks for one in its fragments of x.
#pragma once

#include "gemm.h"

namespace gsr {

namespace {

constexpr int kNarrowThreads = 256;

// Rows of a workgroup's tile: as many as leave room for two workgroups on a compute unit, in LDS and in registers.
constexpr int narrow_tile_rows(int out, int in, int planes, bool fast)
{
    if (out == 128 && in == 128) return planes == 1 && fast ? 64 : 32;
    return out >= 64 || in >= 64 ? 64 : 128;
}

__device__ __forceinline__ int narrow_hash(int row) { return (row & 6) | ((row >> 3) & 1); }

// Address of vector v (8 columns) of a row in a matrix of `rows` rows.
__device__ __forceinline__ int narrow_at(int rows, int row, int v)
{
    return (v >> 3) * rows * 128 + row * 128 + ((v & 7) ^ narrow_hash(row)) * 16;
}

// Fragment of 16 columns (group n) over rows [r0, r0 + 32), r0 a multiple of 16.
template <typename T>
__device__ __forceinline__ typename Mma<T>::Frag narrow_columns(const char* lds, int rows, int n, int r0)
{
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, r = 4 * g + (i >> 2);
    const char* at = lds + narrow_at(rows, r, 2 * n + ((i >> 1) & 1)) + (i & 1) * 8 + r0 * 128;
    s16x4 both[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at),
                     __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * 128))};
    typename Mma<T>::Frag out;
    __builtin_memcpy(&out, both, 16);
    return out;
}

// Fragment of rows [r0, r0 + 16) over columns [32 s, 32 s + 32).
template <typename T>
__device__ __forceinline__ typename Mma<T>::Frag narrow_rows(const char* lds, int rows, int r0, int s)
{
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    s16x4 both[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
        both[t] = *reinterpret_cast<const s16x4*>(lds + narrow_at(rows, r0 + i, 4 * s + 2 * t + (g >> 1)) + (g & 1) * 8);
    typename Mma<T>::Frag out;
    __builtin_memcpy(&out, both, 16);
    return out;
}

// The halves of a word of two 16-bit values whose exponents are all ones (infinite or undefined): their highest bits.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w)
{
    return ((w & 0x7FFF7FFFu) + (__is_same(T, f16) ? 0x04000400u : 0x00800080u)) & 0x80008000u;
}

// v with such values as 0
template <typename T, typename V>
__device__ __forceinline__ V finite_of(V v)
{
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t one = not_finite<T>(w[e]) >> 15;
        w[e] &= ~((one << 16) - one);
    }
    return __builtin_bit_cast(V, w);
}

// FAST: rows of dy, z and x are whole aligned vectors, and come through buffer loads whose range check turns what lies
// beyond the matrix into zeros; otherwise they are loaded at any alignment.
template <typename T, int OUT, int IN, int P, bool FAST>
__global__ __launch_bounds__(kNarrowThreads, 2) void k_narrow_bwd(NarrowArgs a)
{
    constexpr int R = narrow_tile_rows(OUT, IN, P, FAST), VO = OUT / 8, VI = IN / 8;
    constexpr int NO = R * VO / kNarrowThreads, NI = R * VI / kNarrowThreads;   // vectors of a thread
    constexpr int FO = OUT / 32, FI = IN / 32;                                  // fragments of a wave's part of dW
    // dx: a wave takes 16 rows and all columns at a time, or with 32 rows half of the columns
    constexpr int kBlocksX = R < 64 ? 1 : R / 64, FX = IN / 16 / (R < 64 ? 2 : 1);
    // (rows of 128 bytes at least)
    constexpr int kDz = R * (OUT < 64 ? 64 : OUT) * 2, kX = R * (IN < 64 ? 64 : IN) * 2;
    constexpr int kW = OUT * (IN < 64 ? 64 : IN) * 2, kBlock16 = 16 * FX * 16 * 2;
    typedef typename Mma<T>::Frag Frag;
    typedef typename Vec<T>::Packed Packed;
    __shared__ __attribute__((aligned(1024))) char lds[P * kDz + kX + kW + 4 * kBlock16];
    char* lds_dz = lds;
    char* lds_x = lds + P * kDz;
    char* lds_w = lds_x + kX;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lg = lane >> 4, li = lane & 15;
    char* block = lds_w + kW + wave * kBlock16;   // a wave's 16 rows of dx on their way out

    if (a.dx)
#pragma unroll
        for (int q = tid; q < OUT * VI; q += kNarrowThreads) {
            const int r = q / VI, v = q % VI;
            *reinterpret_cast<Packed*>(lds_w + narrow_at(OUT, r, v)) =
                load_any((const T*)a.w + r * a.ldw + v * 8, r < a.out ? a.in - v * 8 : 0);
        }

    Packed ry[NO], rz[NO], rx[NI];
    const int vo = tid % VO, ro = tid / VO, vi = tid % VI, ri = tid / VI;
    auto rows_of = [&](auto& regs, const void* p, int64_t ld, int64_t r0, int cols, int v, int first, int per) {
        constexpr int n = sizeof(regs) / 16;
        if constexpr (FAST) {
            const int left = (int)(a.rows - r0 < R ? a.rows - r0 : R);
            __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<T*>((const T*)p + r0 * ld), 0, left * (int)ld * 2, 0x00027000);
            const uint32_t off = v * 8 < cols ? (uint32_t)(first * (int)ld * 2 + v * 16) : kOutOfRange;
#pragma unroll
            for (int k = 0; k < n; ++k)
                regs[k] = __builtin_bit_cast(
                    Packed, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + (uint32_t)(k * per * (int)ld * 2), 0, 0));
        } else if (r0 + R + 8 <= a.rows) {
            // whole vectors at any alignment, the values beyond the row turned into zeros; what they reach beyond the
            // last row of the tile lies in the 8 rows behind it
            const int left = cols - v * 8;
            const T* src = (const T*)p + (r0 + first) * ld + (left > 0 ? v * 8 : 0);
#pragma unroll
            for (int k = 0; k < n; ++k) regs[k] = *reinterpret_cast<const typename Vec<T>::Any*>(src + k * per * ld);
            if (left < 8)
#pragma unroll
                for (int k = 0; k < n; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e >= left) regs[k][e] = (T)0.f;
        } else {
#pragma unroll
            for (int k = 0; k < n; ++k) {
                const int64_t r = r0 + first + k * per;
                regs[k] = load_any((const T*)p + r * ld + v * 8, r < a.rows ? cols - v * 8 : 0);
            }
        }
    };
    auto fetch = [&](int64_t r0) {
        rows_of(ry, a.dy, a.lddy, r0, a.out, vo, ro, kNarrowThreads / VO);
        if (a.act != GS_ACT_NONE) rows_of(rz, a.z, a.ldz, r0, a.out, vo, ro, kNarrowThreads / VO);
        if (a.dw) rows_of(rx, a.x, a.ldx, r0, a.in, vi, ri, kNarrowThreads / VI);
    };
    f32x4 dw[FO][FI] = {};
    float db[8] = {};
    const int wo = (wave >> 1) * (OUT / 32), wn = (wave & 1) * (IN / 32);   // first groups of 16 of the wave's part of dW
    const int64_t tiles = (a.rows + R - 1) / R;
    if (blockIdx.x < tiles) fetch((int64_t)blockIdx.x * R);
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            const int r = ro + k * (kNarrowThreads / VO);
            float v[8], z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = (float)ry[k][e];
                z[e] = (float)rz[k][e];
            }
            times_slope<8>(a.act, v, z);
            // (beyond the matrix dy is 0, and so is dz)
#pragma unroll
            for (int e = 0; e < 8; ++e) db[e] += v[e];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                Packed h;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[e] = (T)v[e];
                    // what the plane leaves; an infinite or undefined value is the first plane's alone
                    const float rest = v[e] - (float)h[e];
                    v[e] = fabsf(rest) < __builtin_inff() ? (__is_same(T, f16) ? rest * (1.f / kF16Plane) : rest) : 0.f;
                }
                *reinterpret_cast<Packed*>(lds_dz + p * kDz + narrow_at(R, r, vo)) = h;
            }
        }
        if (a.dw)
#pragma unroll
            for (int k = 0; k < NI; ++k)
                *reinterpret_cast<Packed*>(lds_x + narrow_at(R, ri + k * (kNarrowThreads / VI), vi)) = rx[k];
        __syncthreads();
        if (t + gridDim.x < tiles) fetch((t + gridDim.x) * R);
        if (a.dx)
#pragma unroll
            for (int k = 0; k < kBlocksX; ++k) {
                const int row = 16 * (R < 64 ? wave & 1 : wave * kBlocksX + k), group = R < 64 ? (wave >> 1) * FX : 0;
                f32x4 acc[FX] = {};
#pragma unroll
                for (int s = 0; s < OUT / 32; ++s) {
                    const Frag f = narrow_rows<T>(lds_dz, R, row, s);
#pragma unroll
                    for (int n = 0; n < FX; ++n)
                        acc[n] = Mma<T>::mma(narrow_columns<T>(lds_w, OUT, group + n, 32 * s), f, acc[n]);
                }
                // acc[n][r]: row li, column 16 (group + n) + 4 lg + r
#pragma unroll
                for (int n = 0; n < FX; ++n) {
                    typedef T V4 __attribute__((ext_vector_type(4)));
                    V4 h;
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[e] = (T)acc[n][e];
                    *reinterpret_cast<V4*>(block + li * (FX * 32) + ((2 * n + (lg >> 1)) ^ (li & 7 & (2 * FX - 1))) * 16 +
                                           (lg & 1) * 8) = h;
                }
                store_block<T, 16, FX * 16>(block, (T*)a.dx, a.lddx, t * R + row, a.rows, 16 * group, a.in);
            }
        if (a.dw) {
#pragma unroll
            for (int s = 0; s < R / 32; ++s) {
                Frag fx[FI];
#pragma unroll
                for (int n = 0; n < FI; ++n) fx[n] = narrow_columns<T>(lds_x, R, wn + n, 32 * s);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    Frag fz[FO];
#pragma unroll
                    for (int n = 0; n < FO; ++n) fz[n] = narrow_columns<T>(lds_dz + p * kDz, R, wo + n, 32 * s);
                    if (p == 1) {
                        uint32_t found = 0;   // values that are not finite
#pragma unroll
                        for (int n = 0; n < FI; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) found |= not_finite<T>(__builtin_bit_cast(u32x4, fx[n])[e]);
                        if (found)
#pragma unroll
                            for (int n = 0; n < FI; ++n) fx[n] = finite_of<T>(fx[n]);
                    }
#pragma unroll
                    for (int m = 0; m < FO; ++m)
#pragma unroll
                        for (int n = 0; n < FI; ++n) {
                            if (__is_same(T, f16) && p == 1) {
                                const f32x4 low = Mma<T>::mma(fx[n], fz[m], f32x4{});
#pragma unroll
                                for (int e = 0; e < 4; ++e) dw[m][n][e] = fmaf(low[e], kF16Plane, dw[m][n][e]);
                            } else {
                                dw[m][n] = Mma<T>::mma(fx[n], fz[m], dw[m][n]);
                            }
                        }
                }
            }
        }
        __syncthreads();   // LDS is free again
    }
    float* part = a.part + (int64_t)blockIdx.x * narrow_part(a.out, a.in);
    if (a.dw)
        // dw[m][n][r]: row 16 (wo + m) + li, columns 16 (wn + n) + 4 lg + r
#pragma unroll
        for (int m = 0; m < FO; ++m)
#pragma unroll
            for (int n = 0; n < FI; ++n) {
                const int i = 16 * (wo + m) + li, j = 16 * (wn + n) + 4 * lg;
                float v[4] = {dw[m][n][0], dw[m][n][1], dw[m][n][2], dw[m][n][3]};
                if (i < a.out) store_vec(part + i * a.in + j, a.in - j, v);
            }
    if (!a.db) return;
    static_assert(kNarrowThreads / VO * OUT * 4 <= (int)sizeof(lds), "the sums fit");
    float* s = reinterpret_cast<float*>(lds);   // [kNarrowThreads / VO][OUT]
#pragma unroll
    for (int e = 0; e < 8; ++e) s[ro * OUT + vo * 8 + e] = db[e];
    __syncthreads();
    for (int c = tid; c < a.out; c += kNarrowThreads) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kNarrowThreads / VO; ++k) v += s[k * OUT + c];
        part[a.out * a.in + c] = v;
    }
}

// dW and db: the sums of the workgroups' parts. A workgroup takes 16 places of 4 values, 16 threads share a place.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_narrow_join(NarrowArgs a, int parts)
{
    __shared__ f32x4 sums[kBlock];
    const int place = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int size = a.out * a.in + a.out, at = (blockIdx.x * 16 + place) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (at < size) {
#pragma unroll 8
        for (int k = slice; k < parts; k += 16)
            v += *reinterpret_cast<const f32x4*>(a.part + (int64_t)k * narrow_part(a.out, a.in) + at);
    }
    sums[threadIdx.x] = v;
    __syncthreads();
    if (slice != 0) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) v += sums[k * 16 + place];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int k = at + e;
        if (k >= size) return;
        if (k >= a.out * a.in) {
            if (a.db) a.db[k - a.out * a.in] = v[e];
        } else if (a.dw) {
            const int i = k / a.in;
            const int64_t o = i * a.lddw + (k - i * a.in);
            if (a.dw_f32)
                ((float*)a.dw)[o] = v[e];
            else
                ((T*)a.dw)[o] = (T)v[e];
        }
    }
}

// Forward of such a layer. W is in LDS; a wave takes 16 rows at a time and goes through them without a barrier: x comes
// from memory in the layout of the MFMAs' fragments, the next rows' while these are worked on, and the results leave
// through the wave's part of LDS as whole rows. Bound by HBM: 1,000,000 x 128 x 128 in binary16 with gelu and a residual
// 162 us, 4.7 TB/s (242 in tiles of the general product).
template <typename T, int OUT, int IN, bool FAST>
__global__ __launch_bounds__(kNarrowThreads) void k_narrow_fwd(GemmArgs g)
{
    constexpr int FJ = OUT / 16, KS = IN / 32, kRow = (IN < 64 ? 64 : IN) * 2, kBlock16 = 16 * OUT * 2;
    typedef typename Mma<T>::Frag Frag;
    typedef typename Vec<T>::Packed Packed;
    using W = Tile<T, OUT < 32 ? 32 : OUT, false, true, 64>;   // for its hash of a row
    __shared__ __attribute__((aligned(1024))) char lds[OUT * kRow + 4 * kBlock16];
    __shared__ float bias[OUT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lg = lane >> 4, li = lane & 15, in = (int)g.len, out = (int)g.cols;
    char* block = lds + OUT * kRow + wave * kBlock16;
    auto at = [](int row, int v) { return (v >> 3) * OUT * 128 + row * 128 + ((v & 7) ^ W::hash(row)) * 16; };
    for (int q = tid; q < OUT * (IN / 8); q += kNarrowThreads) {
        const int r = q / (IN / 8), v = q % (IN / 8);
        *reinterpret_cast<Packed*>(lds + at(r, v)) = load_any((const T*)g.b + r * g.ldb + v * 8, r < out ? in - v * 8 : 0);
    }
    for (int c = tid; c < OUT; c += kNarrowThreads) bias[c] = g.bias && c < out ? g.bias[c] : 0.f;
    __syncthreads();

    const int64_t blocks = (g.rows + 15) / 16, step = (int64_t)gridDim.x * 4;
    Packed next[KS];
    auto fetch = [&](int64_t b) {
        const int64_t r = b * 16 + li < g.rows ? b * 16 + li : g.rows - 1;   // (rows beyond are not stored)
        const T* src = (const T*)g.a + r * g.lda + lg * 8;
        if (FAST || b * 16 + 24 <= g.rows) {
            // whole vectors; what they reach beyond the last row (not FAST) lies in the 8 rows behind it
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int left = in - 32 * s - lg * 8;
                Packed t = {};
                if (left > 0) t = *reinterpret_cast<const typename Vec<T>::Any*>(src + 32 * s);
                if (!FAST)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e >= left) t[e] = (T)0.f;
                next[s] = t;
            }
        } else {
#pragma unroll
            for (int s = 0; s < KS; ++s) next[s] = load_any(src + 32 * s, in - 32 * s - lg * 8);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * 4 + wave;
    if (first < blocks) fetch(first);
    for (int64_t b = first; b < blocks; b += step) {
        Frag x[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) x[s] = next[s];
        if (b + step < blocks) fetch(b + step);
        const int64_t i = b * 16 + li;
        Packed r[FJ / 2];   // the residual, 8 columns of row i each
        if (g.residual)
#pragma unroll
            for (int q = 0; q < FJ / 2; ++q) {
                const int j = 32 * q + 8 * lg;
                r[q] = load_any((const T*)g.residual + i * g.ldr + j, i < g.rows ? out - j : 0);
            }
        f32x4 acc[FJ] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int f = 0; f < FJ; ++f) {
                // columns of f, f + 1 interleave in fours: a lane ends up with 8 neighbouring ones
                const int row = 32 * (f >> 1) + 4 * (f & 1) + 8 * (li >> 2) + (li & 3);
                const Frag w = *reinterpret_cast<const Frag*>(lds + at(row, 4 * s + lg));
                acc[f] = Mma<T>::mma(w, x[s], acc[f]);
            }
        float v[FJ / 2][8];
#pragma unroll
        for (int q = 0; q < FJ / 2; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[q][e] = acc[2 * q + e / 4][e & 3] + bias[32 * q + 8 * lg + e];
        auto put = [&]() {
#pragma unroll
            for (int q = 0; q < FJ / 2; ++q) {
                Packed t;
#pragma unroll
                for (int e = 0; e < 8; ++e) t[e] = (T)v[q][e];
                *reinterpret_cast<Packed*>(block + li * (OUT * 2) + ((4 * q + lg) ^ (li & 7 & (OUT / 8 - 1))) * 16) = t;
            }
        };
        if (g.z) {
            put();
            store_block<T, 16, OUT>(block, (T*)g.z, g.ldz, b * 16, g.rows, 0, out);
        }
#pragma unroll
        for (int q = 0; q < FJ / 2; ++q) {
            activate<8>(g.act, v[q]);
            if (g.residual)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[q][e] += (float)r[q][e];
        }
        put();
        store_block<T, 16, OUT>(block, (T*)g.out, g.ldo, b * 16, g.rows, 0, out);
    }
}

// Calls f with the number of columns that a narrow kernel is built for: 32, 64 or 128.
template <typename F>
void with_width(int n, F f)
{
    if (n <= 32)
        f(std::integral_constant<int, 32>());
    else if (n <= 64)
        f(std::integral_constant<int, 64>());
    else
        f(std::integral_constant<int, 128>());
}

template <typename T, int OUT, int IN, bool FAST>
void run_narrow(const NarrowArgs& a, int planes, int blocks, hipStream_t s)
{
    constexpr int kMost = __is_same(T, f16) ? 2 : 3;
    if (planes == 1)
        hipLaunchKernelGGL((k_narrow_bwd<T, OUT, IN, 1, FAST>), dim3(blocks), dim3(kNarrowThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_narrow_bwd<T, OUT, IN, kMost, FAST>), dim3(blocks), dim3(kNarrowThreads), 0, s, a);
}

template <typename T, bool FAST>
void run_narrow(const NarrowArgs& a, int planes, int blocks, hipStream_t s)
{
    with_width(a.out, [&](auto out) {
        with_width(a.in, [&](auto in) {
            run_narrow<T, decltype(out)::value, decltype(in)::value, FAST>(a, planes, blocks, s);
        });
    });
}

}  // namespace

template <typename T>
hipError_t NarrowOps<T>::backward(const NarrowArgs& a, bool fast, int planes, int blocks, hipStream_t s)
{
    fast ? run_narrow<T, true>(a, planes, blocks, s) : run_narrow<T, false>(a, planes, blocks, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !(a.dw || a.db)) return e;
    hipLaunchKernelGGL((k_narrow_join<T>), dim3((unsigned)div_up(a.out * a.in + a.out, 64)), dim3(kBlock), 0, s, a,
                       blocks);
    return hipGetLastError();
}

template <typename T>
hipError_t NarrowOps<T>::forward(const GemmArgs& g, bool fast, int blocks, hipStream_t s)
{
    with_width((int)g.cols, [&](auto out) {
        with_width((int)g.len, [&](auto in) {
            constexpr int OUT = decltype(out)::value, IN = decltype(in)::value;
            if (fast)
                hipLaunchKernelGGL((k_narrow_fwd<T, OUT, IN, true>), dim3(blocks), dim3(kNarrowThreads), 0, s, g);
            else
                hipLaunchKernelGGL((k_narrow_fwd<T, OUT, IN, false>), dim3(blocks), dim3(kNarrowThreads), 0, s, g);
        });
    });
    return hipGetLastError();
}

}  // namespace gsr
