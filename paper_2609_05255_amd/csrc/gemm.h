// Matrix product on the matrix cores with the linear operators' epilogue, one
// template for binary16, bfloat16 (16x16x32 MFMA) and fp32 (16x16x4 MFMA).
//
// A workgroup computes a BI x BJ tile of C with WI x WJ waves. The operands'
// tiles (64 bytes along the sum: 32 16-bit or 16 fp32 values) go from memory to
// LDS with buffer loads that write LDS directly, through a ring of STAGES tiles:
// STAGES - 1 of them are on their way while one is worked on, and a wait for the
// oldest alone (vmcnt) replaces a wait for all. Every step issues its loads, past
// the end too (the descriptor's range check turns those, like rows beyond the
// matrix, into zeros without reading), so that the counts stay the same.
// With AHEAD, a wave's fragments of the next tile are read under the MFMAs of
// this one.
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
    static constexpr int kStep = 32;                      // values along the sum per fragment
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
    static constexpr int kStep = 16;
    static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// ---- operand tiles ----------------------------------------------------------

// s_waitcnt until at most n vector memory operations are under way (the other counters: any number).
template <int n>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14));
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// NT: X rows of 4 KS slots along the sum; fragment rows are base + i (A) or the interleaved columns
// base + (i & 3) + 8 (i >> 2) (B), i = lane % 16. A 16-byte LDS read of half a wave takes two turns of 16 lanes, {0..3,
// 12..15, 20..23, 24..27} and the others (found from the conflict counter); the hash gives each turn's lanes different
// slots of the 256 bytes that the banks hold.
template <int KS, bool IS_B>
__device__ __forceinline__ int nt_hash(int row)
{
    if constexpr (KS == 1) return -(IS_B ? row >> 3 : row >> 2) & 3;
    return IS_B ? ((row >> 2) & 6) | ((row >> 1) & 1) : (row >> 1) & 7;
}

// TT: rows c of X * sizeof(T) / 16 slots.
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
template <typename T, int X, int KS, bool TT, bool IS_B, int THREADS>
struct Tile {
    static constexpr int kVec = 16 / (int)sizeof(T);
    static constexpr int kRowSlots = TT ? X / kVec : 4 * KS;
    static constexpr int kSlotsTotal = X * 4 * KS;
    static constexpr int kPasses = kSlotsTotal / THREADS;
    static constexpr int kBytes = X * 64 * KS;
    static_assert(kSlotsTotal % THREADS == 0, "whole passes");

    static __device__ __forceinline__ int row(int q) { return q / kRowSlots; }
    static __device__ __forceinline__ int vec(int q)
    {
        const int r = row(q), s = q % kRowSlots;
        return s ^ (TT ? tt_hash<T, X>(r) : nt_hash<KS, IS_B>(r));
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
        const int range = bytes > 0x7FFFFFF0 ? 0x7FFFFFF0 : bytes < 0 ? 0 : (int)bytes;
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

    // Fragment f of step s of a wave whose first row or column of the tile is wx.
    static __device__ __forceinline__ typename Mma<T>::Frag frag(const char* lds, int wx, int f, int s)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
        if constexpr (!TT) {
            const int r = IS_B ? wx + 32 * (f >> 1) + 4 * (f & 1) + 8 * (i >> 2) + (i & 3) : wx + 16 * f + i;
            const int slot = (4 * s + g) ^ nt_hash<KS, IS_B>(r);
            return *reinterpret_cast<const typename Mma<T>::Frag*>(lds + r * (64 * KS) + slot * 16);
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

// BI, BJ: the workgroup's tile; WI, WJ: its waves; KS: steps of the sum per tile in LDS; STAGES: tiles in the ring;
// AHEAD: fragments are read a tile ahead of their MFMAs. FAST: the operand that may be the caller's (A in NT, B in TT)
// is loaded asynchronously as well, as the other always is; otherwise it goes through registers, at any alignment.
template <bool TT_, int BI_, int BJ_, int WI_, int WJ_, int KS_, int STAGES_, bool AHEAD_, bool FAST_>
struct Shape {
    static constexpr bool TT = TT_, AHEAD = AHEAD_, FAST = FAST_;
    static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_, KS = KS_, STAGES = STAGES_;
    static constexpr int THREADS = WI * WJ * 64;
};

// Stores a wave's WR x WC block of results whose 8-value groups are in LDS, whole rows of it at a time: row r's
// vector v is at slot v ^ (r & 7) of its row.
template <typename T, int WR, int WC>
__device__ __forceinline__ void store_block(const char* lds, T* out, int64_t ld, int64_t i, int64_t rows, int64_t j,
                                            int64_t cols)
{
    constexpr int N = Vec<T>::N, kVecs = WC / N, kRowBytes = WC * (int)sizeof(T);
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < WR * kVecs / 64; ++k) {
        const int q = k * 64 + lane, r = q / kVecs, v = q % kVecs;
        const int64_t left = cols - (j + v * N);
        if (i + r >= rows || left <= 0) continue;
        const typename Vec<T>::Packed t =
            *reinterpret_cast<const typename Vec<T>::Packed*>(lds + r * kRowBytes + (v ^ (r & 7 & (kVecs - 1))) * 16);
        T* o = out + (i + r) * ld + j + v * N;
        if (left >= N) {
            *reinterpret_cast<typename Vec<T>::Any*>(o) = t;
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (e < left) o[e] = t[e];
        }
    }
}

template <typename T, class S>
__global__ __launch_bounds__(S::THREADS) void k_gemm(GemmArgs g)
{
    constexpr bool TT = S::TT;
    constexpr int BI = S::BI, BJ = S::BJ, WI = S::WI, WJ = S::WJ, KS = S::KS, kStages = S::STAGES;
    constexpr int WR = BI / WI, WC = BJ / WJ, FI = WR / 16, FJ = WC / 16;
    constexpr int kBK = Mma<T>::kStep * KS;
    using TA = Tile<T, BI, KS, TT, false, S::THREADS>;
    using TB = Tile<T, BJ, KS, TT, true, S::THREADS>;
    constexpr int kTileBytes = TA::kBytes + TB::kBytes;
    constexpr bool kAsyncA = S::FAST || TT, kAsyncB = S::FAST || !TT;
    static_assert(TT || FJ % 2 == 0, "columns interleave between pairs of fragments");
    static_assert(TT || WI * WJ * WR * WC * (int)sizeof(T) <= kStages * kTileBytes, "the results pass through LDS");
    __shared__ __attribute__((aligned(1024))) char lds[kStages * kTileBytes];

    const int64_t tiles_i = (g.rows + BI - 1) / BI, tiles_j = (g.cols + BJ - 1) / BJ;
    int64_t ti, tj;
    tile_of(blockIdx.x, tiles_i, tiles_j, &ti, &tj);
    const int64_t i0 = ti * BI, j0 = tj * BJ;
    const int part = blockIdx.y, plane = part / g.splits, split = part - plane * g.splits;
    const int64_t c_begin = split * g.split_len;
    const int64_t c_end = c_begin + g.split_len < g.len ? c_begin + g.split_len : g.len;
    const T* a = (const T*)g.a + plane * g.plane_stride;
    const T* b = (const T*)g.b;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = (wave / WJ) * WR, wj = (wave % WJ) * WC;
    const int lane = threadIdx.x & 63, lg = lane >> 4, li = lane & 15;

    typedef typename Mma<T>::Frag Frag;
    f32x4 acc[FI][FJ] = {};
    auto read = [&](const char* from, Frag(&fa)[KS][FI], Frag(&fb)[KS][FJ]) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
#pragma unroll
            for (int f = 0; f < FJ; ++f) fb[s][f] = TB::frag(from + TA::kBytes, wj, f, s);
#pragma unroll
            for (int f = 0; f < FI; ++f) fa[s][f] = TA::frag(from, wi, f, s);
        }
    };
    auto multiply = [&](const Frag(&fa)[KS][FI], const Frag(&fb)[KS][FJ]) {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int q = 0; q < FJ; ++q) acc[p][q] = Mma<T>::mma(fb[s][q], fa[s][p], acc[p][q]);
    };
    const int steps = c_end > c_begin ? (int)((c_end - c_begin + kBK - 1) / kBK) : 0;
    if constexpr (S::FAST) {
        constexpr int kLoads = TA::kPasses + TB::kPasses;   // of a thread per tile
        int64_t c0 = c_begin;
        auto fetch = [&](char* to) {
            TA::load_async(to, a, g.lda, g.a_rows, i0, g.rows, c0, c_end);
            TB::load_async(to + TA::kBytes, b, g.ldb, g.b_rows, j0, g.cols, c0, c_end);
            c0 += kBK;
        };
        char* cur = lds;
        char* to = lds;
        auto next = [&](char* p) { return p + kTileBytes == lds + kStages * kTileBytes ? lds : p + kTileBytes; };
        for (int k = 0; k < kStages - 1; ++k, to = next(to)) fetch(to);   // (AHEAD: all of them)
        if constexpr (S::AHEAD) {
            static_assert(KS == 2 && kStages == 2, "two halves of two tiles");
            Frag fa[2][FI], fb[2][FJ];
            auto half = [&](const char* from, int s, Frag(&ra)[FI], Frag(&rb)[FJ]) {
#pragma unroll
                for (int f = 0; f < FJ; ++f) rb[f] = TB::frag(from + TA::kBytes, wj, f, s);
#pragma unroll
                for (int f = 0; f < FI; ++f) ra[f] = TA::frag(from, wi, f, s);
            };
            auto product = [&](const Frag(&ma)[FI], const Frag(&mb)[FJ]) {
#pragma unroll
                for (int p = 0; p < FI; ++p)
#pragma unroll
                    for (int q = 0; q < FJ; ++q) acc[p][q] = Mma<T>::mma(mb[q], ma[p], acc[p][q]);
                // the reads spread over the MFMAs
                constexpr int kReads = (FI + FJ) * (TT ? 2 : 1);
#pragma unroll
                for (int k = 0; k < kReads; ++k) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x008, FI * FJ / kReads, 0);
                }
            };
            fetch(to);
            wait_loads<kLoads>();
            barrier();
            half(cur, 0, fa[0], fb[0]);
            for (int t = 0; t < steps; ++t) {
                half(cur, 1, fa[1], fb[1]);
                product(fa[0], fb[0]);
                __builtin_amdgcn_sched_barrier(0);
                wait_loads<0>();
                __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): this wave is done with tile t
                barrier();                            // as all are, and tile t + 1 is here
                fetch(cur);                           // tile t + 2
                cur = next(cur);
                half(cur, 0, fa[0], fb[0]);
                product(fa[1], fb[1]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            Frag fa[KS][FI], fb[KS][FJ];
            for (int t = 0; t < steps; ++t) {
                wait_loads<(kStages - 2) * kLoads>();
                barrier();   // tile t is here, and all waves are done with tile t - 1
                fetch(to);
                read(cur, fa, fb);
                multiply(fa, fb);
                cur = next(cur);
                to = next(to);
            }
        }
        wait_loads<0>();   // nothing may still write to LDS
    } else {
        static_assert(kStages == 2, "two stages");
        Frag fa[KS][FI], fb[KS][FJ];
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
        if (steps > 0) {
            fetch(lds, c_begin);
            settle(lds);
        }
        for (int t = 0; t < steps; ++t) {
            char* nxt = lds + ((t + 1) & 1) * kTileBytes;
            __syncthreads();   // tile t has arrived, and the other is no longer read
            if (t + 1 < steps) fetch(nxt, c_begin + (int64_t)(t + 1) * kBK);
            read(lds + (t & 1) * kTileBytes, fa, fb);
            multiply(fa, fb);
            if (t + 1 < steps) settle(nxt);
        }
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
        return;
    }
    const int64_t i1 = i0 + wi, j1 = j0 + wj;
    if (g.part) {
#pragma unroll
        for (int q = 0; q < FJ; q += 2) {
            const int64_t j = j1 + 16 * q + 8 * lg;
#pragma unroll
            for (int p = 0; p < FI; ++p) {
                const int64_t i = i1 + 16 * p + li;
                if (i >= g.rows || j >= g.cols) continue;
                float* o = g.part + ((int64_t)part * g.rows + i) * g.cols + j;
                float lo[4], hi[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    lo[e] = acc[p][q][e];
                    hi[e] = acc[p][q + 1][e];
                }
                store_vec(o, g.cols - j, lo);
                store_vec(o + 4, g.cols - j - 4, hi);
            }
        }
        return;
    }
    // A wave's results go through its own part of LDS, so that they are stored as whole rows of its block: z, then y.
    constexpr int N = Vec<T>::N, kVecs = WC / N;
    char* block = lds + wave * (WR * WC * (int)sizeof(T));
    auto put = [&](int p, int q, const float* v) {
        const int r = 16 * p + li;
#pragma unroll
        for (int e = 0; e < 8; e += N) {
            typename Vec<T>::Packed t;
#pragma unroll
            for (int k = 0; k < N; ++k) t[k] = (T)v[e + k];
            const int vec = (16 * q + 8 * lg + e) / N;
            *reinterpret_cast<typename Vec<T>::Packed*>(block + r * (WC * (int)sizeof(T)) +
                                                        (vec ^ (r & 7 & (kVecs - 1))) * 16) = t;
        }
    };
    barrier();   // all waves are done with the tiles
#pragma unroll
    for (int q = 0; q < FJ; ++q) {
        const int64_t j = j1 + 16 * (q & ~1) + 8 * lg + 4 * (q & 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float bias = g.bias && j + e < g.cols ? g.bias[j + e] : 0.f;
#pragma unroll
            for (int p = 0; p < FI; ++p) acc[p][q][e] += bias;
        }
    }
    if (g.z) {
#pragma unroll
        for (int p = 0; p < FI; ++p)
#pragma unroll
            for (int q = 0; q < FJ; q += 2) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = acc[p][q + (e >> 2)][e & 3];
                put(p, q, v);
            }
        store_block<T, WR, WC>(block, (T*)g.z, g.ldz, i1, g.rows, j1, g.cols);
    }
#pragma unroll
    for (int p = 0; p < FI; ++p)
#pragma unroll
        for (int q = 0; q < FJ; q += 2) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[p][q + (e >> 2)][e & 3];
            activate<8>(g.act, v);
            const int64_t i = i1 + 16 * p + li, j = j1 + 16 * q + 8 * lg;
            if (g.residual && i < g.rows && j < g.cols) {
                const T* r = (const T*)g.residual + i * g.ldr + j;
                float t[8];
#pragma unroll
                for (int e = 0; e < 8; e += N) load_vec(r + e, g.cols - j - e, t + e);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += t[e];
            }
            put(p, q, v);
        }
    store_block<T, WR, WC>(block, (T*)g.out, g.ldo, i1, g.rows, j1, g.cols);
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

template <typename T, class S>
hipError_t run_gemm(const GemmArgs& g, hipStream_t s)
{
    const int64_t tiles = div_up(g.rows, S::BI) * div_up(g.cols, S::BJ);
    hipLaunchKernelGGL((k_gemm<T, S>), dim3((unsigned)tiles, (unsigned)(g.planes * g.splits)), dim3(S::THREADS), 0, s,
                       g);
    return hipGetLastError();
}

template <typename T, bool TT, int BI, int BJ, int WI, int WJ>
hipError_t run_any(bool fast, const GemmArgs& g, hipStream_t s)
{
    return fast ? run_gemm<T, Shape<TT, BI, BJ, WI, WJ, 2, 2, false, true>>(g, s)
                : run_gemm<T, Shape<TT, BI, BJ, WI, WJ, 2, 2, false, false>>(g, s);
}

}  // namespace

template <typename T>
hipError_t LinearOps<T>::gemm_nt(int tile, bool fast_a, const GemmArgs& g, hipStream_t s)
{
    if (tile == kTile256) {   // fast_a, 16-bit
        if constexpr (sizeof(T) == 2) return run_gemm<T, Shape<false, 256, 256, 2, 4, 2, 2, true, true>>(g, s);
    }
    if (tile == kTile128) return run_any<T, false, 128, 128, 2, 2>(fast_a, g, s);
    if (tile == kTile128x64) return run_any<T, false, 128, 64, 4, 1>(fast_a, g, s);
    return run_any<T, false, 64, 64, 2, 2>(fast_a, g, s);
}

template <typename T>
hipError_t LinearOps<T>::gemm_tt(int tile, bool fast_b, const GemmArgs& g, hipStream_t s)
{
    if (tile == kTile256) {   // fast_b, 16-bit
        if constexpr (sizeof(T) == 2) return run_gemm<T, Shape<true, 256, 256, 2, 4, 2, 2, true, true>>(g, s);
    }
    if (tile == kTile128) return run_any<T, true, 128, 128, 2, 2>(fast_b, g, s);
    return run_any<T, true, 64, 64, 2, 2>(fast_b, g, s);
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
