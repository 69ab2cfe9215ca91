// Matrix product on the matrix cores with the linear operators' epilogue, one
// template for binary16, bfloat16 (16x16x32 MFMA) and fp32 (16x16x4 MFMA).
//
// A workgroup computes a BI x BJ tile of C with WI x WJ waves. The operands'
// tiles (128 bytes along the sum: 64 16-bit or 32 fp32 values) go from memory to
// LDS with buffer loads that write LDS directly, the next tile's under the current
// one's MFMAs. What lies beyond a matrix the descriptor's range check turns into
// zeros without reading. The 256 x 256 tile, whose workgroup is alone on its
// compute unit, also reads its fragments ahead and spreads its loads between the
// MFMAs (AHEAD); two workgroups of the 128 x 128 tile and five of the 64 x 64 one
// overlap each other.
// Measured at 8,192 x 4,096 x 4,096 in bfloat16: 1,110, 870 and 580 TFLOP/s (NT),
// 1,060, 780 and 590 (TT); the MFMAs of the largest tile alone reach 1,480 under
// the power limit, a library's product 1,320 (NT) and 1,060 (TT). What the largest
// tile loses lies before its first MFMA and behind its last one, about 27 us in a
// launch of two rounds of workgroups. In fp32, 131 of a library's 151.
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

#include <type_traits>

#include "activation.h"
#include "linear.h"

namespace gsr {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr uint32_t kOutOfRange = 0x80000000u;   // beyond any descriptor's range (at most 2^31 - 1 bytes)

// D[j][i] += sum over kStep values of B[j] A[i], 16 x 16. A lane holds one row (lane % 16) of an operand, 16 bytes of
// it, and of D the column i = lane % 16, rows j = 4 (lane / 16) + r.
template <typename T>
struct Mma {
    typedef T Frag __attribute__((ext_vector_type(8)));
    static constexpr int kStep = 32;
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

// (behind a barrier LDS that a wave has read is written again: its reads have ended before it, by this wait and not only
// where their use happens to stand in front of the barrier)
__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Geometry of one operand's tile in LDS: X rows or columns, 128 bytes of the sum, slots of 16 bytes.
//
// NT: X rows of 8 slots along the sum. A fragment's lane i reads row base + i (A) or base + interleaved(i) (B). A
// 16-byte LDS read of half a wave takes two turns of 16 lanes, {0..3, 12..15, 20..23, 24..27} and the others (found
// from the conflict counter); the hash gives the lanes of a turn different slots of the 256 bytes that the banks hold.
//
// TT: blocks of 128 bytes across (64 16-bit or 32 fp32 columns), each kBK rows of 8 slots. 16-bit fragments come
// through the transposing read, which gives 16 lanes the columns of 4 rows of 32 bytes; the sum's order within a
// fragment is free as long as A and B agree: value 4 t + e of lane group g is row 16 t + 4 g + e, so that the hash, and
// with it the address but for a constant, does not depend on t or on the step.
template <typename T, int X, bool TT, bool IS_B, int THREADS>
struct Tile {
    static constexpr int kVec = 16 / (int)sizeof(T);
    static constexpr int kBK = 128 / (int)sizeof(T);       // values along the sum
    static constexpr int kSlotsTotal = X * 8;
    static constexpr int kPasses = kSlotsTotal / THREADS;
    static constexpr int kBytes = X * 128;
    static constexpr int kBlockBytes = kBK * 128;          // TT
    static_assert(kSlotsTotal % THREADS == 0, "whole passes");
    typedef typename Mma<T>::Frag Frag;

    // (the threads of a workgroup that load one tile together: THREADS neighbours)
    static __device__ __forceinline__ int thread() { return threadIdx.x % THREADS; }
    static __device__ __forceinline__ int hash(int row)
    {
        if constexpr (TT) return sizeof(T) == 2 ? row & 6 : (row & 2) << 1;
        return IS_B ? ((row >> 2) & 6) | ((row >> 1) & 1) : (row >> 1) & 7;
    }
    // The row of LDS, and the vector of the operand's row, that slot q holds.
    static __device__ __forceinline__ int row(int q) { return TT ? q / 8 % kBK : q / 8; }
    static __device__ __forceinline__ int vec(int q)
    {
        const int v = (q & 7) ^ hash(row(q));
        return TT ? q / (8 * kBK) * 8 + v : v;
    }

    // LDS <- memory, 16 bytes per lane and pass. Issued by hand, and waited for by hand (wait_loads): the compiler would
    // wait for all of them before each transposing read, as it takes the two for accesses to the same memory. The
    // instruction has no destination register. Every pass of every tile is issued: what lies beyond the operand, or
    // beyond the part of the sum that ends at c_end, is turned into zeros by the descriptor's range check.
    struct Source {
        const T* p;             // the tile's first row (NT) or column (TT), at its position along the sum
        int64_t step;           // values per tile along the sum, in p
        int row_bytes, x_bytes;
        int x_left, c_left;     // rows (NT) or columns (TT), and values of the sum from here on
        int wave_bytes;         // this wave's part of a pass
        uint32_t off[kPasses];  // of each pass, from p
        __device__ __forceinline__ Source(const T* base, int64_t ld, int64_t x0, int64_t x_end, int64_t c0, int64_t c_end)
        {
            p = TT ? base + c0 * ld + x0 : base + x0 * ld + c0;
            step = (int64_t)kBK * (TT ? ld : 1);
            row_bytes = (int)(ld * (int64_t)sizeof(T));
            x_bytes = TT ? (int)(x0 * (int64_t)sizeof(T)) : 0;
            x_left = (int)(x_end - x0);
            c_left = (int)(c_end - c0);
            wave_bytes = __builtin_amdgcn_readfirstlane(thread() >> 6) * 1024;
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const int q = k * THREADS + thread();
                off[k] = (uint32_t)(row(q) * row_bytes) + vec(q) * 16;
                if (TT && vec(q) * kVec >= x_left) off[k] = kOutOfRange;
            }
            cut();
        }
        // (vectors are whole in this form: the sum ends between them)
        __device__ __forceinline__ void cut()
        {
            if (!TT && c_left < kBK)
#pragma unroll
                for (int k = 0; k < kPasses; ++k)
                    if (vec(k * THREADS + thread()) * kVec >= c_left) off[k] = kOutOfRange;
        }
        __device__ __forceinline__ void pass(char* lds, int k) const
        {
            // bytes from p to the end of the tile's last row: of X rows, or of the tile's part of the sum. At most 2^30.
            const int rows = TT ? min(max(c_left, 0), kBK) : min(x_left, X);
            const uint64_t at = reinterpret_cast<uint64_t>(p);
            u32x4 rsrc;   // base, no stride, range, untyped
            rsrc[0] = __builtin_amdgcn_readfirstlane((uint32_t)at);
            rsrc[1] = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xFFFF);
            rsrc[2] = __builtin_amdgcn_readfirstlane(max(rows * row_bytes - x_bytes, 0));
            rsrc[3] = 0x00027000;
            const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)lds) + k * (THREADS * 16) +
                                wave_bytes;
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                         :
                         : "v"(off[k]), "s"(rsrc), "s"(to)
                         : "memory", "m0");
        }
        __device__ __forceinline__ void advance()
        {
            p += step;
            c_left -= kBK;
            cut();
        }
        __device__ __forceinline__ void load(char* lds)
        {
#pragma unroll
            for (int k = 0; k < kPasses; ++k) pass(lds, k);
            advance();
        }
    };

    // registers <- memory at any alignment. Rows beyond the matrix read as its last one (NT: their results are never
    // stored) or, along the sum, as zeros (TT).
    typedef typename Vec<T>::Packed Packed;
    static __device__ __forceinline__ void load_regs(Packed (&r)[kPasses], const T* p, int64_t ld, int64_t x0,
                                                     int64_t x_end, int64_t c0, int64_t c_end)
    {
        const int64_t r0 = TT ? c0 : x0, rows_end = TT ? c_end : x_end;
        const int64_t v0 = TT ? x0 : c0, v_end = TT ? x_end : c_end;
        const bool whole = v0 + (TT ? X : kBK) <= v_end;   // no vector of the tile ends beyond the matrix
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int q = k * THREADS + thread();
            const int64_t rr = r0 + row(q), v = v0 + (int64_t)vec(q) * kVec;
            const T* src = p + (rr < rows_end ? rr : rows_end - 1) * ld + v;
            Packed t = {};
            if (whole) {
                if (!TT || r0 < rows_end) t = *reinterpret_cast<const typename Vec<T>::Any*>(src);
            } else if (r0 < rows_end) {
                t = load_any(src, v_end - v);
            }
            if (TT && rr >= rows_end) t = Packed{};
            r[k] = t;
        }
    }
    static __device__ __forceinline__ void store_regs(char* lds, const Packed (&r)[kPasses])
    {
#pragma unroll
        for (int k = 0; k < kPasses; ++k) *reinterpret_cast<Packed*>(lds + (k * THREADS + thread()) * 16) = r[k];
    }

    // Fragment f of step s of a wave whose first row or column of the tile is wx.
    static __device__ __forceinline__ Frag frag(const char* lds, int wx, int f, int s)
    {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
        if constexpr (!TT) {
            const int r = IS_B ? wx + 32 * (f >> 1) + 4 * (f & 1) + 8 * (i >> 2) + (i & 3) : wx + 16 * f + i;
            const int slot = (4 * s + g) ^ hash(r);
            return *reinterpret_cast<const Frag*>(lds + r * 128 + slot * 16);
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes: 4 rows of one group of 16 columns
            const int n = wx / 16 + f, r = 4 * g + (i >> 2);
            const char* at = lds + (n >> 2) * kBlockBytes + r * 128 + ((((n & 3) * 2) ^ hash(r)) + ((i >> 1) & 1)) * 16 +
                             (i & 1) * 8 + s * (32 * 128);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * 128));
            s16x4 both[2] = {lo, hi};
            Frag out;
            __builtin_memcpy(&out, both, 16);
            return out;
        } else {
            const int col = wx + 16 * f + i;
            const char* at = lds + (col >> 5) * kBlockBytes + g * 128 + ((((col & 31) >> 2) ^ hash(g)) * 4 + (col & 3)) * 4;
            Frag out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = *reinterpret_cast<const float*>(at + (16 * s + 4 * e) * 128);
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

// BI, BJ: the workgroup's tile; WI, WJ: the waves that share it; AHEAD: fragments are read half a tile ahead of their
// MFMAs. FAST: the operand that may be the caller's (A in NT, B in TT) is loaded asynchronously as well, as the other
// always is; otherwise it goes through registers, at any alignment. WAYS: so many groups of WI x WJ waves, each with
// LDS of its own, take a part of the sum each, and the first adds the others' results to its own. Where there are no
// more workgroups than compute units, one group alone would wait for each tile's loads and LDS reads in turn; four
// overlap (1,024 x 1,024, 64 x 64 tiles, bfloat16: 21 us against 33 with a sum of 4,096, 11.3 against 13.9 with 2,048,
// but 6.5 against 6.1 with 512).
template <bool TT_, int BI_, int BJ_, int WI_, int WJ_, bool AHEAD_, bool FAST_, int WAYS_ = 1>
struct Shape {
    static constexpr bool TT = TT_, AHEAD = AHEAD_, FAST = FAST_;
    static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_, WAYS = WAYS_;
    static constexpr int THREADS = WI * WJ * 64;   // of a group
    // LDS of the kernel itself, or of the launch for a sum of so many tiles
    static constexpr bool STATIC_LDS = AHEAD || WAYS > 1;
    static constexpr int lds_bytes(int64_t tiles, int size)
    {
        const int tile = (BI + BJ) * 128, results = TT ? 0 : BI * BJ * size;
        return tiles > 1 || results > tile || STATIC_LDS ? 2 * tile : tile;
    }
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
__global__ __launch_bounds__(S::THREADS * S::WAYS) void k_gemm(GemmArgs g)
{
    constexpr bool TT = S::TT;
    constexpr int BI = S::BI, BJ = S::BJ, WI = S::WI, WJ = S::WJ;
    constexpr int WR = BI / WI, WC = BJ / WJ, FI = WR / 16, FJ = WC / 16;
    using Mm = Mma<T>;
    using TA = Tile<T, BI, TT, false, S::THREADS>;
    using TB = Tile<T, BJ, TT, true, S::THREADS>;
    constexpr int kBK = TA::kBK, kSteps = kBK / Mm::kStep;   // of the sum, and of MFMAs, per tile
    constexpr int kTileBytes = TA::kBytes + TB::kBytes;
    [[maybe_unused]] constexpr bool kAsyncA = S::FAST || TT, kAsyncB = S::FAST || !TT;
    static_assert(TT || FJ % 2 == 0, "columns interleave between pairs of fragments");
    static_assert(TT || BI * BJ * (int)sizeof(T) <= S::lds_bytes(1, sizeof(T)), "the results pass through LDS");
    // (as much as the launch gives: two tiles, or one if the sum has no more, so that more workgroups fit)
    extern __shared__ __attribute__((aligned(1024))) char lds_given[];
    __shared__ __attribute__((aligned(1024))) char lds_own[S::AHEAD  ? 2 * kTileBytes + TA::kBytes
                                                           : S::WAYS > 1 ? S::WAYS * 2 * kTileBytes
                                                                         : 16];
    const int group = S::WAYS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / S::THREADS) : 0;
    char* lds = S::STATIC_LDS ? lds_own + group * 2 * kTileBytes : lds_given;

    const int64_t tiles_i = (g.rows + BI - 1) / BI, tiles_j = (g.cols + BJ - 1) / BJ;
    int64_t ti, tj;
    tile_of(blockIdx.x, tiles_i, tiles_j, &ti, &tj);
    const int64_t i0 = ti * BI, j0 = tj * BJ;
    int64_t c_begin = blockIdx.y * g.split_len;
    int64_t c_end = c_begin + g.split_len < g.len ? c_begin + g.split_len : g.len;
    int steps = c_end > c_begin ? (int)((c_end - c_begin + kBK - 1) / kBK) : 0;
    if constexpr (S::WAYS > 1) {
        // the group's part; beyond the sum's end there is nothing to load, and zeros are added
        steps = (steps + S::WAYS - 1) / S::WAYS;
        c_begin += group * ((int64_t)steps * kBK);
        c_end = c_begin + (int64_t)steps * kBK < c_end ? c_begin + (int64_t)steps * kBK : c_end;
    }
    const T* b = (const T*)g.b;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x % S::THREADS >> 6);
    const int wi = (wave / WJ) * WR, wj = (wave % WJ) * WC;
    const int lane = threadIdx.x & 63;

    typedef typename Mm::Frag Frag;
    f32x4 acc[FI][FJ] = {};
    auto read = [&](const char* from, Frag(&fa)[kSteps][FI], Frag(&fb)[kSteps][FJ]) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
#pragma unroll
            for (int f = 0; f < FJ; ++f) fb[s][f] = TB::frag(from + TA::kBytes, wj, f, s);
#pragma unroll
            for (int f = 0; f < FI; ++f) fa[s][f] = TA::frag(from, wi, f, s);
        }
    };
    auto multiply = [&](const Frag(&fa)[kSteps][FI], const Frag(&fb)[kSteps][FJ]) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int q = 0; q < FJ; ++q) acc[p][q] = Mm::mma(fb[s][q], fa[s][p], acc[p][q]);
    };
    // A's planes, the least significant one first, whose sums are scaled into the next one's
    for (int plane = (TT ? g.planes : 1) - 1; plane >= 0; --plane) {
        const T* a = (const T*)g.a + (TT ? plane * g.plane_stride : 0);
        if constexpr (S::FAST) {
            constexpr int kLoads = TA::kPasses + TB::kPasses;   // of a thread per tile
            typename TA::Source sa(a, g.lda, i0, g.rows, c_begin, c_end);
            typename TB::Source sb(b, g.ldb, j0, g.cols, c_begin, c_end);
            if constexpr (S::AHEAD) {
                // Three tiles of A and two of B in LDS, each of two halves along the sum. While a half's MFMAs run, the next
                // half's fragments are read; A's tile t + 2 is loaded under the first half of tile t, B's under the second,
                // where tile t's own fragments have all been read. Behind each row of MFMAs stand a few reads and loads:
                // issued together they would hold the wave, and the MFMAs behind them, until the memory pipe takes them.
                constexpr int kHalf = kSteps / 2, kRows = kHalf * FI;   // rows of MFMAs in a half
                static_assert(kRows == 2 * TA::kPasses && kRows == 2 * TB::kPasses &&
                                  kHalf * (FI + FJ) <= 2 * (kRows - 1), "the loads and reads of a half fit its rows");
                char* a_lds[3] = {lds, lds + TA::kBytes, lds + 2 * TA::kBytes};
                char* b_lds[2] = {lds + 3 * TA::kBytes, lds + 3 * TA::kBytes + TB::kBytes};
                Frag fa[2][kHalf][FI], fb[2][kHalf][FJ];
                for (int k = 0; k < 2; ++k) {
                    sa.load(a_lds[k]);
                    sb.load(b_lds[k]);
                }
                wait_loads<kLoads>();
                barrier();
                auto fetch = [&](const char* from_a, const char* from_b, int half, int k, Frag(&na)[kHalf][FI],
                                 Frag(&nb)[kHalf][FJ]) {
                    const int s = k / (FI + FJ), f = k % (FI + FJ);
                    if (s >= kHalf) return;
                    if (f < FJ)
                        nb[s][f] = TB::frag(from_b, wj, f, half * kHalf + s);
                    else
                        na[s][f - FJ] = TA::frag(from_a, wi, f - FJ, half * kHalf + s);
                };
#pragma unroll
                for (int k = 0; k < 2 * kRows; ++k) fetch(a_lds[0], b_lds[0], 0, k, fa[0], fb[0]);
                auto half = [&](const Frag(&ma)[kHalf][FI], const Frag(&mb)[kHalf][FJ], const char* from_a,
                                const char* from_b, int h, Frag(&na)[kHalf][FI], Frag(&nb)[kHalf][FJ], auto load) {
#pragma unroll
                    for (int u = 0; u < kRows; ++u) {
                        const int s = u / FI, p = u % FI;
#pragma unroll
                        for (int q = 0; q < FJ; ++q) acc[p][q] = Mm::mma(mb[s][q], ma[s][p], acc[p][q]);
                        __builtin_amdgcn_sched_barrier(0);
                        fetch(from_a, from_b, h, 2 * u, na, nb);
                        fetch(from_a, from_b, h, 2 * u + 1, na, nb);
                        if (u % 2 == 0) load(u / 2);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                for (int t = 0; t < steps; ++t) {
                    half(fa[0], fb[0], a_lds[0], b_lds[0], 1, fa[1], fb[1], [&](int k) { sa.pass(a_lds[2], k); });
                    sa.advance();
                    wait_loads<TA::kPasses>();
                    barrier();   // all waves have tile t's fragments, and tile t + 1 is here
                    half(fa[1], fb[1], a_lds[1], b_lds[1], 0, fa[0], fb[0], [&](int k) { sb.pass(b_lds[0], k); });
                    sb.advance();
                    char* x = a_lds[0];
                    a_lds[0] = a_lds[1];
                    a_lds[1] = a_lds[2];
                    a_lds[2] = x;
                    x = b_lds[0];
                    b_lds[0] = b_lds[1];
                    b_lds[1] = x;
                }
            } else {
                Frag fa[kSteps][FI], fb[kSteps][FJ];
                sa.load(lds);
                sb.load(lds + TA::kBytes);
                for (int t = 0; t < steps; ++t) {
                    char* cur = lds + (t & 1) * kTileBytes;
                    char* nxt = lds + ((t + 1) & 1) * kTileBytes;
                    wait_loads<0>();
                    barrier();   // tile t is here, and all waves are done with tile t - 1
                    if (t + 1 < steps) {
                        sa.load(nxt);
                        sb.load(nxt + TA::kBytes);
                    }
                    read(cur, fa, fb);
                    multiply(fa, fb);
                }
            }
            wait_loads<0>();   // nothing may still write to LDS
        } else {
            using TR = std::conditional_t<kAsyncA, TB, TA>;   // the operand that goes through registers
            Frag fa[kSteps][FI], fb[kSteps][FJ];
            typename TR::Packed regs[TR::kPasses];
            typename TA::Source sa(a, g.lda, i0, g.rows, c_begin, c_end);
            typename TB::Source sb(b, g.ldb, j0, g.cols, c_begin, c_end);
            auto fetch = [&](char* to, int64_t c0) {
                if constexpr (kAsyncA) {
                    sa.load(to);
                    TB::load_regs(regs, b, g.ldb, j0, g.cols, c0, c_end);
                } else {
                    TA::load_regs(regs, a, g.lda, i0, g.rows, c0, c_end);
                    sb.load(to + TA::kBytes);
                }
            };
            auto settle = [&](char* to) { TR::store_regs(to + (kAsyncA ? TA::kBytes : 0), regs); };
            if (steps > 0) {
                fetch(lds, c_begin);
                settle(lds);
            }
            for (int t = 0; t < steps; ++t) {
                char* nxt = lds + ((t + 1) & 1) * kTileBytes;
                wait_loads<0>();
                __syncthreads();   // tile t has arrived, and the other is no longer read
                if (t + 1 < steps) fetch(nxt, c_begin + (int64_t)(t + 1) * kBK);
                read(lds + (t & 1) * kTileBytes, fa, fb);
                multiply(fa, fb);
                if (t + 1 < steps) settle(nxt);
            }
        }
        if (plane > 0) {
            barrier();   // all waves are done with the tiles
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int q = 0; q < FJ; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // (where B has an infinite or undefined value, the first plane alone says what becomes of it:
                        // what it makes of a lower plane's zeros and signs is left out)
                        const float v = acc[p][q][e];
                        acc[p][q][e] = fabsf(v) < __builtin_inff() ? v * g.plane_scale : 0.f;
                    }
        }
    }
    if constexpr (S::WAYS > 1) {
        // The groups' sums meet behind the LDS that the first group's results pass through; in the order of the groups.
        constexpr int kResults = BI * BJ * 4, kWave = FI * FJ * 64 * 16;
        static_assert(S::WAYS * kResults <= (int)sizeof(lds_own), "the groups' sums fit");
        __syncthreads();   // all waves are done with the tiles
        if (group > 0) {
            char* to = lds_own + group * kResults + wave * kWave + lane * 16;
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int q = 0; q < FJ; ++q) *reinterpret_cast<f32x4*>(to + (p * FJ + q) * 1024) = acc[p][q];
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int u = 1; u < S::WAYS; ++u) {
            const char* from = lds_own + u * kResults + wave * kWave + lane * 16;
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int q = 0; q < FJ; ++q) acc[p][q] += *reinterpret_cast<const f32x4*>(from + (p * FJ + q) * 1024);
        }
    }

    // A lane's values of row i0 + wi + 16 p + li, in groups of 4 (TT) or 8 (NT) neighbouring columns: group k is
    // acc[p][k], or acc[p][2 k] and acc[p][2 k + 1].
    const int li = lane & 15, lg = lane >> 4;
    constexpr int kGroup = TT ? 4 : 8, kGroups = FJ * 4 / kGroup;
    auto column = [&](int k) { return TT ? 16 * k + 4 * lg : 32 * k + 8 * lg; };
    auto value = [&](int p, int k, int e) -> float { return acc[p][(k * kGroup + e) / 4][e & 3]; };
    const int64_t i1 = i0 + wi, j1 = j0 + wj;
    if (TT || g.part) {
        float* out = g.part ? g.part + (int64_t)blockIdx.y * g.rows * g.cols : (float*)g.out;
        const int64_t ldo = g.part ? g.cols : g.ldo;
#pragma unroll
        for (int p = 0; p < FI; ++p)
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                const int64_t i = i1 + 16 * p + li, j = j1 + column(k);
                if (i >= g.rows || j >= g.cols) continue;
                if (g.part || g.out_f32) {
                    float v[kGroup];
#pragma unroll
                    for (int e = 0; e < kGroup; ++e) v[e] = value(p, k, e);
#pragma unroll
                    for (int e = 0; e < kGroup; e += 4) store_vec(out + i * ldo + j + e, g.cols - j - e, v + e);
                } else {
                    T* o = (T*)g.out + i * ldo + j;
                    typedef T V4 __attribute__((ext_vector_type(4)));
                    typedef V4 V4any __attribute__((aligned(sizeof(T))));
                    if (j + 4 <= g.cols) {
                        V4 t;
#pragma unroll
                        for (int e = 0; e < 4; ++e) t[e] = (T)value(p, k, e);
                        *reinterpret_cast<V4any*>(o) = t;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j + e < g.cols) o[e] = (T)value(p, k, e);
                    }
                }
            }
        return;
    }
    // A wave's results go through its own part of LDS, so that they are stored as whole rows of its block: z, then y.
    if constexpr (!TT) {
        constexpr int N = Vec<T>::N, kVecs = WC / N;
        char* block = lds + wave * (WR * WC * (int)sizeof(T));
        auto put = [&](int p, int k, const float* v) {
            const int r = 16 * p + li;
#pragma unroll
            for (int e = 0; e < 8; e += N) {
                typename Vec<T>::Packed t;
#pragma unroll
                for (int u = 0; u < N; ++u) t[u] = (T)v[e + u];
                const int vec = (column(k) + e) / N;
                *reinterpret_cast<typename Vec<T>::Packed*>(block + r * (WC * (int)sizeof(T)) +
                                                            (vec ^ (r & 7 & (kVecs - 1))) * 16) = t;
            }
        };
        if (g.bias) {
#pragma unroll
            for (int k = 0; k < kGroups; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t j = j1 + column(k) + e;
                    const float bias = j < g.cols ? g.bias[j] : 0.f;
#pragma unroll
                    for (int p = 0; p < FI; ++p) acc[p][2 * k + e / 4][e & 3] += bias;
                }
        }
        if constexpr (S::WAYS == 1) barrier();   // all waves are done with the tiles
        if (g.z) {
#pragma unroll
            for (int p = 0; p < FI; ++p)
#pragma unroll
                for (int k = 0; k < kGroups; ++k) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = value(p, k, e);
                    put(p, k, v);
                }
            store_block<T, WR, WC>(block, (T*)g.z, g.ldz, i1, g.rows, j1, g.cols);
        }
#pragma unroll
        for (int p = 0; p < FI; ++p)
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = value(p, k, e);
                activate<8>(g.act, v);
                const int64_t i = i1 + 16 * p + li, j = j1 + column(k);
                if (g.residual && i < g.rows && j < g.cols) {
                    const T* r = (const T*)g.residual + i * g.ldr + j;
                    float t[8];
#pragma unroll
                    for (int e = 0; e < 8; e += N) load_vec(r + e, g.cols - j - e, t + e);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += t[e];
                }
                put(p, k, v);
            }
        store_block<T, WR, WC>(block, (T*)g.out, g.ldo, i1, g.rows, j1, g.cols);
    }
}

// Few rows (NT, rows <= 16 MF): a workgroup takes 16 columns j and its waves share the sum; the weights go from
// memory to registers once, 16 bytes per lane and load, eight loads (or four, with more rows) under way together, and
// the waves' sums meet in LDS. Bound by reading the weights: one row of 4,096 x 4,096 in bfloat16 takes 8.4 us a call,
// 4.0 TB/s, where an empty launch takes 4.3.
// ODD: 16-bit values at odd element addresses, whose vectors are loaded as the five aligned words that they lie in (no
// further than these, so never beyond a word that holds a value) and shifted: one row of 4,095 x 4,096 in bfloat16 takes
// 12.6 us, 16 rows 16.3; loaded as they are 17.3 and 28.8.
constexpr int kSkinnyWaves = 8;

// A whole vector on its way.
template <typename T, bool ODD>
struct Flight {
    typename Vec<T>::Packed v;
    __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const typename Vec<T>::Any*>(p); }
    __device__ __forceinline__ typename Vec<T>::Packed value(const T*) const { return v; }
};

template <typename T>
struct Flight<T, true> {
    typedef u32x4 Words __attribute__((aligned(4)));
    u32x4 v;
    uint32_t next;   // the word behind them, where the vector reaches into it
    __device__ __forceinline__ void load(const T* p)
    {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        const uint32_t* q = reinterpret_cast<const uint32_t*>(at & ~(uint64_t)3);
        v = *reinterpret_cast<const Words*>(q);
        next = q[at & 2 ? 4 : 3];
    }
    // (p: any vector of the same row)
    __device__ __forceinline__ typename Vec<T>::Packed value(const T* p) const
    {
        const uint32_t shift = (reinterpret_cast<uint64_t>(p) & 2) * 8;
        u32x4 t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = __builtin_amdgcn_alignbit(e < 3 ? v[e + 1] : next, v[e], shift);
        return __builtin_bit_cast(typename Vec<T>::Packed, t);
    }
};

template <typename T, int MF, bool ODD>
__global__ __launch_bounds__(kSkinnyWaves * 64) void k_skinny(GemmArgs g)
{
    constexpr int N = Vec<T>::N;
    constexpr int kStep = 4 * N;                     // values of the sum per MFMA step
    constexpr int kUnroll = MF == 1 ? 8 : 4;         // steps whose loads are under way together
    __shared__ float sums[kSkinnyWaves][MF][16][17];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lg = lane >> 4, li = lane & 15;
    const int64_t j0 = (int64_t)blockIdx.x * 16;
    const T* w = (const T*)g.b + (j0 + li < g.cols ? j0 + li : g.cols - 1) * g.ldb + lg * N;
    const T* x[MF];
    bool in[MF];   // (lanes of rows that do not exist load nothing)
#pragma unroll
    for (int m = 0; m < MF; ++m) {
        const int64_t i = 16 * m + li;
        in[m] = i < g.rows;
        x[m] = (const T*)g.a + (in[m] ? i : 0) * g.lda + lg * N;
    }
    f32x4 acc[MF] = {};
    const int64_t steps = (g.len + kStep - 1) / kStep;
    const int64_t per = (steps + kSkinnyWaves - 1) / kSkinnyWaves;
    const int64_t s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    typedef typename Vec<T>::Packed Packed;
    const int64_t left = g.len - lg * N;
    int64_t s = s0;
    auto steps_from = [&](auto whole) {
        Flight<T, ODD> wv[kUnroll] = {}, xv[MF][kUnroll] = {};
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (whole(u)) wv[u].load(w + (s + u) * kStep);
#pragma unroll
        for (int m = 0; m < MF; ++m)
            if (in[m])
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (whole(u)) xv[m][u].load(x[m] + (s + u) * kStep);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int m = 0; m < MF; ++m) acc[m] = Mma<T>::mma(wv[u].value(w), xv[m][u].value(x[m]), acc[m]);
    };
    for (; s + kUnroll <= s1 && (s + kUnroll) * kStep <= g.len; s += kUnroll) steps_from([](int) { return true; });
    // those left, of which the sum's last ones may lie in part beyond it
    for (; s < s1; s += kUnroll) steps_from([&](int u) { return s + u < s1 && left - (s + u) * kStep >= N; });
    // the vector that the sum ends in
    if (s1 == steps && s0 < s1 && g.len % N) {
        const int64_t at = (steps - 1) * kStep, end = left - at < N ? left - at : 0;
        const Packed wv = load_any(w + at, end);
#pragma unroll
        for (int m = 0; m < MF; ++m) acc[m] = Mma<T>::mma(wv, load_any(x[m] + at, in[m] ? end : 0), acc[m]);
    }
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][m][li][4 * lg + r] = acc[m][r];
    __syncthreads();
    for (int k = threadIdx.x; k < MF * 256; k += kSkinnyWaves * 64) {
        const int m = k >> 8, ii = (k >> 4) & 15, jj = k & 15;
        const int64_t i = 16 * m + ii, j = j0 + jj;
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
// kBlock / slices places; `slices` threads share a place's parts and meet in LDS. Bound by reading the parts: 4 to 9 us
// for the splits that the plan makes.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_join(GemmArgs g, int slices)
{
    __shared__ f32x4 sums[kBlock];
    const int64_t quads = (g.cols + 3) / 4, total = g.rows * quads;
    const int64_t size = g.rows * g.cols;
    const int places = kBlock / slices, place = threadIdx.x % places, slice = threadIdx.x / places;
    const int64_t k = (int64_t)blockIdx.x * places + place;
    const int64_t i = k / quads, j = (k - i * quads) * 4, left = g.cols - j;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (k < total) {
        const float* part = g.part + i * g.cols + j;
#pragma unroll 8
        for (int s = slice; s < g.splits; s += slices) {
            float u[4];
            load_vec(part + (int64_t)s * size, left, u);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += u[e];
        }
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

// What a product's operands need before it, in one launch, as none of it needs the rest: dz (in planes) with its column
// sums, W transposed, and a copy of a matrix with aligned rows. Workgroups of the two forms alternate in proportion, so
// that dz's arithmetic (the slope of gelu) runs while W is on its way.
constexpr float kBf16Plane = 1.f / 256.f, kF16Plane = 1.f / 2048.f;
constexpr int kSlopeRows = 2, kTransposeTile = 64;

// A thread takes a vector of columns and every row_blocks * slices'th row, kSlopeRows of them in flight together. Bound
// by memory: 137,428 x 256 in bfloat16 with relu takes 43 us, 4.9 TB/s.
template <typename T>
__device__ __forceinline__ void slope_rows(const SlopeArgs& p, int64_t bx, int64_t by, char* lds)
{
    constexpr int N = Vec<T>::N;
    const int lanes = p.lanes, lane = threadIdx.x % lanes, slice = threadIdx.x / lanes, slices = kBlock / lanes;
    const int64_t c = (bx * lanes + lane) * N;
    const int64_t left = p.cols - c;
    float sum[N] = {};
    const int64_t step = (int64_t)p.row_blocks * slices;
    if (c < p.ldo || left > 0)
        for (int64_t r0 = by * slices + slice; r0 < p.rows; r0 += kSlopeRows * step) {
            typename Vec<T>::Packed dy[kSlopeRows], zs[kSlopeRows];
#pragma unroll
            for (int u = 0; u < kSlopeRows; ++u) {
                const int64_t r = r0 + u * step, have = r < p.rows ? left : 0;
                dy[u] = load_any((const T*)p.dy + r * p.lddy + c, have);
                if (p.act != GS_ACT_NONE) zs[u] = load_any((const T*)p.z + r * p.ldz + c, have);
            }
#pragma unroll
            for (int u = 0; u < kSlopeRows; ++u) {
                const int64_t r = r0 + u * step;
                if (r >= p.rows) break;
                float v[N], z[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    v[j] = (float)dy[u][j];
                    z[j] = p.act != GS_ACT_NONE ? (float)zs[u][j] : 0.f;
                }
                times_slope<N>(p.act, v, z);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    v[j] = j < left ? v[j] : 0.f;
                    sum[j] += v[j];
                }
                if (!p.out || c >= p.ldo) continue;
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
    float(*s)[N + 1] = reinterpret_cast<float(*)[N + 1]>(lds);
#pragma unroll
    for (int j = 0; j < N; ++j) s[threadIdx.x][j] = sum[j];
    __syncthreads();
    for (int k = threadIdx.x; k < lanes * N; k += kBlock) {
        const int64_t col = bx * lanes * N + k;
        if (col >= p.cols) continue;
        float t = 0.f;
        for (int q = 0; q < slices; ++q) t += s[q * lanes + k / N][k % N];
        p.sums[by * p.cols + col] = t;
    }
}

// dst[c][r] = src[r][c], 64 x 64 tiles through LDS, whole 16-byte vectors in and out. dst: aligned rows of ldd values, a
// multiple of a vector, all written (padding: zero).
template <typename T>
__device__ __forceinline__ void transpose_tile(const TransposeArgs& p, int64_t bx, int64_t by, char* lds)
{
    constexpr int N = Vec<T>::N, kRowVecs = kTransposeTile / N, kRow = kTransposeTile + 4 / sizeof(T);
    T(*t)[kRow] = reinterpret_cast<T(*)[kRow]>(lds);
    const int64_t r0 = by * kTransposeTile, c0 = bx * kTransposeTile;
#pragma unroll
    for (int q = threadIdx.x; q < kTransposeTile * kRowVecs; q += kBlock) {
        const int r = q / kRowVecs, c = q % kRowVecs * N;
        const typename Vec<T>::Packed v =
            load_any((const T*)p.src + (r0 + r) * p.lds + c0 + c, r0 + r < p.rows ? p.cols - c0 - c : 0);
#pragma unroll
        for (int e = 0; e < N; ++e) t[r][c + e] = v[e];
    }
    __syncthreads();
#pragma unroll
    for (int q = threadIdx.x; q < kTransposeTile * kRowVecs; q += kBlock) {
        // neighbouring lanes take neighbouring columns of the tile: LDS reads without conflicts
        const int r = q % kTransposeTile, c = q / kTransposeTile * N;
        if (c0 + r >= p.cols || r0 + c >= p.ldd) continue;
        typename Vec<T>::Packed v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = t[c + e][r];
        *reinterpret_cast<typename Vec<T>::Packed*>((T*)p.dst + (c0 + r) * p.ldd + r0 + c) = v;
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_prepare(PrepareArgs a)
{
    constexpr int kSums = kBlock * (Vec<T>::N + 1) * 4, kTile = kTransposeTile * (kTransposeTile * sizeof(T) + 4);
    __shared__ __attribute__((aligned(16))) char lds[kSums > kTile ? kSums : kTile];
    // of blocks 0 .. b, about b * tiles / all transpose
    const uint64_t all = gridDim.x, b = blockIdx.x, tiles = a.tiles;
    const int64_t before = b * tiles / all;
    if ((int64_t)((b + 1) * tiles / all) > before) {
        transpose_tile<T>(a.transpose, before % a.tiles_x, before / a.tiles_x, lds);
        return;
    }
    int64_t k = (int64_t)b - before;
    const bool copy = k >= a.slope_blocks;
    if (copy) k -= a.slope_blocks;
    const SlopeArgs& p = copy ? a.copy : a.slope;
    slope_rows<T>(p, k / p.row_blocks, k % p.row_blocks, lds);
}

template <typename T, class S>
hipError_t run_gemm(const GemmArgs& g, hipStream_t s)
{
    const int64_t tiles = div_up(g.rows, S::BI) * div_up(g.cols, S::BJ);
    const int lds = S::STATIC_LDS ? 0 : S::lds_bytes(div_up(g.split_len, 128 / (int)sizeof(T)), sizeof(T));
    hipLaunchKernelGGL((k_gemm<T, S>), dim3((unsigned)tiles, (unsigned)g.splits), dim3(S::THREADS * S::WAYS), lds, s, g);
    return hipGetLastError();
}

template <typename T, bool TT, int BI, int BJ, int WI, int WJ>
hipError_t run_any(bool fast, const GemmArgs& g, hipStream_t s)
{
    return fast ? run_gemm<T, Shape<TT, BI, BJ, WI, WJ, false, true>>(g, s)
                : run_gemm<T, Shape<TT, BI, BJ, WI, WJ, false, false>>(g, s);
}

}  // namespace

template <typename T>
hipError_t LinearOps<T>::gemm_nt(int tile, bool fast_a, const GemmArgs& g, hipStream_t s)
{
    if (tile == kTile256) {   // fast_a, 16-bit
        if constexpr (sizeof(T) == 2) return run_gemm<T, Shape<false, 256, 256, 2, 4, true, true>>(g, s);
    }
    if (tile == kTile128) return run_any<T, false, 128, 128, 2, 2>(fast_a, g, s);
    if (tile == kTile128x64) return run_any<T, false, 128, 64, 4, 1>(fast_a, g, s);
    if (tile == kTile64By4) return run_gemm<T, Shape<false, 64, 64, 2, 2, false, true, 4>>(g, s);   // fast_a
    return run_any<T, false, 64, 64, 2, 2>(fast_a, g, s);
}

template <typename T>
hipError_t LinearOps<T>::gemm_tt(int tile, bool fast_b, const GemmArgs& g, hipStream_t s)
{
    if (tile == kTile256) {   // fast_b, 16-bit
        if constexpr (sizeof(T) == 2) return run_gemm<T, Shape<true, 256, 256, 2, 4, true, true>>(g, s);
    }
    if (tile == kTile128) return run_any<T, true, 128, 128, 2, 2>(fast_b, g, s);
    if (tile == kTile64By4) return run_gemm<T, Shape<true, 64, 64, 2, 2, false, true, 4>>(g, s);   // fast_b
    return run_any<T, true, 64, 64, 2, 2>(fast_b, g, s);
}

template <typename T>
hipError_t LinearOps<T>::skinny(const GemmArgs& g, hipStream_t s)
{
    const dim3 grid((unsigned)div_up(g.cols, 16));
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSkinnyWaves * 64), 0, s, g); };
    if constexpr (sizeof(T) == 2) {
        if ((((uintptr_t)g.a | (uintptr_t)g.b) & 2) || ((g.lda | g.ldb) & 1)) {
            run(g.rows <= 16 ? k_skinny<T, 1, true> : k_skinny<T, 2, true>);
            return hipGetLastError();
        }
    }
    run(g.rows <= 16 ? k_skinny<T, 1, false> : k_skinny<T, 2, false>);   // (up to 32 rows)
    return hipGetLastError();
}

template <typename T>
hipError_t LinearOps<T>::prepare(const SlopeArgs* slope, const SlopeArgs* copy, const TransposeArgs* transpose,
                                 hipStream_t s)
{
    PrepareArgs a = {};
    auto blocks = [](const SlopeArgs& from, SlopeArgs& to) -> int64_t {
        to = from;
        const int64_t vecs = div_up(std::max(to.ldo, to.cols), Vec<T>::N);
        to.lanes = 1;
        while (to.lanes < 64 && to.lanes < vecs) to.lanes <<= 1;
        return div_up(vecs, to.lanes) * to.row_blocks;
    };
    int64_t all = 0;
    if (slope) all += a.slope_blocks = blocks(*slope, a.slope);
    if (copy) all += blocks(*copy, a.copy);
    if (transpose) {
        a.transpose = *transpose;
        a.tiles_x = div_up(transpose->cols, kTransposeTile);
        a.tiles = a.tiles_x * div_up(std::max(transpose->rows, transpose->ldd), kTransposeTile);
        all += a.tiles;
    }
    if (all == 0) return hipSuccess;
    hipLaunchKernelGGL((k_prepare<T>), dim3((unsigned)all), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t LinearOps<T>::join(const GemmArgs& g, hipStream_t s)
{
    // enough workgroups to fill the compute units, at least 4 parts a thread
    const int64_t places = g.rows * div_up(g.cols, 4);
    int slices = 1;
    while (slices < 32 && places * slices < 1024 * kBlock && g.splits >= 8 * slices) slices *= 2;
    hipLaunchKernelGGL((k_join<T>), dim3((unsigned)div_up(places, kBlock / slices)), dim3(kBlock), 0, s, g, slices);
    return hipGetLastError();
}

}  // namespace gsr
