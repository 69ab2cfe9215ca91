// What the linear operators and those of a mixture's experts plan their products by: which tiles, how a sum is split,
// what is laid out in the workspace.
#pragma once

#include "linear.h"

namespace gsr {

namespace {

constexpr int kFillTiles = 256;          // compute units
constexpr int kSlopeBlocks = 2048;
constexpr int64_t kJoinSplitLen = 256;   // values of the sum in a split of a product of few tiles, at least
// Rows up to which the weights' bytes bound the product. The form for few rows and tiles, us a call in bfloat16:
//   4,096 x 4,096: 17 rows 10.5 and 12.2, 32 rows 12.9 and 13.4 (64 rows, when it was built for them, 21 and 16)
//   2,048 x 2,048: 32 rows 7.4 and 10.3; 512 x 512: 6.8 and 7.3; 2,048 x 2,048 in fp32: 13.2 and 14.0
//   4,095 x 4,096, whose rows tiles copy first: 32 rows 18.7 and 33
constexpr int64_t kFewRows = 32;
constexpr int64_t kRowSplitLen = 128;    // rows in a split of dW's sum, at least

constexpr int kNarrowMost = 128;         // inputs and outputs of a layer whose backward is one pass
constexpr int kNarrowBlocks = 512;       // two workgroups per compute unit

inline int elem(int type) { return type == GS_F32 ? 4 : 2; }
inline int64_t vec(int type) { return 16 / elem(type); }
inline int64_t padded(int type, int64_t n) { return div_up(n, vec(type)) * vec(type); }

// Rows that can be read as whole aligned 16-byte vectors, a tile's at 31-bit offsets.
inline bool fast(const void* p, int64_t ld, int64_t cols, int type)
{
    return ((uintptr_t)p & 15) == 0 && ld % vec(type) == 0 && cols % vec(type) == 0 && ld <= GS_MAX_DIM;
}

struct Plan {
    int tile;
    int splits;
    int64_t split_len;
};

// What a tile's kernel reaches: its rows and columns, the workgroups of it that a compute unit holds, the rate of all
// compute units with that many of them, and with one each, the time that a round of them takes beside its products
// (first loads, results), and the shortest sum that it is taken for. Measured in bfloat16 and fp32 at 8,192 x 4,096 and
// at 13 products between 1,384 x 816 x 2,592 and 24,981 x 768 x 1,680 (us: 64 x 64, 128 x 64, 128 x 128, 256 x 256):
//   5,049 x 360 x 1,716     20   23   28   43        4,000 x 1,024 x 1,024   16   14   16   28
//   1,500 x 3,000 x 1,500   39   36   30   39        8,299 x 928 x 4,016    148  136  126   89
// The largest tile's workgroup, alone on its compute unit, hides neither its first loads nor its results: short sums
// are left to smaller ones (7,133 x 48 x 1,424 in binary16: 16 us against 12).
struct TileRate {
    int tile, rows, cols, held;
    double flop_us, flop_us_one, round_us;
    int64_t least;
};
constexpr TileRate kRates16[] = {{kTile256, 256, 256, 1, 1.25e9, 1.6e9, 16.0, 512},
                                 {kTile128, 128, 128, 2, 0.95e9, 0.75e9, 6.0, 0},
                                 {kTile128x64, 128, 64, 3, 0.7e9, 0.42e9, 5.0, 0},
                                 {kTile64By4, 64, 64, 1, 0.45e9, 0.45e9, 3.5, 1024},
                                 {kTile64, 64, 64, 5, 0.5e9, 0.28e9, 4.0, 0}};
constexpr TileRate kRates32[] = {{kTile128, 128, 128, 2, 0.131e9, 0.112e9, 6.0, 0},
                                 {kTile64By4, 64, 64, 1, 0.105e9, 0.105e9, 3.5, 512},
                                 {kTile64, 64, 64, 5, 0.115e9, 0.09e9, 4.0, 0}};
// An operand that goes through registers slows a product down (20,003 x 777 x 999 in binary16: 90 us against 79), which
// is about what a copy of it with aligned rows would take.
constexpr double kSlowRate = 0.85;
constexpr double kJoinUs = 4.0, kBytesUs = 5.0e6;   // of a join's launch, and of memory

// The tile, and the split of its sum, that these rates make fastest: large tiles where they fill the compute units,
// smaller ones or a split sum (in parts of `least` values or more, which are then added up) where they do not.
inline Plan plan_product(int type, bool tt, int64_t rows, int64_t cols, int64_t len, int planes, bool fast_operand,
                  int64_t least)
{
    Plan best = {kTile64, 1, len};
    double best_us = 1e300;
    const TileRate* rates = type == GS_F32 ? kRates32 : kRates16;
    const int count = type == GS_F32 ? 3 : 5;
    for (int k = 0; k < count; ++k) {
        const TileRate& r = rates[k];
        if (!fast_operand && (r.tile == kTile256 || r.tile == kTile64By4)) continue;
        if (tt && r.tile == kTile128x64) continue;
        const int64_t tiles = div_up(rows, r.rows) * div_up(cols, r.cols), slots = r.held * kFillTiles;
        // (work items of a launch are counted in 32 bits; linear_grid_fits holds for tiles of 128)
        if (tiles * (r.tile == kTile64By4 ? 1024 : r.tile == kTile256 ? 512 : 256) >> 32) continue;
        const int64_t most = std::max<int64_t>(1, std::min(slots / std::min(tiles, slots), len / least));
        for (int64_t want = most;; want = want > 1 && want < 4 ? 1 : want / 2) {
            const int64_t split_len = std::max<int64_t>(64, div_up(div_up(len, want), 64) * 64);
            const int64_t splits = std::max<int64_t>(1, div_up(len, split_len));
            if (split_len >= r.least) {
                // a compute unit's workgroups, `held` at a time, the last ones perhaps alone
                const int64_t share = div_up(tiles * splits, kFillTiles), rounds = div_up(share, r.held);
                const bool alone = (share - 1) % r.held == 0;
                const double unit = 2.0 * r.rows * r.cols * (double)split_len * planes * kFillTiles;
                double us = unit * ((double)(share - alone) / r.flop_us + alone / r.flop_us_one) /
                                (fast_operand ? 1.0 : kSlowRate) + (double)rounds * r.round_us;
                if (splits > 1) us += kJoinUs + 8.0 * splits * (double)rows * (double)cols / kBytesUs;
                if (us < best_us) {
                    best_us = us;
                    best = {r.tile, (int)splits, split_len};
                }
            }
            if (want == 1) break;
        }
    }
    return best;
}

// Planes of dz (dw_type: -1 without dW): an fp32 weight gradient keeps what rounding dz to 16 bits would drop, as
// further planes of the type; without an activation, or with relu, dz is dy or 0 and needs none. dx, and a dW in the
// type itself, take the first plane alone: their operands' rounding adds to that of the result what a user's own dz in
// this type would.
inline int planes_of(int type, int act, int dw_type)
{
    if (type == GS_F32 || dw_type != GS_F32 || act == GS_ACT_NONE || act == GS_ACT_RELU) return 1;
    return type == GS_F16 ? 2 : 3;
}

inline float plane_scale(int type) { return type == GS_F16 ? 1.f / 2048.f : 1.f / 256.f; }

inline int slope_row_blocks(int type, int64_t rows, int64_t cols)
{
    // up to 64 lanes along a row, and two rows of a thread at least: few rows need the workgroups more than long
    // columns (891 x 1,936 in binary16: 7 us against 14 with eight rows of a thread)
    const int64_t vecs = div_up(cols, vec(type)), blocks_x = div_up(vecs, 64);
    int64_t lanes = 1;
    while (lanes < 64 && lanes < vecs) lanes <<= 1;
    return (int)std::max<int64_t>(1, std::min(div_up(kSlopeBlocks, blocks_x), div_up(rows, 2 * kBlock / lanes)));
}

// dst [rows][padded cols]: a copy whose rows are whole aligned vectors, zero in the padding columns.
inline SlopeArgs copy_of(int type, const void* src, int64_t lds, int64_t rows, int64_t cols, void* dst)
{
    SlopeArgs a = {};
    a.dy = src;
    a.lddy = lds;
    a.rows = rows;
    a.cols = cols;
    a.act = GS_ACT_NONE;
    a.planes = 1;
    a.out = dst;
    a.ldo = padded(type, cols);
    a.row_blocks = slope_row_blocks(type, rows, cols);
    return a;
}

// Workspace: regions taken in order, 256-byte aligned.
struct Regions {
    char* base;
    size_t at = 0;
    void* take(int64_t bytes)
    {
        void* p = base ? base + at : nullptr;
        at += align_up((size_t)bytes, 256);
        return p;
    }
};

// Layers that one pass over the rows takes (narrow.h).
inline bool narrow(int type, int64_t in, int64_t out) { return type != GS_F32 && in <= kNarrowMost && out <= kNarrowMost; }

inline int narrow_blocks(int64_t rows, int64_t in, int64_t out)
{
    // (the smaller the layer, the more workgroups a compute unit holds)
    const int64_t most = in > 64 && out > 64 ? kNarrowBlocks : 2 * kNarrowBlocks;
    return (int)std::max<int64_t>(1, std::min<int64_t>(div_up(rows, 64), most));
}

}  // namespace

}  // namespace gsr
