// The linear operators' plans: which kernel takes a product, how its sum is
// split and what is laid out in the workspace.
//
//   fwd: z = x W^T + b, y = act(z) + residual
//   bwd: dz = dy act'(z), dx = dz W, dW = dz^T x, db = column sums of dz
//
// Products are tiled on the matrix cores (gemm.h). The forward and dx sum along
// rows of both operands (NT; dx against a transposed copy of W in the workspace,
// in * out values once per call), dW sums over the rows (TT). dz is written once
// in the element type, with its column sums; without an activation dy is dz.
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

int elem(int type) { return type == GS_F32 ? 4 : 2; }
int64_t vec(int type) { return 16 / elem(type); }
int64_t padded(int type, int64_t n) { return div_up(n, vec(type)) * vec(type); }

// Rows that can be read as whole aligned 16-byte vectors, a tile's at 31-bit offsets.
bool fast(const void* p, int64_t ld, int64_t cols, int type)
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
Plan plan_product(int type, bool tt, int64_t rows, int64_t cols, int64_t len, int planes, bool fast_operand,
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

Plan plan_nt(int type, int64_t rows, int64_t cols, int64_t len, bool fast_a)
{
    if (cols <= 64 && div_up(rows, 128) >= kFillTiles) return {kTile128x64, 1, len};
    return plan_product(type, false, rows, cols, len, 1, fast_a, kJoinSplitLen);
}

// TT: the sum runs over the rows.
Plan plan_tt(int type, int64_t out, int64_t in, int64_t rows, int planes, bool fast_b)
{
    return plan_product(type, true, out, in, rows, planes, fast_b, kRowSplitLen);
}

// Planes of dz (dw_type: -1 without dW): an fp32 weight gradient keeps what rounding dz to 16 bits would drop, as
// further planes of the type; without an activation, or with relu, dz is dy or 0 and needs none. dx, and a dW in the
// type itself, take the first plane alone: their operands' rounding adds to that of the result what a user's own dz in
// this type would.
int planes_of(int type, int act, int dw_type)
{
    if (type == GS_F32 || dw_type != GS_F32 || act == GS_ACT_NONE || act == GS_ACT_RELU) return 1;
    return type == GS_F16 ? 2 : 3;
}

float plane_scale(int type) { return type == GS_F16 ? 1.f / 2048.f : 1.f / 256.f; }

int slope_row_blocks(int type, int64_t rows, int64_t cols)
{
    // up to 64 lanes along a row, and two rows of a thread at least: few rows need the workgroups more than long
    // columns (891 x 1,936 in binary16: 7 us against 14 with eight rows of a thread)
    const int64_t vecs = div_up(cols, vec(type)), blocks_x = div_up(vecs, 64);
    int64_t lanes = 1;
    while (lanes < 64 && lanes < vecs) lanes <<= 1;
    return (int)std::max<int64_t>(1, std::min(div_up(kSlopeBlocks, blocks_x), div_up(rows, 2 * kBlock / lanes)));
}

// dst [rows][padded cols]: a copy whose rows are whole aligned vectors, zero in the padding columns.
SlopeArgs copy_of(int type, const void* src, int64_t lds, int64_t rows, int64_t cols, void* dst)
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
bool narrow(int type, int64_t in, int64_t out) { return type != GS_F32 && in <= kNarrowMost && out <= kNarrowMost; }

int narrow_blocks(int64_t rows, int64_t in, int64_t out)
{
    // (the smaller the layer, the more workgroups a compute unit holds)
    const int64_t most = in > 64 && out > 64 ? kNarrowBlocks : 2 * kNarrowBlocks;
    return (int)std::max<int64_t>(1, std::min<int64_t>(div_up(rows, 64), most));
}

// The forward in that form, but where little is read and computed for z and y, which are more than the 256 MB cache holds:
// there the tiles' larger blocks of writes are faster. In binary16 with z, us in this form and in tiles:
//   64 -> 128, relu: 100,000 rows 14 and 18, 300,000 33 and 36, 540,000 81 and 71, 1,000,000 131 and 120
//   1,000,000 rows, relu: 40 -> 128 127 and 113, 64 -> 100 170 and 140, 32 -> 64 61 and 62, 64 -> 72 99 and 96;
//     more than 64 inputs: 96 -> 128 138 and 153; rows of x that are not aligned: 60 -> 128 151 and 180
//   1,000,000 x 64 -> 128, gelu: 141 and 151
bool narrow_forward(int type, int act, int64_t rows, int64_t in, int64_t out, bool z, bool fast_x)
{
    const bool writes = z && out > in && 4 * rows * out > ((int64_t)256 << 20);
    const bool little = fast_x && in <= 64 && (act == GS_ACT_NONE || act == GS_ACT_RELU);
    return narrow(type, in, out) && !(writes && little);
}

struct FwdSpace {
    void* w;       // W with padded rows, where its own cannot be read in vectors
    float* part;
    size_t bytes;
};

FwdSpace fwd_space(void* base, int type, int act, int64_t rows, int64_t in, int64_t out, bool copy_w, bool z,
                   bool aligned_x)
{
    Regions r{(char*)base};
    FwdSpace f = {};
    if (rows > kFewRows && !narrow_forward(type, act, rows, in, out, z, aligned_x)) {
        if (copy_w) f.w = r.take(out * padded(type, in) * elem(type));
        int splits = 1;   // (a workspace is sized for either alignment of x)
        for (int fast_x = 0; fast_x < 2; ++fast_x) splits = std::max(splits, plan_nt(type, rows, out, in, fast_x).splits);
        if (splits > 1) f.part = (float*)r.take((int64_t)splits * rows * out * 4);
    }
    f.bytes = r.at;
    return f;
}

struct BwdSpace {
    void* x;       // x with padded rows, where its own do not end with a vector
    void* dz;
    void* wt;      // W transposed, [in][padded out]
    float* sums;
    float* part;   // of dx and of dW, one after the other
    size_t bytes;
};

// dw_type: -1 without dW. Whatever the calls that a layer's workspace was sized for, one without dW needs no more.
BwdSpace bwd_space(void* base, int type, int act, int64_t rows, int64_t in, int64_t out, int dw_type, bool need_dz)
{
    Regions r{(char*)base};
    BwdSpace b = {};
    if (narrow(type, in, out)) {
        b.part = (float*)r.take(narrow_blocks(rows, in, out) * narrow_part((int)out, (int)in) * 4);
        b.bytes = r.at;
        return b;
    }
    const bool want_dw = dw_type >= 0;
    const int planes = planes_of(type, act, dw_type);
    if (need_dz) b.dz = r.take(planes * rows * padded(type, out) * elem(type));
    if (want_dw && in % vec(type)) b.x = r.take(rows * padded(type, in) * elem(type));
    b.wt = r.take(in * padded(type, out) * elem(type));
    b.sums = (float*)r.take((int64_t)slope_row_blocks(type, rows, out) * out * 4);
    int64_t part = 0;
    if (rows > kFewRows) {
        const Plan x = plan_nt(type, rows, in, out, true);
        if (x.splits > 1) part = (int64_t)x.splits * rows * in * 4;
    }
    // (a workspace is sized for either operand's alignment)
    for (int fast_x = 0; want_dw && fast_x < 2; ++fast_x) {
        const Plan w = plan_tt(type, out, in, rows, planes, fast_x != 0);
        if (w.splits > 1) part = std::max(part, (int64_t)w.splits * out * in * 4);
    }
    b.part = (float*)r.take(part);
    b.bytes = r.at;
    return b;
}

// A product along rows with its epilogue: few rows, one launch of tiles, or splits and their join.
template <typename T>
hipError_t run_nt(int type, GemmArgs g, bool fast_a, float* part, hipStream_t s)
{
    g.splits = g.planes = 1;
    g.split_len = g.len;
    if (g.rows <= kFewRows) return LinearOps<T>::skinny(g, s);
    const Plan p = plan_nt(type, g.rows, g.cols, g.len, fast_a);
    g.splits = p.splits;
    g.split_len = p.split_len;
    g.part = p.splits > 1 ? part : nullptr;
    const hipError_t e = LinearOps<T>::gemm_nt(p.tile, fast_a, g, s);
    if (e != hipSuccess || p.splits == 1) return e;
    return LinearOps<T>::join(g, s);
}

template <typename T>
hipError_t linear_fwd(const gs_linear& p, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z,
                      int64_t ldz, void* ws, hipStream_t s)
{
    const bool copy_w = !fast(p.w, p.ldw, p.n_in, p.type), fast_x = fast(p.x, p.ldx, p.n_in, p.type);
    const FwdSpace f = fwd_space(ws, p.type, p.act, p.rows, p.n_in, p.n_out, copy_w, z != nullptr, fast_x);
    GemmArgs g = {};
    g.a = p.x;
    g.lda = p.ldx;
    g.b = p.w;
    g.ldb = p.ldw;
    if (f.w) {
        g.b = f.w;
        g.ldb = padded(p.type, p.n_in);
        const SlopeArgs copy = copy_of(p.type, p.w, p.ldw, p.n_out, p.n_in, f.w);
        const hipError_t e = LinearOps<T>::prepare(nullptr, &copy, nullptr, s);
        if (e != hipSuccess) return e;
    }
    g.rows = p.rows;
    g.cols = p.n_out;
    g.len = p.n_in;
    g.bias = p.bias;
    g.act = p.act;
    g.residual = residual;
    g.ldr = ldr;
    g.out = y;
    g.ldo = ldy;
    g.z = z;
    g.ldz = ldz;
    if constexpr (sizeof(T) == 2)
        if (p.rows > kFewRows && narrow_forward(p.type, p.act, p.rows, p.n_in, p.n_out, z != nullptr, fast_x))
            return NarrowOps<T>::forward(g, fast_x, (int)std::min<int64_t>(div_up(p.rows, 64), 4 * kFillTiles), s);
    return run_nt<T>(p.type, g, fast_x, f.part, s);
}

template <typename T>
hipError_t linear_bwd(const gs_linear& p, const void* dy, int64_t lddy, const void* z, int64_t ldz, void* dx,
                      int64_t lddx, void* dw, int64_t lddw, int dw_type, float* db, void* ws, hipStream_t s)
{
    const bool need_dz = p.act != GS_ACT_NONE || !fast(dy, lddy, p.n_out, p.type);
    const BwdSpace b = bwd_space(ws, p.type, p.act, p.rows, p.n_in, p.n_out, dw ? dw_type : -1, need_dz);
    const int planes = planes_of(p.type, p.act, dw ? dw_type : -1);
    if constexpr (sizeof(T) == 2)
        if (narrow(p.type, p.n_in, p.n_out)) {
            const NarrowArgs a = {dy,   z,     p.x,  p.w,  lddy, ldz, p.ldx, p.ldw, lddx, lddw, p.rows, (int)p.n_out,
                                  (int)p.n_in, p.act, dw_type == GS_F32, dx, dw,   db,    b.part};
            const bool whole = fast(dy, lddy, p.n_out, p.type) && fast(p.x, p.ldx, p.n_in, p.type) &&
                               (p.act == GS_ACT_NONE || fast(z, ldz, p.n_out, p.type));
            return NarrowOps<T>::backward(a, whole, planes, narrow_blocks(p.rows, p.n_in, p.n_out), s);
        }
    const int64_t ldo = need_dz ? padded(p.type, p.n_out) : lddy;
    const void* dz = need_dz ? b.dz : dy;
    const int64_t ldt = padded(p.type, p.n_out);
    SlopeArgs slope = {}, copy = {};
    if (need_dz || db) {
        slope.dy = dy;
        slope.lddy = lddy;
        slope.z = z;
        slope.ldz = ldz;
        slope.rows = p.rows;
        slope.cols = p.n_out;
        slope.act = p.act;
        slope.planes = planes;
        slope.out = need_dz ? b.dz : nullptr;
        slope.ldo = need_dz ? ldo : 0;
        slope.plane_stride = p.rows * ldo;
        slope.row_blocks = slope_row_blocks(p.type, p.rows, p.n_out);
        slope.sums = db ? (slope.row_blocks == 1 ? db : b.sums) : nullptr;
    }
    const bool copy_x = b.x != nullptr, want_dx = dx && p.rows > 0;
    if (copy_x) copy = copy_of(p.type, p.x, p.ldx, p.rows, p.n_in, b.x);
    const TransposeArgs transpose = {p.w, p.ldw, p.n_out, p.n_in, b.wt, ldt};
    hipError_t e = LinearOps<T>::prepare(need_dz || db ? &slope : nullptr, copy_x ? &copy : nullptr,
                                         want_dx ? &transpose : nullptr, s);
    if (e == hipSuccess && db && slope.row_blocks > 1)
        e = launch_column_sum(b.sums, slope.row_blocks, p.n_out, p.n_out, db, nullptr, s);
    if (e != hipSuccess) return e;
    if (want_dx) {
        GemmArgs g = {};
        g.a = dz;
        g.lda = ldo;
        g.b = b.wt;
        g.ldb = ldt;
        g.rows = p.rows;
        g.cols = p.n_in;
        g.len = p.n_out;
        g.out = dx;
        g.ldo = lddx;
        e = run_nt<T>(p.type, g, true, b.part, s);
        if (e != hipSuccess) return e;
    }
    if (dw) {
        GemmArgs g = {};
        const void* x = copy_x ? b.x : p.x;
        const int64_t ldx = copy_x ? padded(p.type, p.n_in) : p.ldx;
        const bool fast_x = copy_x || fast(x, ldx, p.n_in, p.type);
        const Plan plan = plan_tt(p.type, p.n_out, p.n_in, p.rows, planes, fast_x);
        g.a = dz;
        g.lda = ldo;
        g.b = x;
        g.ldb = ldx;
        g.rows = p.n_out;
        g.cols = p.n_in;
        g.len = p.rows;
        g.splits = plan.splits;
        g.split_len = plan.split_len;
        g.planes = planes;
        g.plane_stride = p.rows * ldo;
        g.plane_scale = plane_scale(p.type);
        g.out = dw;
        g.ldo = lddw;
        g.out_f32 = dw_type == GS_F32;
        g.part = plan.splits > 1 ? b.part : nullptr;
        e = LinearOps<T>::gemm_tt(plan.tile, fast_x, g, s);
        if (e == hipSuccess && g.part) e = LinearOps<T>::join(g, s);
    }
    return e;
}

}  // namespace

size_t linear_fwd_workspace(const gs_linear& p, bool z)
{
    return fwd_space(nullptr, p.type, p.act, p.rows, p.n_in, p.n_out, !fast(p.w, p.ldw, p.n_in, p.type), z,
                     fast(p.x, p.ldx, p.n_in, p.type)).bytes;
}

size_t linear_bwd_workspace(const gs_linear& p, const void* dy, int64_t lddy, int dw_type)
{
    return bwd_space(nullptr, p.type, p.act, p.rows, p.n_in, p.n_out, dw_type,
                     p.act != GS_ACT_NONE || !fast(dy, lddy, p.n_out, p.type)).bytes;
}

size_t linear_workspace(int type, int act, int64_t rows, int64_t in, int64_t out, int dw_type)
{
    // (the forward that needs most: with z, W and x as they may come, whatever the activation)
    const size_t fwd = fwd_space(nullptr, type, GS_ACT_NONE, rows, in, out, true, true, true).bytes;
    if (dw_type < 0) return fwd;
    // (fewer planes of dz can mean more splits of dW: the size for an fp32 dW does for one in the type as well)
    return std::max({fwd, bwd_space(nullptr, type, act, rows, in, out, dw_type, true).bytes,
                     bwd_space(nullptr, type, act, rows, in, out, type, true).bytes});
}

// Work items of a launch are counted in 32 bits.
bool linear_grid_fits(int64_t rows, int64_t cols)
{
    return div_up(rows, 128) * div_up(cols, cols <= 64 ? 64 : 128) * 256 < ((int64_t)1 << 32);
}

// The launch that transposes W for dx, beside dz and x of up to 2^12 workgroups each.
bool linear_dx_fits(int64_t in, int64_t out)
{
    return (div_up(in, 64) * div_up(out, 64) + 8192) * kBlock < ((int64_t)1 << 32);
}

hipError_t launch_linear_fwd(const gs_linear& p, const void* residual, int64_t ldr, void* y, int64_t ldy, void* z,
                             int64_t ldz, void* ws, hipStream_t s)
{
    if (p.type == GS_F16) return linear_fwd<f16>(p, residual, ldr, y, ldy, z, ldz, ws, s);
    if (p.type == GS_BF16) return linear_fwd<bf16>(p, residual, ldr, y, ldy, z, ldz, ws, s);
    return linear_fwd<float>(p, residual, ldr, y, ldy, z, ldz, ws, s);
}

hipError_t launch_linear_bwd(const gs_linear& p, const void* dy, int64_t lddy, const void* z, int64_t ldz, void* dx,
                             int64_t lddx, void* dw, int64_t lddw, int dw_type, float* db, void* ws, hipStream_t s)
{
    if (p.type == GS_F16) return linear_bwd<f16>(p, dy, lddy, z, ldz, dx, lddx, dw, lddw, dw_type, db, ws, s);
    if (p.type == GS_BF16) return linear_bwd<bf16>(p, dy, lddy, z, ldz, dx, lddx, dw, lddw, dw_type, db, ws, s);
    return linear_bwd<float>(p, dy, lddy, z, ldz, dx, lddx, dw, lddw, dw_type, db, ws, s);
}

}  // namespace gsr
