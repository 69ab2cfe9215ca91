// The layers of a mixture's experts over rows that are sorted by expert: plans, workspaces, launches.
//
//   fwd: z = x W_e^T + b_e, y = act(z)                          for the rows of expert e
//   bwd: dz = dy act'(z), dx = dz W_e, dW_e = dz^T x, db_e = column sums of dz, both over the expert's rows
//
// Where an expert's rows begin is on the device only. The kernels are those of the linear operators (gemm.h, narrow.h):
// the rows are cut into units of up to so many rows of one expert, and a workgroup finds its unit in the offsets by a scan
// over the experts. A grid holds as many units as there can be, rows / size and one more for each expert, and the
// workgroups behind the last one leave. Weights of experts without rows are not read. Bound, as there: by HBM for narrow
// layers, by reading the weights for few rows, by the matrix cores for the rest.
//
// Measured (us; one linear layer over all the rows beside it): 1,000,000 x 64 -> 128 in binary16, 16 experts of uneven
// shares, silu, backward 179 and 179, forward with z 131 and 134; 16,384 x 2,048 -> 2,048 in bfloat16, 8 experts, gelu,
// forward with z 171 (of even shares 151, one expert 136) and 154, backward with fp32 dW 647 and 547; 50,000 x 256 -> 512 in
// binary16, 16 experts, backward 153 and 154; 5,003 x 333 -> 215 in fp32, 7 experts, backward 40 and 45; 8 rows of
// 2,048 -> 2,048 in bfloat16 by five of 16 experts 11.3 (42 MB of weights at 3.7 TB/s).
//
// In the 16-bit types dx, and dW in the type, take dz rounded to the type, as the linear layer's do: that rounding joins the
// result's own (1,000,000 x 64 -> 128 with silu: dx 2.9e-4 off in norm in binary16 and 2.3e-3 in bfloat16, where dz in fp32
// would give 2.1e-4 and 1.7e-3). Planes of dz for dx as well, whether or not there is an fp32 dW, would be two or three times
// its products and the bytes of dz.
#include "linear_plan.h"

namespace gsr {

namespace {

constexpr int kDzBlocks = 2048;          // workgroups of dz, about
constexpr int64_t kNarrowRows = 128;     // of a unit of a narrow layer, at least
constexpr int64_t kPlaces = 5 * kFillTiles;   // workgroups that the compute units hold at once, of any tile at most
// Workgroups of a narrow layer's forward, about, and of its backward kNarrowBlocks. The forward's number matters little: with
// 512, 1,024, 2,048 and 4,096 1,000,000 rows of 16 experts take 133, 140, 132 and 126 us (64 -> 128 in binary16), 171, 172,
// 180 and 191 (128 -> 128) and 51, 44, 46 and 42 (32 -> 32), so that none is the best for all three, and 355, 356, 358 and
// 359 together. The backward takes with 512 and 1,024 200 and 205 (64 -> 128), 59 and 60 (32 -> 32), of 200,000 x 64 -> 64
// and 64 experts in bfloat16 41 and 45.
constexpr int64_t kNarrowForward = 2048;
constexpr int64_t kMostSplits = 8;       // parts of one of the last tiles
constexpr double kSplitGain = 2.0;       // us that a split of the last tiles has to gain by the plan

int64_t units_most(int64_t rows, int64_t experts, int64_t size) { return rows / size + std::min(rows, experts); }

// The tile, and for dW the rows of a unit, that the rates of plan_product make fastest for experts of about equal shares.
// NT: the tiles that do not fill the compute units another time may be split along the sum (MixTail in gemm.h). 528 tiles of
// 256 x 256 on 256 compute units (16,384 x 2,048 -> 2,048 in bfloat16, 8 experts of uneven shares): the last 16 split into
// 8 parts each 172 us, where tiles of 128 x 128, whole, take 204.
Plan plan_mix(int type, bool tt, int64_t rows, int64_t cols, int64_t len, int64_t experts, int planes, bool fast_operand)
{
    Plan best = {kTile64, 1, std::min<int64_t>(std::max<int64_t>(len, 64), 1 << 30)};
    double best_us = 1e300;
    const TileRate* rates = type == GS_F32 ? kRates32 : kRates16;
    const int count = type == GS_F32 ? 3 : 5;
    const int64_t some = std::max<int64_t>(1, std::min(tt ? len : rows, experts));
    for (int k = 0; k < count; ++k) {
        const TileRate& r = rates[k];
        if (!fast_operand && (r.tile == kTile256 || r.tile == kTile64By4)) continue;
        if (tt && r.tile == kTile128x64) continue;
        const double slow = fast_operand ? 1.0 : kSlowRate, area = 2.0 * r.rows * r.cols * kFillTiles;
        const int threads = r.tile == kTile64By4 ? 1024 : r.tile == kTile256 ? 512 : 256;
        if (!tt) {
            if (len < r.least) continue;
            if ((units_most(rows, experts, r.rows) * div_up(cols, r.cols) + kPlaces) * threads >> 32) continue;
            // rounds of tiles that fill the compute units, and the rest, whole or split along the sum
            const int64_t places = r.held * kFillTiles;
            const int64_t tiles = std::max(some, rows / r.rows + some / 2) * div_up(cols, r.cols), rest = tiles % places;
            const auto round = [&](int64_t count, int64_t sum) {   // of so many tiles, places at most
                const int64_t share = div_up(count, kFillTiles);
                return area * (double)sum * (share > 1 ? share / r.flop_us : 1 / r.flop_us_one) / slow + r.round_us;
            };
            const double whole = (double)(tiles / places) * round(places, len) + (rest ? round(rest, len) : 0.0);
            if (whole < best_us) {
                best_us = whole;
                best = {r.tile, 1, len};
            }
            const int64_t least = 4 * 128 / elem(type);   // values of a part
            const int64_t splits = rest ? std::min({places / 2 / rest, len / least, kMostSplits}) : 1;
            if (splits < 2 || r.tile == kTile64By4 || !fast_operand) continue;
            const double us = (double)(tiles / places) * round(places, len) + round(rest * splits, div_up(len, splits)) +
                              kJoinUs + 8.0 * rest * splits * r.rows * r.cols / kBytesUs;
            if (us + kSplitGain < best_us) {
                best_us = us;
                best = {r.tile, (int)splits, len};
            }
            continue;
        }
        const int64_t tiles = div_up(rows, r.rows) * div_up(cols, r.cols);
        if (tiles * threads >> 32) continue;
        for (int64_t want = 1; want == 1 || len / want >= kRowSplitLen; want *= 2) {
            const int64_t size = std::min<int64_t>(std::max<int64_t>(64, div_up(div_up(len, want), 64) * 64), 1 << 30);
            if (units_most(len, experts, size) + experts > 65535) break;
            // A larger share than most: three times the mean (two: 16,384 x 1,024 -> 1,024 in bfloat16 of 8 experts, shares
            // as 1 / (e + 1), 340 us instead of 256, even ones 234 and 238; four: 20,000 x 512 -> 1,024 of 32 317 for 235).
            const double longest = (double)std::min<int64_t>(size, 3 * div_up(len, some));
            const double units = (double)len / size + 0.5 * some, each = (double)len / units;
            const int64_t share = div_up((int64_t)(units * tiles) + 1, kFillTiles), rounds = div_up(share, r.held);
            double us = std::max(area * each * share / r.flop_us, area * longest / r.flop_us_one) * planes / slow +
                        (double)rounds * r.round_us;
            if ((double)size < longest * 1.01 && want > 1) us += kJoinUs + 8.0 * units * (double)rows * (double)cols / kBytesUs;
            if (us < best_us) {
                best_us = us;
                best = {r.tile, (int)want, size};
            }
        }
    }
    return best;
}

// Parts of dW: the units of experts that have several.
int64_t parts_most(const Plan& p, int64_t rows, int64_t experts)
{
    return p.split_len >= rows ? 0 : std::min(units_most(rows, experts, p.split_len), 2 * (rows / p.split_len));
}

// Rows of a unit of dz: two of each thread, more where that would be more workgroups than it takes.
int64_t dz_size(int type, int64_t rows, int64_t cols)
{
    const int64_t vecs = div_up(cols, vec(type)), across = div_up(vecs, 64);
    int64_t lanes = 1;
    while (lanes < 64 && lanes < vecs) lanes <<= 1;
    const int64_t least = 2 * kBlock / lanes;
    return div_up(std::max(least, div_up(rows * across, kDzBlocks)), least) * least;
}

// Rows of a unit of a narrow layer: as many units as there are places for workgroups, those of the experts' ends with them.
int64_t narrow_size(int64_t rows, int64_t experts, bool backward)
{
    const int64_t most = backward ? kNarrowBlocks : kNarrowForward;
    return std::max(kNarrowRows, div_up(div_up(rows, std::max(most / 2, most - experts)), 64) * 64);
}

bool narrow_taken(int type, int64_t rows, int64_t in, int64_t out) { return rows > kFewRows && narrow(type, in, out); }

bool fast_w(const gs_experts& p)
{
    return fast(p.layer.w, p.layer.ldw, p.layer.n_in, p.layer.type) && p.w_stride % vec(p.layer.type) == 0;
}

// Bytes of the parts that the last tiles of a product along rows are split into.
int64_t tail_bytes(int type, const Plan& p)
{
    if (p.splits < 2) return 0;
    for (const TileRate* r = type == GS_F32 ? kRates32 : kRates16;; ++r)
        if (r->tile == p.tile) return (int64_t)r->held * kFillTiles / 2 * r->rows * r->cols * 4;
}

Plan plan_rows(int type, int64_t rows, int64_t experts, int64_t cols, int64_t len, bool fast_a)
{
    if (rows <= kFewRows) return {kTile64, 1, len};
    return plan_mix(type, false, rows, cols, len, experts, 1, fast_a);
}

struct FwdSpace {
    void* w;       // W with padded rows, where its own cannot be read in vectors
    float* part;
    size_t bytes;
};

FwdSpace fwd_space(void* base, int type, int64_t rows, int64_t experts, int64_t in, int64_t out, bool copy_w)
{
    Regions r{(char*)base};
    FwdSpace f = {};
    if (rows > kFewRows && !narrow(type, in, out)) {
        if (copy_w) f.w = r.take(experts * out * padded(type, in) * elem(type));
        // (a workspace is sized for either alignment of x)
        f.part = (float*)r.take(std::max(tail_bytes(type, plan_rows(type, rows, experts, out, in, false)),
                                         tail_bytes(type, plan_rows(type, rows, experts, out, in, true))));
    }
    f.bytes = r.at;
    return f;
}

struct BwdSpace {
    void *x, *dz, *wt;   // x with padded rows, dz in planes, each W transposed
    float *sums, *part;
    size_t bytes;
};

// dw_type: -1 without dW
BwdSpace bwd_space(void* base, int type, int act, int64_t rows, int64_t experts, int64_t in, int64_t out, int dw_type,
                   bool need_dz)
{
    Regions r{(char*)base};
    BwdSpace b = {};
    if (narrow(type, in, out)) {
        b.part = (float*)r.take(units_most(rows, experts, narrow_size(rows, experts, true)) *
                                narrow_part((int)out, (int)in) * 4);
        b.bytes = r.at;
        return b;
    }
    const bool want_dw = dw_type >= 0;
    const int planes = planes_of(type, act, dw_type);
    if (need_dz) b.dz = r.take(planes * rows * padded(type, out) * elem(type));
    if (want_dw && in % vec(type)) b.x = r.take(rows * padded(type, in) * elem(type));
    b.wt = r.take(experts * in * padded(type, out) * elem(type));
    b.sums = (float*)r.take(units_most(rows, experts, dz_size(type, rows, out)) * out * 4);
    int64_t parts = 0;
    // (a workspace is sized for either operand's alignment)
    for (int fast_x = 0; want_dw && fast_x < 2; ++fast_x)
        parts = std::max(parts, parts_most(plan_mix(type, true, out, in, rows, experts, planes, fast_x != 0), rows, experts));
    b.part = (float*)r.take(std::max(parts * out * in * 4, tail_bytes(type, plan_rows(type, rows, experts, in, out, true))));
    b.bytes = r.at;
    return b;
}

Mix mix_of(const gs_experts& p, int64_t size)
{
    Mix m = {};
    m.offsets = p.offsets;
    m.experts = (int32_t)p.experts;
    m.rows = p.layer.rows;
    m.w_stride = p.w_stride;
    m.size = (int32_t)size;
    return m;
}

template <typename T>
hipError_t run_nt(int type, GemmArgs g, const Plan& p, bool fast_a, float* part, hipStream_t s)
{
    g.splits = g.planes = 1;
    g.split_len = g.len;
    if (g.rows <= kFewRows) return MixtureOps<T>::skinny(g, s);
    if (p.splits > 1) {
        g.splits = p.splits;
        g.part = part;
        for (const TileRate* r = type == GS_F32 ? kRates32 : kRates16;; ++r)
            if (r->tile == p.tile) {
                g.mix.size = r->held * kFillTiles;
                break;
            }
    }
    return MixtureOps<T>::gemm_nt(p.tile, fast_a, g, s);
}

template <typename T>
hipError_t experts_fwd(const gs_experts& p, void* y, int64_t ldy, void* z, int64_t ldz, void* ws, hipStream_t s)
{
    const gs_linear& l = p.layer;
    const bool fast_x = fast(l.x, l.ldx, l.n_in, l.type);
    GemmArgs g = {};
    g.a = l.x;
    g.lda = l.ldx;
    g.b = l.w;
    g.ldb = l.ldw;
    g.rows = l.rows;
    g.cols = l.n_out;
    g.len = l.n_in;
    g.bias = l.bias;
    g.act = l.act;
    g.out = y;
    g.ldo = ldy;
    g.z = z;
    g.ldz = ldz;
    g.mix = mix_of(p, 0);
    if (narrow_taken(l.type, l.rows, l.n_in, l.n_out)) {
        g.mix.size = (int32_t)narrow_size(l.rows, p.experts, false);
        return MixtureOps<T>::narrow_fwd(g, fast_x, units_most(l.rows, p.experts, g.mix.size), s);
    }
    const FwdSpace f = fwd_space(ws, l.type, l.rows, p.experts, l.n_in, l.n_out, !fast_w(p));
    if (f.w) {
        SlopeArgs copy = copy_of(l.type, l.w, l.ldw, l.n_out, l.n_in, f.w);
        copy.row_blocks = (int)std::max<int64_t>(1, copy.row_blocks / p.experts);
        const int64_t each = l.n_out * padded(l.type, l.n_in);
        const hipError_t e = MixtureOps<T>::prepare(g.mix, 0, nullptr, nullptr, &copy, nullptr, each, s);
        if (e != hipSuccess) return e;
        g.b = f.w;
        g.ldb = padded(l.type, l.n_in);
        g.mix.w_stride = each;
    }
    return run_nt<T>(l.type, g, plan_rows(l.type, l.rows, p.experts, l.n_out, l.n_in, fast_x), fast_x, f.part, s);
}

template <typename T>
hipError_t experts_bwd(const gs_experts& p, const void* dy, int64_t lddy, const void* z, int64_t ldz, void* dx,
                       int64_t lddx, void* dw, int64_t lddw, int64_t dw_stride, int dw_type, float* db, void* ws,
                       hipStream_t s)
{
    const gs_linear& l = p.layer;
    const bool need_dz = l.act != GS_ACT_NONE || !fast(dy, lddy, l.n_out, l.type);
    const int planes = planes_of(l.type, l.act, dw ? dw_type : -1);
    const BwdSpace b = bwd_space(ws, l.type, l.act, l.rows, p.experts, l.n_in, l.n_out, dw ? dw_type : -1, need_dz);
    if (narrow(l.type, l.n_in, l.n_out)) {
        NarrowArgs a = {dy,        z,           l.x,  l.w, lddy,  ldz, l.ldx, l.ldw, lddx, lddw, l.rows, (int)l.n_out,
                        (int)l.n_in, l.act, dw_type == GS_F32, dx, dw,    db,  b.part};
        a.mix = mix_of(p, narrow_size(l.rows, p.experts, true));
        a.mix.dw_stride = dw_stride;
        a.mix.limit = units_most(l.rows, p.experts, a.mix.size);
        const bool whole = fast(dy, lddy, l.n_out, l.type) && fast(l.x, l.ldx, l.n_in, l.type) &&
                           (l.act == GS_ACT_NONE || fast(z, ldz, l.n_out, l.type));
        return MixtureOps<T>::narrow_bwd(a, whole, planes, a.mix.limit, s);
    }
    const int64_t ldo = need_dz ? padded(l.type, l.n_out) : lddy, ldt = padded(l.type, l.n_out);
    const void* dz = need_dz ? b.dz : dy;
    SlopeArgs slope = {}, copy = {};
    Mix rows = mix_of(p, dz_size(l.type, l.rows, l.n_out));
    rows.limit = units_most(l.rows, p.experts, rows.size);
    const bool want_slope = l.rows > 0 && (need_dz || db), want_dx = dx && l.rows > 0, copy_x = b.x && l.rows > 0;
    if (want_slope) {
        slope.dy = dy;
        slope.lddy = lddy;
        slope.z = z;
        slope.ldz = ldz;
        slope.cols = l.n_out;
        slope.act = l.act;
        slope.planes = planes;
        slope.out = need_dz ? b.dz : nullptr;
        slope.ldo = need_dz ? ldo : 0;
        slope.plane_stride = l.rows * ldo;
        slope.sums = db ? b.sums : nullptr;
    }
    if (copy_x) copy = copy_of(l.type, l.x, l.ldx, l.rows, l.n_in, b.x);
    const TransposeArgs transpose = {l.w, l.ldw, l.n_out, l.n_in, b.wt, ldt};
    hipError_t e = MixtureOps<T>::prepare(rows, rows.limit, want_slope ? &slope : nullptr,
                                          copy_x ? &copy : nullptr, nullptr, want_dx ? &transpose : nullptr, l.n_in * ldt, s);
    if (e != hipSuccess) return e;
    GemmArgs gx = {}, gw = {};   // dx's product and dW's
    if (want_dx) {
        gx.a = dz;
        gx.lda = ldo;
        gx.b = b.wt;
        gx.ldb = ldt;
        gx.rows = l.rows;
        gx.cols = l.n_in;
        gx.len = l.n_out;
        gx.out = dx;
        gx.ldo = lddx;
        gx.mix = mix_of(p, 0);
        gx.mix.w_stride = l.n_in * ldt;
    }
    Plan plan = {};
    bool fast_x = true;
    if (dw) {
        const void* x = copy_x ? b.x : l.x;
        const int64_t ldx = copy_x ? padded(l.type, l.n_in) : l.ldx;
        fast_x = copy_x || fast(x, ldx, l.n_in, l.type);
        plan = plan_mix(l.type, true, l.n_out, l.n_in, l.rows, p.experts, planes, fast_x);
        gw.a = dz;
        gw.lda = ldo;
        gw.b = x;
        gw.ldb = ldx;
        gw.rows = l.n_out;
        gw.cols = l.n_in;
        gw.len = l.rows;
        gw.splits = 1;
        gw.split_len = plan.split_len;
        gw.planes = planes;
        gw.plane_stride = l.rows * ldo;
        gw.plane_scale = plane_scale(l.type);
        gw.out = dw;
        gw.ldo = lddw;
        gw.out_f32 = dw_type == GS_F32;
        gw.mix = mix_of(p, 0);
        gw.mix.limit = parts_most(plan, l.rows, p.experts);
        gw.part = gw.mix.limit > 0 ? b.part : nullptr;
        gw.mix.dw_stride = dw_stride;
    }
    // Small tiles of both products: plain ones of 64 x 64, in one launch. (Which they are is a matter of the sizes, so that a
    // gradient has the same bits alone.)
    Plan px = plan_rows(l.type, l.rows, p.experts, l.n_in, l.n_out, true);
    const auto small = [](int tile) { return tile == kTile64 || tile == kTile64By4; };
    if (l.rows > kFewRows && small(px.tile) && px.splits == 1) {
        const bool dw_small = dw && small(plan.tile);
        if (dw_small) plan.tile = kTile64;
        if (small(plan_mix(l.type, true, l.n_out, l.n_in, l.rows, p.experts, 1, true).tile)) {
            px.tile = kTile64;
            const int64_t blocks = (dw_small ? div_up(l.n_out, 64) * (l.rows / plan.split_len + p.experts) : 0) +
                                   units_most(l.rows, p.experts, 64);
            if (want_dx && dw_small && fast_x && blocks * div_up(l.n_in, 64) * 256 >> 32 == 0) {
                gx.splits = gx.planes = 1;
                gx.split_len = gx.len;
                e = MixtureOps<T>::gemm_pair(gw, gx, s);
                return e != hipSuccess ? e : MixtureOps<T>::join(gw, {rows, b.sums, l.n_out, db}, s);
            }
        }
    }
    if (want_dx && (e = run_nt<T>(l.type, gx, px, true, b.part, s)) != hipSuccess) return e;
    if (dw && (e = MixtureOps<T>::gemm_tt(plan.tile, fast_x, gw, s)) != hipSuccess) return e;
    return MixtureOps<T>::join(gw, {rows, b.sums, l.n_out, db}, s);
}

}  // namespace

size_t experts_fwd_workspace(const gs_experts& p)
{
    return fwd_space(nullptr, p.layer.type, p.layer.rows, p.experts, p.layer.n_in, p.layer.n_out, !fast_w(p)).bytes;
}

size_t experts_bwd_workspace(const gs_experts& p, const void* dy, int64_t lddy, int dw_type)
{
    const gs_linear& l = p.layer;
    return bwd_space(nullptr, l.type, l.act, l.rows, p.experts, l.n_in, l.n_out, dw_type,
                     l.act != GS_ACT_NONE || !fast(dy, lddy, l.n_out, l.type)).bytes;
}

size_t experts_workspace(int type, int act, int64_t rows, int64_t experts, int64_t in, int64_t out, int dw_type)
{
    const size_t fwd = fwd_space(nullptr, type, rows, experts, in, out, true).bytes;
    if (dw_type < 0) return fwd;
    // (fewer planes of dz can mean more parts of dW: the size for an fp32 dW does for one in the type as well)
    return std::max({fwd, bwd_space(nullptr, type, act, rows, experts, in, out, dw_type, true).bytes,
                     bwd_space(nullptr, type, act, rows, experts, in, out, type, true).bytes});
}

// Work items of a launch are counted in 32 bits, for the smallest tiles, W transposed or copied, and dz.
bool experts_grid_fits(int64_t rows, int64_t experts, int64_t in, int64_t out)
{
    const int64_t most = std::max(in, out), limit = (int64_t)1 << 32;
    return units_most(rows, experts, 64) * div_up(most, 64) * 256 < limit &&
           (experts * (div_up(in, 64) + 1) * (div_up(out, 64) + 1) + 32768 + experts * div_up(most, 256)) * kBlock < limit;
}

hipError_t launch_experts_fwd(const gs_experts& p, void* y, int64_t ldy, void* z, int64_t ldz, void* ws, hipStream_t s)
{
    if (p.layer.type == GS_F16) return experts_fwd<f16>(p, y, ldy, z, ldz, ws, s);
    if (p.layer.type == GS_BF16) return experts_fwd<bf16>(p, y, ldy, z, ldz, ws, s);
    return experts_fwd<float>(p, y, ldy, z, ldz, ws, s);
}

hipError_t launch_experts_bwd(const gs_experts& p, const void* dy, int64_t lddy, const void* z, int64_t ldz, void* dx,
                              int64_t lddx, void* dw, int64_t lddw, int64_t dw_stride, int dw_type, float* db, void* ws,
                              hipStream_t s)
{
#define CALL(T) experts_bwd<T>(p, dy, lddy, z, ldz, dx, lddx, dw, lddw, dw_stride, dw_type, db, ws, s)
    if (p.layer.type == GS_F16) return CALL(f16);
    if (p.layer.type == GS_BF16) return CALL(bf16);
    return CALL(float);
#undef CALL
}

}  // namespace gsr
