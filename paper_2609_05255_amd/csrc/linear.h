// Shared between the per-type instances of the linear operators (linear_f16.hip,
// linear_bf16.hip, linear_f32.hip) and their dispatch (linear.hip).
#pragma once

#include "gs_internal.h"
#include "mix.h"
#include "vec.h"

namespace gsr {

// One product C[i][j] = sum over c of A(i, c) B(j, c), i < rows, j < cols, c < len.
// NT: A(i, c) = a[i lda + c], B(j, c) = b[j ldb + c] (both contiguous along the sum).
// TT: A(i, c) = a[c lda + i], B(j, c) = b[c ldb + j] (both contiguous across it).
// The sum may be split: part `split` covers c in [split * split_len, ...). In TT A may be given in planes (a + plane *
// plane_stride), whose products are added up with the factors plane_scale^plane.
struct GemmArgs {
    const void* a;
    const void* b;
    int64_t lda, ldb;
    int64_t rows, cols, len;
    int64_t split_len;
    int32_t splits, planes;
    int64_t plane_stride;
    float plane_scale;
    // epilogue: out = act(C + bias) + residual, z = C + bias
    const float* bias;
    const void* residual;
    void* out;
    void* z;
    int64_t ldr, ldo, ldz;
    int32_t act;
    int32_t out_f32;               // out is fp32 whatever the type (residual, z: unused)
    float* part;                   // [splits][rows][cols] fp32 instead of the epilogue, or NULL
    Mix mix;                       // a mixture's products: rows (NT) or len (TT) are those of all experts
};

// dz = dy act'(z) of [rows][cols], as `planes` planes of the element type whose sum it is (plane k scaled by
// plane_scale^k), [rows][ldo] each, zero in the padding columns; and partial column sums of dz.
struct SlopeArgs {
    const void* dy;
    const void* z;
    int64_t lddy, ldz, ldo;
    int64_t rows, cols;
    int32_t act, planes;
    void* out;                     // NULL: column sums only
    int64_t plane_stride;
    float* sums;                   // [workgroups along the rows][cols], or NULL
    int32_t row_blocks;
    int32_t lanes;                 // of a workgroup along a row (set by prepare)
};

// dst[c][r] (ldd) = src[r][c] (lds), zero in the padding columns.
struct TransposeArgs {
    const void* src;
    int64_t lds, rows, cols;
    void* dst;
    int64_t ldd;
};

struct PrepareArgs {
    SlopeArgs slope, copy;
    TransposeArgs transpose;
    int64_t slope_blocks, tiles_x, tiles;
};

// Tiles of a product (rows x columns; By: so many groups of waves share its sum)
enum { kTile256 = 0, kTile128, kTile64, kTile64By4, kTile128x64 };

// A narrow layer in one pass (narrow.h).
struct NarrowArgs {
    const void *dy, *z, *x, *w;
    int64_t lddy, ldz, ldx, ldw, lddx, lddw;
    int64_t rows;
    int32_t out, in, act, dw_f32;
    void* dx;                      // dx, dw, db: NULL where not wanted
    void* dw;
    float* db;
    float* part;                   // [workgroups][narrow_part] dW [out][in], then db
    Mix mix;
};
__host__ __device__ inline int64_t narrow_part(int out, int in) { return (out * in + out + 3) / 4 * 4; }

template <typename T>
struct NarrowOps {   // T 16-bit
    // fast: rows of x are 16-byte aligned and whole 16-byte vectors
    static hipError_t forward(const GemmArgs& g, bool fast, int blocks, hipStream_t s);
    // fast: rows of dy, z and x are 16-byte aligned and whole 16-byte vectors
    static hipError_t backward(const NarrowArgs& a, bool fast, int planes, int blocks, hipStream_t s);
};

// per type T (the files linear_*.hip)
template <typename T>
struct LinearOps {
    // fast_a (NT), fast_b (TT): the operand's rows are 16-byte aligned and whole 16-byte vectors
    static hipError_t gemm_nt(int tile, bool fast_a, const GemmArgs& g, hipStream_t s);
    static hipError_t gemm_tt(int tile, bool fast_b, const GemmArgs& g, hipStream_t s);
    static hipError_t skinny(const GemmArgs& g, hipStream_t s);
    // those that are wanted (not NULL) of dz, a matrix copied (dz without an activation) and W transposed, in one launch
    static hipError_t prepare(const SlopeArgs* slope, const SlopeArgs* copy, const TransposeArgs* transpose,
                              hipStream_t s);
    static hipError_t join(const GemmArgs& g, hipStream_t s);   // adds the parts up, with the epilogue
};

// What the products of a mixture's backward need before them, in one launch: dz with its column sums over units of each
// expert's rows, a copy of x with aligned rows, and each expert's W transposed, or copied with aligned rows.
struct MixPrepareArgs {
    Mix mix;                       // size: rows of dz's units
    SlopeArgs slope, copy, weights;
    TransposeArgs transpose;
    int64_t w_out;                 // values of an expert's W in the copy or transposed
    int64_t slope_x, slope_blocks, copy_blocks, weight_blocks;   // workgroups across dz, in all, of x, of one expert's W
};

// db[e][c]: the sums over expert e's units (mix.size rows) of part [units][cols].
struct MixSums {
    Mix mix;
    const float* part;
    int64_t cols;
    float* db;
};

// per type T (the files experts_*.hip)
template <typename T>
struct MixtureOps {
    static hipError_t gemm_nt(int tile, bool fast_a, const GemmArgs& g, hipStream_t s);
    static hipError_t gemm_tt(int tile, bool fast_b, const GemmArgs& g, hipStream_t s);
    // dW's product and dx's together, in tiles of 64 x 64 (w's B, like x's operands, with whole aligned rows)
    static hipError_t gemm_pair(const GemmArgs& w, const GemmArgs& x, hipStream_t s);
    // the parts of dW (g.part NULL: none) and of db (b.db NULL: none) added up
    static hipError_t join(const GemmArgs& g, const MixSums& b, hipStream_t s);
    static hipError_t skinny(const GemmArgs& g, hipStream_t s);
    // slope, copy, weights, transpose: those that are wanted; units: of dz, at most
    static hipError_t prepare(const Mix& mix, int64_t units, const SlopeArgs* slope, const SlopeArgs* copy,
                              const SlopeArgs* weights, const TransposeArgs* transpose, int64_t w_out, hipStream_t s);
    // 16-bit layers of up to 128 inputs and outputs, in units of mix.size rows
    static hipError_t narrow_fwd(const GemmArgs& g, bool fast, int64_t units, hipStream_t s);
    static hipError_t narrow_bwd(const NarrowArgs& a, bool fast, int planes, int64_t units, hipStream_t s);
};

}  // namespace gsr
