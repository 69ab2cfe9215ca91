// Shared between the per-type instances of the linear operators (linear_f16.hip,
// linear_bf16.hip, linear_f32.hip) and their dispatch (linear.hip).
#pragma once

#include "gs_internal.h"
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

}  // namespace gsr
