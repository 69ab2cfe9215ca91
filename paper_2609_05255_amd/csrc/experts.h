// Kernels of a mixture's layers beside the products of gemm.h and narrow.h.
#pragma once

#include "narrow.h"

namespace gsr {

namespace {

template <typename T>
__global__ __launch_bounds__(kBlock) void k_mix_prepare(MixPrepareArgs a)
{
    constexpr int kSums = kBlock * (Vec<T>::N + 1) * 4, kTile = kTransposeTile * (kTransposeTile * sizeof(T) + 4);
    __shared__ __attribute__((aligned(16))) char lds[kSums > kTile ? kSums : kTile];
    int64_t b = blockIdx.x;
    if (b < a.slope_blocks) {
        const int64_t unit = b / a.slope_x;
        const MixUnit u = mix_unit(a.mix, a.mix.size, 0, unit);
        if (u.expert < 0) return;
        const int64_t first = u.first + (int64_t)u.unit * a.mix.size, left = u.rows - (int64_t)u.unit * a.mix.size;
        SlopeArgs p = a.slope;
        p.rows = left < a.mix.size ? left : a.mix.size;
        p.row_blocks = 1;
        p.dy = (const T*)p.dy + first * p.lddy;
        if (p.act != GS_ACT_NONE) p.z = (const T*)p.z + first * p.ldz;
        if (p.out) p.out = (T*)p.out + first * p.ldo;
        if (p.sums) p.sums += unit * p.cols;
        slope_rows<T>(p, b % a.slope_x, 0, lds);
        return;
    }
    b -= a.slope_blocks;
    if (b < a.copy_blocks) {
        slope_rows<T>(a.copy, b / a.copy.row_blocks, b % a.copy.row_blocks, lds);
        return;
    }
    b -= a.copy_blocks;
    const int64_t e = b / a.weight_blocks;
    b -= e * a.weight_blocks;
    if (mix_offset(a.mix, (int)e + 1) <= mix_offset(a.mix, (int)e)) return;   // nobody reads its weights
    if (a.transpose.src) {
        TransposeArgs p = a.transpose;
        const int64_t tiles_x = (p.cols + kTransposeTile - 1) / kTransposeTile;
        p.src = (const T*)p.src + e * a.mix.w_stride;
        p.dst = (T*)p.dst + e * a.w_out;
        transpose_tile<T>(p, b % tiles_x, b / tiles_x, lds);
    } else {
        SlopeArgs p = a.weights;
        p.dy = (const T*)p.dy + e * a.mix.w_stride;
        p.out = (T*)p.out + e * a.w_out;
        slope_rows<T>(p, b / p.row_blocks, b % p.row_blocks, lds);
    }
}

// Adds up the parts of an expert's dW where it has several, and of its db; blockIdx.y is the expert, and workgroups from
// `join` on take 16 columns of db each, 16 threads one's units.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_mix_join(GemmArgs g, int join, MixSums b)
{
    __shared__ float s[16][16];
    if ((int)blockIdx.x >= join) {
        const MixUnit u = mix_expert(b.mix, b.mix.size, 0, blockIdx.y);
        const int col = threadIdx.x & 15, slice = threadIdx.x >> 4;
        const int64_t c = (int64_t)(blockIdx.x - join) * 16 + col, units = min((int64_t)u.units, b.mix.limit - u.before);
        float t = 0.f;
        if (c < b.cols)
#pragma unroll 8
            for (int64_t k = slice; k < units; k += 16) t += b.part[(u.before + k) * b.cols + c];
        s[slice][col] = t;
        __syncthreads();
        if (slice != 0 || c >= b.cols) return;
#pragma unroll
        for (int k = 1; k < 16; ++k) t += s[k][col];
        b.db[u.expert * b.cols + c] = t;
        return;
    }
    const MixUnit u = mix_expert(g.mix, (int)g.split_len, 1, blockIdx.y);
    if (u.units < 2) return;
    const int64_t quads = (g.cols + 3) / 4, size = g.rows * g.cols;
    const int64_t before = mix_parts_before(g.mix, (int)g.split_len, u.expert);
    const int64_t units = min((int64_t)u.units, g.mix.limit - before);
    const float* parts = g.part + before * size;
    for (int64_t k = (int64_t)blockIdx.x * kBlock + threadIdx.x; k < g.rows * quads; k += (int64_t)join * kBlock) {
        const int64_t i = k / quads, j = (k - i * quads) * 4, left = g.cols - j;
        const float* part = parts + i * g.cols + j;
        float v[4] = {};
#pragma unroll 8
        for (int64_t p = 0; p < units; ++p) {
            float t[4];
            load_vec(part + p * size, left, t);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += t[e];
        }
        const int64_t o = u.expert * g.mix.dw_stride + i * g.ldo + j;
        if (g.out_f32) {
            store_vec((float*)g.out + o, left, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) ((T*)g.out)[o + e] = (T)v[e];
        }
    }
}

}  // namespace

template <typename T>
hipError_t MixtureOps<T>::gemm_nt(int tile, bool fast_a, const GemmArgs& g, hipStream_t s)
{
    return run_nt<T, true>(tile, fast_a, g, s);
}

template <typename T>
hipError_t MixtureOps<T>::gemm_tt(int tile, bool fast_b, const GemmArgs& g, hipStream_t s)
{
    return run_tt<T, true>(tile, fast_b, g, s);
}

template <typename T>
hipError_t MixtureOps<T>::gemm_pair(const GemmArgs& w, const GemmArgs& x, hipStream_t s)
{
    using TT = Shape<true, 64, 64, 2, 2, false, true>;
    using NT = Shape<false, 64, 64, 2, 2, false, true>;
    const int64_t tiles = div_up(w.rows, 64) * div_up(w.cols, 64), units = mix_units(w.len, w.mix.experts, w.split_len, 1);
    const int64_t others = mix_units(x.rows, x.mix.experts, 64, 0) * div_up(x.cols, 64), bk = 128 / (int)sizeof(T);
    const int lds = std::max(TT::lds_bytes(div_up(w.split_len, bk), sizeof(T)), NT::lds_bytes(div_up(x.split_len, bk), sizeof(T)));
    // the longer workgroups first (the other way round 600 x 1,024 -> 1,024 in fp32 of 4 experts takes 72 us for 52, 20,000 x
    // 256 -> 256 in binary16 of 8 50 for 46)
    const bool x_first = x.len >= w.planes * std::min(w.split_len, div_up(w.len, w.mix.experts));
    hipLaunchKernelGGL((k_gemm_pair<T, TT, NT>), dim3((unsigned)(tiles * units + others)), dim3(TT::THREADS), lds, s, w, x,
                       (uint32_t)tiles, x_first ? (uint32_t)others : 0, x_first ? 0 : (uint32_t)(tiles * units));
    return hipGetLastError();
}

template <typename T>
hipError_t MixtureOps<T>::join(const GemmArgs& g, const MixSums& b, hipStream_t s)
{
    const int join = g.part ? (int)std::min<int64_t>(div_up(g.rows * div_up(g.cols, 4), kBlock), 4096) : 0;
    const int64_t sums = b.db ? div_up(b.cols, 16) : 0;
    if (join + sums == 0) return hipSuccess;
    const int experts = g.part ? g.mix.experts : b.mix.experts;
    hipLaunchKernelGGL((k_mix_join<T>), dim3((unsigned)(join + sums), (unsigned)experts), dim3(kBlock), 0, s, g, join, b);
    return hipGetLastError();
}

template <typename T>
hipError_t MixtureOps<T>::skinny(const GemmArgs& g, hipStream_t s)
{
    return run_skinny<T, true>(g, s);
}

template <typename T>
hipError_t MixtureOps<T>::prepare(const Mix& mix, int64_t units, const SlopeArgs* slope, const SlopeArgs* copy,
                                  const SlopeArgs* weights, const TransposeArgs* transpose, int64_t w_out,
                                  hipStream_t s)
{
    MixPrepareArgs a = {};
    a.mix = mix;
    a.w_out = w_out;
    a.slope_x = a.weight_blocks = 1;
    auto lanes = [](const SlopeArgs& from, SlopeArgs& to) -> int64_t {   // workgroups across
        to = from;
        const int64_t vecs = div_up(std::max(to.ldo, to.cols), Vec<T>::N);
        to.lanes = 1;
        while (to.lanes < 64 && to.lanes < vecs) to.lanes <<= 1;
        return div_up(vecs, to.lanes);
    };
    int64_t all = 0;
    if (slope) {
        a.slope_x = lanes(*slope, a.slope);
        all += a.slope_blocks = a.slope_x * units;
    }
    if (copy) all += a.copy_blocks = lanes(*copy, a.copy) * copy->row_blocks;
    if (weights) all += (a.weight_blocks = lanes(*weights, a.weights) * weights->row_blocks) * mix.experts;
    if (transpose) {
        a.transpose = *transpose;
        a.weight_blocks = div_up(transpose->cols, kTransposeTile) *
                          div_up(std::max(transpose->rows, transpose->ldd), kTransposeTile);
        all += a.weight_blocks * mix.experts;
    }
    if (all == 0) return hipSuccess;
    hipLaunchKernelGGL((k_mix_prepare<T>), dim3((unsigned)all), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t MixtureOps<T>::narrow_fwd(const GemmArgs& g, bool fast, int64_t units, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) return run_narrow_fwd<T, true>(g, fast, (int)units, s);
    return hipErrorInvalidValue;
}

template <typename T>
hipError_t MixtureOps<T>::narrow_bwd(const NarrowArgs& a, bool fast, int planes, int64_t units, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) return run_narrow_bwd<T, true>(a, fast, planes, (int)units, s);
    return hipErrorInvalidValue;
}

}  // namespace gsr
