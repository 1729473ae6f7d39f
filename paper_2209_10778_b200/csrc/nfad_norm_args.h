// nfad_norm_args.h -- what the norm kernels are given; plain data, shared by the kernels and the extern "C" boundary.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace nfad {

enum NormKind { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };

struct NormForwardArgs {
    const void *u, *r, *post_gain, *post_bias, *gate, *pre_gain, *pre_bias;
    void *s, *h;
    float4* stats;
    size_t rows, rows_per_gate;
    uint32_t cols, packets;
    int post, pre;
    float alpha, eps, inv_cols;
};

// Column sums in the order they stand in the scratch.
enum NormSum { kSumPreGain, kSumPreBias, kSumPostGain, kSumPostBias, kNormSums };

struct NormBackwardArgs {
    const void *grad_h, *grad_s, *u, *s, *post_gain, *post_bias, *gate, *pre_gain;
    const float4* stats;
    void *grad_u, *grad_r;
    float *sums[kNormSums], *grad_gate;      // results (each may be null)
    float *partial;                          // [chunks][kNormSums][cols], then the gate's [chunks][2][cols]
    float4 *row_means;                       // [rows] (any-shape kernels)
    size_t rows, rows_per_gate, chunk_rows;
    uint32_t cols, packets, chunks;
    int post, pre;
    float alpha, inv_cols;
};

}  // namespace nfad
