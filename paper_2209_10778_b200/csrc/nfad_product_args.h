// nfad_product_args.h -- what the matrix-product kernels are given; plain data, shared by the kernels and the extern "C"
// boundary.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace nfad {

constexpr int kMaxExperts = 1024;            // what a CTA's table of row ranges holds
constexpr int kNoAct = -1;

// The four products.  Rows of x and gz are grouped by expert; w is [experts, out, in].
//   kProdForward   y[m, o]   = f(sum_i x[m, i] w[e, o, i] + bias[e, o])        (and f')
//   kProdInput     gx[m, i]  = (sum_o gz[m, o] w[e, o, i]) prev[m, i]
//   kProdWeight    gw[e,o,i] = sum_{m of e} gz[m, o] x[m, i]
//   kProdBytes     y[m, o]   = f(x_scale[m] w_scale[o] sum_i xq[m, i] wq[o, i] + bias[o])     (8-bit integers, one expert)
enum ProdOp { kProdForward, kProdInput, kProdWeight, kProdBytes };

struct ProdArgs {
    const void *a, *b;               // kProdForward x, w; kProdInput gz, w; kProdWeight gz, x; kProdBytes xq, wq
    const void *bias;                // or null
    const void *prev;                // kProdInput: a factor for each result, or null
    const float *a_scale, *b_scale;  // kProdBytes
    const int *offsets;              // [experts + 1] on the device; null: one expert with every row
    void *out, *slope;               // slope: f', or null
    size_t rows;
    uint32_t in, outs, experts;
    int act;                         // a Kind or kNoAct
    int b_ready;                     // the kernel in front of this one does not write b, and began after whatever did
};

}  // namespace nfad
