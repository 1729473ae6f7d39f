// nfad_api_block.cu -- the extern "C" boundary of the operators around the activation: argument validation, aliasing rules
// and dispatch.  No arithmetic lives here.
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/nfad.h"
#include "nfad_dropout_args.h"
#include "nfad_internal.h"
#include "nfad_norm_args.h"
#include "nfad_product_args.h"

namespace {

size_t elem_size(int dtype) { return dtype == NFAD_F32 ? 4 : 2; }

struct Span { const void* p; size_t bytes, align; };

bool overlap(const Span& a, const Span& b)
{
    if (!a.p || !b.p || !a.bytes || !b.bytes) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

int aligned(std::initializer_list<Span> spans)
{
    for (const Span& s : spans)
        if (s.p && reinterpret_cast<uintptr_t>(s.p) % s.align) return NFAD_E_ALIGN;
    return NFAD_OK;
}

// Outputs must not overlap one another; an output may be one of the inputs of `same` exactly, and overlaps no other input.
int aliasing(std::initializer_list<Span> outs, std::initializer_list<Span> same, std::initializer_list<Span> others)
{
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        for (auto q = outs.begin(); q != o; ++q)
            if (overlap(*o, *q)) return NFAD_E_OVERLAP;
        for (const Span& s : same)
            if (overlap(*o, s) && !(o->p == s.p && o->bytes == s.bytes)) return NFAD_E_OVERLAP;
        for (const Span& s : others)
            if (overlap(*o, s)) return NFAD_E_OVERLAP;
    }
    return NFAD_OK;
}

// rows * cols elements: cols fits 31 bits, the bytes (and an fp32 copy's) a size_t
int element_count(size_t rows, size_t cols, size_t* n)
{
    if (cols >= (size_t(1) << 31)) return NFAD_E_TOO_LARGE;
    if (rows && cols > (~size_t(0) / 64) / rows) return NFAD_E_TOO_LARGE;
    *n = rows * cols;
    return NFAD_OK;
}

int finish(cudaError_t e)
{
    if (e == cudaSuccess) return NFAD_OK;
    nfad::note_cuda_error(e);
    return NFAD_E_CUDA;
}

// a product's sizes: every one below 2^31, and each tensor's bytes countable
int check_product(int kind, int dtype, size_t rows, size_t in, size_t out, size_t experts)
{
    if (kind < nfad::kNoAct || kind > 3) return NFAD_E_KIND;
    if (dtype != NFAD_BF16 && dtype != NFAD_F16) return NFAD_E_DTYPE;
    const size_t most = (size_t(1) << 31) - 256;                      // tile indices past the end stay below 2^31
    if (rows > most || in > most || out > most || experts > NFAD_MAX_EXPERTS) return NFAD_E_TOO_LARGE;
    if (out && in > (size_t(1) << 39) / out) return NFAD_E_TOO_LARGE; // bytes of one expert's weights: a tensor copy's largest stride
    if (experts == 0 && rows) return NFAD_E_VALUE;
    return NFAD_OK;
}

// the same for a layer with two weights [out, in]
int check_gated(int kind, int dtype, size_t rows, size_t in, size_t out, size_t experts)
{
    if (out >= (size_t(1) << 31)) return NFAD_E_TOO_LARGE;
    return check_product(kind, dtype, rows, in, 2 * out, experts);
}

int check_mask(const nfad_dropout_mask* mask, int dtype, nfad::DropoutArgs* a)
{
    if (!mask) return NFAD_E_NULL;
    if (dtype < 0 || dtype > 2) return NFAD_E_DTYPE;
    if (!(mask->p >= 0.0 && mask->p <= 1.0)) return NFAD_E_VALUE;
    const uint32_t dropped = uint32_t(rint(mask->p * 65536.0));
    a->dropped = dropped << 16;
    a->scale = dropped < 65536 ? float(65536.0 / double(65536 - dropped)) : 0.0f;          // 0: everything is dropped
    a->seed = mask->seed;
    a->offset = mask->offset;
    a->step = mask->step;
    return NFAD_OK;
}

int check_norm(const nfad_block_norm* norm, int dtype, size_t rows, size_t cols, size_t* n)
{
    if (!norm) return NFAD_E_NULL;
    if (norm->post < 0 || norm->post > 2 || norm->pre < 0 || norm->pre > 2) return NFAD_E_KIND;
    if (dtype < 0 || dtype > 2) return NFAD_E_DTYPE;
    int rc = element_count(rows, cols, n);
    if (rc) return rc;
    if (!(norm->eps > 0.0f) || isinf(norm->eps)) return NFAD_E_VALUE;
    if (norm->gate && (norm->gate_rows == 0 ? rows != 0 : rows % norm->gate_rows != 0)) return NFAD_E_VALUE;
    return NFAD_OK;
}

// ---- 8-bit floating point; weights: 1, or 2 for a gated layer

size_t f8_blocks(size_t n) { return (n + NFAD_F8_BLOCK - 1) / NFAD_F8_BLOCK; }

int f8_launch(int weights, int kind, int dtype, const void* xq, const float* x_scale, const void* wq, const float* w_scale, const void* bias, void* y,
              size_t rows, size_t in, size_t out, int b_ready, cudaStream_t st)
{
    nfad::ProdArgs g = {};
    g.a = xq; g.b = wq; g.bias = bias; g.a_scale = x_scale; g.b_scale = w_scale; g.out = y;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = 1; g.act = kind; g.b_ready = b_ready;
    return finish(weights == 2 ? nfad::launch_product_scaled_gated(dtype, g, st) : nfad::launch_product_scaled(dtype, g, st));
}

int check_f8(int weights, int kind, int dtype, size_t rows, size_t in, size_t out)
{
    return weights == 2 ? check_gated(kind, dtype, rows, in, out, 1) : check_product(kind, dtype, rows, in, out, 1);
}

int f8_product(int weights, int kind, int dtype, const unsigned char* xq, const float* x_scale, const unsigned char* wq, const float* w_scale,
               const void* bias, void* y, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    int rc = check_f8(weights, kind, dtype, rows, in, out);
    if (rc) return rc;
    if (rows == 0 || out == 0) return NFAD_OK;
    if ((in && (!xq || !wq || !x_scale || !w_scale)) || !y) return NFAD_E_NULL;
    const Span sx{xq, rows * in, 1}, sxs{x_scale, f8_blocks(in) * rows * 4, 4}, sw{wq, weights * out * in, 1},
        sws{w_scale, weights * f8_blocks(out) * f8_blocks(in) * 4, 4}, sb{bias, weights * out * 2, 2};
    const Span oy{y, rows * out * 2, 2};
    if ((rc = aligned({sx, sxs, sw, sws, sb, oy}))) return rc;
    if ((rc = aliasing({oy}, {}, {sx, sxs, sw, sws, sb}))) return rc;
    return f8_launch(weights, kind, dtype, xq, x_scale, wq, w_scale, bias, y, rows, in, out, 0, static_cast<cudaStream_t>(stream));
}

int f8_dynamic(int weights, int kind, int dtype, const void* x, const unsigned char* wq, const float* w_scale, const void* bias, void* y, void* scratch,
               size_t scratch_bytes, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    int rc = check_f8(weights, kind, dtype, rows, in, out);
    if (rc) return rc;
    if (rows == 0 || out == 0) return NFAD_OK;
    const size_t need = nfad_f8_linear_dynamic_scratch_bytes(rows, in);
    if ((in && (!x || !wq || !w_scale)) || !y || (need && !scratch)) return NFAD_E_NULL;
    const Span sx{x, rows * in * 2, 2}, sw{wq, weights * out * in, 1}, sws{w_scale, weights * f8_blocks(out) * f8_blocks(in) * 4, 4},
        sb{bias, weights * out * 2, 2};
    const Span oy{y, rows * out * 2, 2}, sc{need ? scratch : nullptr, need, 16};
    if ((rc = aligned({sx, sw, sws, sb, oy, sc}))) return rc;
    if (scratch_bytes < need) return NFAD_E_SCRATCH;
    if ((rc = aliasing({oy, sc}, {}, {sx, sw, sws, sb}))) return rc;
    unsigned char* q = static_cast<unsigned char*>(scratch);
    float* scale = reinterpret_cast<float*>(q + ((rows * in + 15) & ~size_t(15)));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (in && (rc = finish(nfad::launch_f8_groups(dtype, x, q, scale, rows, uint32_t(in), st)))) return rc;
    // the quantiser lets its successor start only after its own wait
    return f8_launch(weights, kind, dtype, q, scale, wq, w_scale, bias, y, rows, in, out, 1, st);
}

}  // namespace

extern "C" {

int nfad_block_norm_forward(const nfad_block_norm* norm, int dtype, const void* u, const void* r, void* s_out, void* h, float* stats,
                            size_t rows, size_t cols, nfad_stream_t stream)
{
    size_t n = 0;
    int rc = check_norm(norm, dtype, rows, cols, &n);
    if (rc) return rc;
    if (n == 0) return NFAD_OK;
    if (!u || (norm->pre != NFAD_NORM_NONE) != (h != nullptr) || (!s_out && !h)) return NFAD_E_NULL;
    const size_t es = elem_size(dtype), row = cols * es;
    const bool post = norm->post != NFAD_NORM_NONE, pre = norm->pre != NFAD_NORM_NONE;
    const Span su{u, n * es, es}, sr{r, n * es, es}, ss{s_out, n * es, es}, sh{h, n * es, es}, st{stats, rows * 16, 16};
    const Span pg{post ? norm->post_gain : nullptr, row, es}, pb{post ? norm->post_bias : nullptr, row, es},
        gt{norm->gate, norm->gate_rows * row, es}, qg{pre ? norm->pre_gain : nullptr, row, es}, qb{pre ? norm->pre_bias : nullptr, row, es};
    if ((rc = aligned({su, sr, ss, sh, st, pg, pb, gt, qg, qb}))) return rc;
    if ((rc = aliasing({ss, sh}, {su, sr}, {st, pg, pb, gt, qg, qb}))) return rc;
    if ((rc = aliasing({st}, {}, {su, sr, pg, pb, gt, qg, qb}))) return rc;
    nfad::NormForwardArgs a = {};
    a.u = u; a.r = r; a.post_gain = pg.p; a.post_bias = pb.p; a.gate = norm->gate; a.pre_gain = qg.p; a.pre_bias = qb.p;
    a.s = s_out; a.h = h; a.stats = reinterpret_cast<float4*>(stats);
    a.rows = rows; a.rows_per_gate = norm->gate ? rows / norm->gate_rows : rows;
    a.cols = uint32_t(cols);
    a.post = norm->post; a.pre = norm->pre;
    a.alpha = norm->residual_scale; a.eps = norm->eps; a.inv_cols = float(1.0 / double(cols));
    return finish(nfad::launch_norm_forward(dtype, a, static_cast<cudaStream_t>(stream)));
}

size_t nfad_block_norm_backward_scratch_bytes(int dtype, size_t rows, size_t cols)
{
    size_t n = 0, bytes = 0;
    if (dtype < 0 || dtype > 2 || element_count(rows, cols, &n) || n == 0) return 0;
    return finish(nfad::norm_backward_scratch(dtype, rows, cols, &bytes)) ? 0 : bytes;
}

int nfad_block_norm_backward(const nfad_block_norm* norm, int dtype, const void* grad_h, const void* grad_s, const void* u, const void* s,
                             const float* stats, void* grad_u, void* grad_r, const nfad_block_norm_grads* grads, void* scratch,
                             size_t scratch_bytes, size_t rows, size_t cols, nfad_stream_t stream)
{
    size_t n = 0;
    int rc = check_norm(norm, dtype, rows, cols, &n);
    if (rc) return rc;
    if (cols == 0) return NFAD_OK;
    const nfad_block_norm_grads none = {};
    const nfad_block_norm_grads& g = grads ? *grads : none;
    const bool post = norm->post != NFAD_NORM_NONE, pre = norm->pre != NFAD_NORM_NONE;
    if ((!post && (g.post_gain || g.post_bias)) || (!pre && (g.pre_gain || g.pre_bias)) || (!norm->gate && g.gate)) return NFAD_E_VALUE;
    if (n) {
        if (pre != (grad_h != nullptr) || (pre && !s) || (!pre && !grad_s) || ((post || norm->gate) && !u) || !stats || !grad_u || !scratch)
            return NFAD_E_NULL;
    }
    const size_t es = elem_size(dtype), row = cols * es, frow = cols * sizeof(float);
    const Span sgh{grad_h, n * es, es}, sgs{grad_s, n * es, es}, su{u, n * es, es}, ss{s, n * es, es}, st{stats, rows * 16, 16};
    const Span ogu{grad_u, n * es, es}, ogr{grad_r, n * es, es};
    const Span pg{post ? norm->post_gain : nullptr, row, es}, pb{post ? norm->post_bias : nullptr, row, es},
        gt{norm->gate, norm->gate_rows * row, es}, qg{pre ? norm->pre_gain : nullptr, row, es};
    const Span w1{g.post_gain, frow, 4}, w2{g.post_bias, frow, 4}, w3{g.gate, norm->gate_rows * frow, 4}, w4{g.pre_gain, frow, 4},
        w5{g.pre_bias, frow, 4};
    size_t need = 0;
    if (n && (rc = finish(nfad::norm_backward_scratch(dtype, rows, cols, &need)))) return rc;
    const Span sc{scratch, need, 16};
    if ((rc = aligned({sgh, sgs, su, ss, st, ogu, ogr, pg, pb, gt, qg, w1, w2, w3, w4, w5, sc}))) return rc;
    if (n && scratch_bytes < need) return NFAD_E_SCRATCH;
    if ((rc = aliasing({ogu, ogr}, {sgh, sgs, su, ss}, {st, pg, pb, gt, qg, w1, w2, w3, w4, w5, sc}))) return rc;
    if ((rc = aliasing({w1, w2, w3, w4, w5, sc}, {}, {sgh, sgs, su, ss, st, pg, pb, gt, qg}))) return rc;
    nfad::NormBackwardArgs a = {};
    a.grad_h = pre ? grad_h : nullptr; a.grad_s = grad_s; a.u = post || norm->gate ? u : nullptr; a.s = pre ? s : nullptr;
    a.post_gain = pg.p; a.post_bias = pb.p; a.gate = norm->gate; a.pre_gain = qg.p;
    a.stats = reinterpret_cast<const float4*>(stats);
    a.grad_u = grad_u; a.grad_r = grad_r;
    a.sums[nfad::kSumPreGain] = g.pre_gain; a.sums[nfad::kSumPreBias] = g.pre_bias;
    a.sums[nfad::kSumPostGain] = g.post_gain; a.sums[nfad::kSumPostBias] = g.post_bias;
    a.grad_gate = g.gate;
    a.rows = rows; a.rows_per_gate = norm->gate && norm->gate_rows ? rows / norm->gate_rows : rows;
    a.cols = uint32_t(cols);
    a.post = norm->post; a.pre = norm->pre;
    a.alpha = norm->residual_scale; a.inv_cols = float(1.0 / double(cols));
    if (n == 0 && g.gate && norm->gate_rows) {
        cudaError_t e = cudaMemsetAsync(g.gate, 0, norm->gate_rows * frow, static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return finish(e);
    }
    return finish(nfad::launch_norm_backward(dtype, a, scratch, static_cast<cudaStream_t>(stream)));
}

int nfad_dropout(int dtype, const nfad_dropout_mask* mask, const void* x, const void* residual, void* y, size_t n, nfad_stream_t stream)
{
    nfad::DropoutArgs a = {};
    int rc = check_mask(mask, dtype, &a);
    if (rc) return rc;
    if (n > ~size_t(0) / 64) return NFAD_E_TOO_LARGE;
    if (n == 0) return NFAD_OK;
    if (!x || !y) return NFAD_E_NULL;
    const size_t es = elem_size(dtype);
    const Span sx{x, n * es, es}, sr{residual, n * es, es}, ss{a.step, 8, 8}, oy{y, n * es, es};
    if ((rc = aligned({sx, sr, ss, oy}))) return rc;
    if ((rc = aliasing({oy}, {sx, sr}, {ss}))) return rc;
    a.x = x; a.other = residual; a.y = y; a.n = n;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.scale == 0.0f) {
        if (residual == y) return NFAD_OK;
        return finish(residual ? cudaMemcpyAsync(y, residual, n * es, cudaMemcpyDeviceToDevice, st) : cudaMemsetAsync(y, 0, n * es, st));
    }
    return finish(dtype == NFAD_F32 ? nfad::launch_dropout_f32(nfad::kNoAct, a, st) : nfad::launch_dropout_16(nfad::kNoAct, dtype, a, st));
}

int nfad_bias_act_dropout_forward(int kind, int dtype, const nfad_dropout_mask* mask, const void* x, const void* bias, void* y, void* dfdx, size_t rows,
                                  size_t cols, nfad_stream_t stream)
{
    if (kind < 0 || kind > 3) return NFAD_E_KIND;
    nfad::DropoutArgs a = {};
    size_t n = 0;
    int rc = check_mask(mask, dtype, &a);
    if (rc || (rc = element_count(rows, cols, &n))) return rc;
    if (n == 0) return NFAD_OK;
    if (!x || !y || !dfdx) return NFAD_E_NULL;
    const size_t es = elem_size(dtype);
    const Span sx{x, n * es, es}, sb{bias, cols * es, es}, ss{a.step, 8, 8}, oy{y, n * es, es}, od{dfdx, n * es, es};
    if ((rc = aligned({sx, sb, ss, oy, od}))) return rc;
    if ((rc = aliasing({oy, od}, {sx}, {sb, ss}))) return rc;
    a.x = x; a.other = bias; a.y = y; a.slope = dfdx; a.n = n; a.cols = uint32_t(cols);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.scale == 0.0f) {
        if ((rc = finish(cudaMemsetAsync(y, 0, n * es, st)))) return rc;
        return finish(cudaMemsetAsync(dfdx, 0, n * es, st));
    }
    return finish(dtype == NFAD_F32 ? nfad::launch_dropout_f32(kind, a, st) : nfad::launch_dropout_16(kind, dtype, a, st));
}

int nfad_expert_linear(int kind, int dtype, const void* x, const void* w, const void* bias, const int* offsets, void* y, void* dfdx, size_t rows,
                       size_t in, size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_product(kind, dtype, rows, in, out, experts);
    if (rc) return rc;
    if (kind == NFAD_NO_ACT && dfdx) return NFAD_E_VALUE;
    if (rows == 0 || out == 0) return NFAD_OK;
    if ((in && (!x || !w)) || !offsets || !y) return NFAD_E_NULL;
    const Span sx{x, rows * in * 2, 2}, sw{w, experts * out * in * 2, 2}, sb{bias, experts * out * 2, 2}, so{offsets, (experts + 1) * 4, 4};
    const Span oy{y, rows * out * 2, 2}, od{dfdx, rows * out * 2, 2};
    if ((rc = aligned({sx, sw, sb, so, oy, od}))) return rc;
    if ((rc = aliasing({oy, od}, {}, {sx, sw, sb, so}))) return rc;
    nfad::ProdArgs g = {};
    g.a = x; g.b = w; g.bias = bias; g.offsets = offsets; g.out = y; g.slope = dfdx;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = uint32_t(experts); g.act = kind;
    return finish(nfad::launch_product_forward(dtype, g, static_cast<cudaStream_t>(stream)));
}

size_t nfad_expert_act_backward_scratch_bytes(size_t rows, size_t out)
{
    size_t n = 0, bytes = 0;
    if (element_count(rows, out, &n) || n == 0) return 0;
    return finish(nfad::expert_act_backward_scratch(rows, out, &bytes)) ? 0 : bytes;
}

int nfad_expert_act_backward(int dtype, const void* grad_out, const void* dfdx, const int* offsets, void* grad_z, float* grad_bias, void* scratch,
                             size_t scratch_bytes, size_t rows, size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_product(nfad::kNoAct, dtype, rows, 0, out, experts);
    if (rc) return rc;
    if (out == 0 || experts == 0) return NFAD_OK;
    const size_t bytes = rows * out * 2;
    if (!offsets || (bytes && (!grad_out || (dfdx && !grad_z)))) return NFAD_E_NULL;
    size_t need = 0;
    if (grad_bias && bytes) {
        if ((rc = finish(nfad::expert_act_backward_scratch(rows, out, &need)))) return rc;
        if (!scratch) return NFAD_E_NULL;
        if (scratch_bytes < need) return NFAD_E_SCRATCH;
    }
    const Span sg{grad_out, bytes, 2}, sd{dfdx, bytes, 2}, so{offsets, (experts + 1) * 4, 4};
    const Span oz{grad_z, bytes, 2}, ob{grad_bias, experts * out * 4, 4}, sc{need ? scratch : nullptr, need, 16};
    if ((rc = aligned({sg, sd, so, oz, ob, sc}))) return rc;
    if ((rc = aliasing({oz}, {sg, sd}, {so, ob, sc}))) return rc;
    if ((rc = aliasing({ob, sc}, {}, {sg, sd, so}))) return rc;
    return finish(nfad::launch_expert_act_backward(dtype, grad_out, dfdx, offsets, grad_z, grad_bias, scratch, rows, uint32_t(out),
                                                   uint32_t(experts), static_cast<cudaStream_t>(stream)));
}

int nfad_expert_linear_backward_input(int dtype, const void* grad_z, const void* w, const int* offsets, const void* dfdx_x, void* grad_x, size_t rows,
                                      size_t in, size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_product(nfad::kNoAct, dtype, rows, in, out, experts);
    if (rc) return rc;
    if (rows == 0 || in == 0) return NFAD_OK;
    if ((out && (!grad_z || !w)) || !offsets || !grad_x) return NFAD_E_NULL;
    const Span sg{grad_z, rows * out * 2, 2}, sw{w, experts * out * in * 2, 2}, so{offsets, (experts + 1) * 4, 4}, sd{dfdx_x, rows * in * 2, 2};
    const Span ox{grad_x, rows * in * 2, 2};
    if ((rc = aligned({sg, sw, so, sd, ox}))) return rc;
    if ((rc = aliasing({ox}, {sd}, {sg, sw, so}))) return rc;
    nfad::ProdArgs g = {};
    g.a = grad_z; g.b = w; g.prev = dfdx_x; g.offsets = offsets; g.out = grad_x;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = uint32_t(experts); g.act = nfad::kNoAct;
    return finish(nfad::launch_product_input(dtype, g, static_cast<cudaStream_t>(stream)));
}

int nfad_expert_linear_backward_weight(int dtype, const void* grad_z, const void* x, const int* offsets, void* grad_w, size_t rows, size_t in,
                                       size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_product(nfad::kNoAct, dtype, rows, in, out, experts);
    if (rc) return rc;
    if (in == 0 || out == 0 || experts == 0) return NFAD_OK;
    if ((rows && (!grad_z || !x)) || !offsets || !grad_w) return NFAD_E_NULL;
    const Span sg{grad_z, rows * out * 2, 2}, sx{x, rows * in * 2, 2}, so{offsets, (experts + 1) * 4, 4}, ow{grad_w, experts * out * in * 2, 2};
    if ((rc = aligned({sg, sx, so, ow}))) return rc;
    if ((rc = aliasing({ow}, {}, {sg, sx, so}))) return rc;
    nfad::ProdArgs g = {};
    g.a = grad_z; g.b = x; g.offsets = offsets; g.out = grad_w;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = uint32_t(experts); g.act = nfad::kNoAct;
    return finish(nfad::launch_product_weight(dtype, g, static_cast<cudaStream_t>(stream)));
}

int nfad_expert_gated_linear(int kind, int dtype, const void* x, const void* w, const void* bias, const int* offsets, void* y, void* partials,
                             size_t rows, size_t in, size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_gated(kind, dtype, rows, in, out, experts);
    if (rc) return rc;
    if (rows == 0 || out == 0) return NFAD_OK;
    if ((in && (!x || !w)) || !offsets || !y) return NFAD_E_NULL;
    const Span sx{x, rows * in * 2, 2}, sw{w, experts * 2 * out * in * 2, 2}, sb{bias, experts * 2 * out * 2, 2}, so{offsets, (experts + 1) * 4, 4};
    const Span oy{y, rows * out * 2, 2}, op{partials, rows * 2 * out * 2, 2};
    if ((rc = aligned({sx, sw, sb, so, oy, op}))) return rc;
    if ((rc = aliasing({oy, op}, {}, {sx, sw, sb, so}))) return rc;
    nfad::ProdArgs g = {};
    g.a = x; g.b = w; g.bias = bias; g.offsets = offsets; g.out = y; g.slope = partials;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = uint32_t(experts); g.act = kind;
    return finish(nfad::launch_product_gated(dtype, g, static_cast<cudaStream_t>(stream)));
}

int nfad_expert_gated_backward(int dtype, const void* grad_out, const void* partials, const int* offsets, void* grad_z, float* grad_bias, void* scratch,
                               size_t scratch_bytes, size_t rows, size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_gated(nfad::kNoAct, dtype, rows, 0, out, experts);
    if (rc) return rc;
    if (out == 0 || experts == 0) return NFAD_OK;
    const size_t bytes = rows * out * 2;
    if (!offsets || (bytes && (!grad_out || !partials || !grad_z))) return NFAD_E_NULL;
    size_t need = 0;
    if (grad_bias && bytes) {
        if ((rc = finish(nfad::expert_act_backward_scratch(rows, 2 * out, &need)))) return rc;
        if (!scratch) return NFAD_E_NULL;
        if (scratch_bytes < need) return NFAD_E_SCRATCH;
    }
    const Span sg{grad_out, bytes, 2}, sp{partials, 2 * bytes, 2}, so{offsets, (experts + 1) * 4, 4};
    const Span oz{grad_z, 2 * bytes, 2}, ob{grad_bias, experts * 2 * out * 4, 4}, sc{need ? scratch : nullptr, need, 16};
    if ((rc = aligned({sg, sp, so, oz, ob, sc}))) return rc;
    if ((rc = aliasing({oz}, {sp}, {sg, so, ob, sc}))) return rc;
    if ((rc = aliasing({ob, sc}, {}, {sg, sp, so}))) return rc;
    return finish(nfad::launch_expert_gated_backward(dtype, grad_out, partials, offsets, grad_z, grad_bias, scratch, rows, uint32_t(out),
                                                     uint32_t(experts), static_cast<cudaStream_t>(stream)));
}

int nfad_expert_linear_backward_gated(int dtype, const void* grad_z, const void* w, const int* offsets, const void* partials, void* grad, size_t rows,
                                      size_t in, size_t out, size_t experts, nfad_stream_t stream)
{
    int rc = check_gated(nfad::kNoAct, dtype, rows, out, in, experts);            // `in` is the gated layer's width here
    if (rc) return rc;
    if (rows == 0 || in == 0) return NFAD_OK;
    if ((out && (!grad_z || !w)) || !offsets || !partials || !grad) return NFAD_E_NULL;
    const Span sg{grad_z, rows * out * 2, 2}, sw{w, experts * out * in * 2, 2}, so{offsets, (experts + 1) * 4, 4}, sp{partials, rows * 2 * in * 2, 2};
    const Span ox{grad, rows * 2 * in * 2, 2};
    if ((rc = aligned({sg, sw, so, sp, ox}))) return rc;
    if ((rc = aliasing({ox}, {sp}, {sg, sw, so}))) return rc;
    nfad::ProdArgs g = {};
    g.a = grad_z; g.b = w; g.prev = partials; g.offsets = offsets; g.out = grad;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = uint32_t(experts); g.act = nfad::kNoAct;
    return finish(nfad::launch_product_input_gated(dtype, g, static_cast<cudaStream_t>(stream)));
}

int nfad_i8_quantize_rows(int dtype, const void* x, signed char* q, float* scale, size_t rows, size_t cols, nfad_stream_t stream)
{
    if (dtype < 0 || dtype > 2) return NFAD_E_DTYPE;
    size_t n = 0;
    int rc = element_count(rows, cols, &n);
    if (rc) return rc;
    if (rows == 0) return NFAD_OK;
    if (rows >= (size_t(1) << 31)) return NFAD_E_TOO_LARGE;
    if ((n && (!x || !q)) || !scale) return NFAD_E_NULL;
    const size_t es = elem_size(dtype);
    const Span sx{x, n * es, es}, oq{q, n, 1}, os{scale, rows * 4, 4};
    if ((rc = aligned({sx, oq, os}))) return rc;
    if ((rc = aliasing({oq, os}, {}, {sx}))) return rc;
    return finish(nfad::launch_quantize_rows(dtype, x, q, scale, rows, uint32_t(cols), static_cast<cudaStream_t>(stream)));
}

int nfad_i8_linear(int kind, int dtype, const signed char* xq, const float* x_scale, const signed char* wq, const float* w_scale, const void* bias,
                   void* y, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    int rc = check_product(kind, dtype, rows, in, out, 1);
    if (rc) return rc;
    if (in > NFAD_I8_MAX_IN) return NFAD_E_TOO_LARGE;
    if (rows == 0 || out == 0) return NFAD_OK;
    if ((in && (!xq || !wq)) || !x_scale || !w_scale || !y) return NFAD_E_NULL;
    const Span sx{xq, rows * in, 1}, sxs{x_scale, rows * 4, 4}, sw{wq, out * in, 1}, sws{w_scale, out * 4, 4}, sb{bias, out * 2, 2};
    const Span oy{y, rows * out * 2, 2};
    if ((rc = aligned({sx, sxs, sw, sws, sb, oy}))) return rc;
    if ((rc = aliasing({oy}, {}, {sx, sxs, sw, sws, sb}))) return rc;
    nfad::ProdArgs g = {};
    g.a = xq; g.b = wq; g.bias = bias; g.a_scale = x_scale; g.b_scale = w_scale; g.out = y;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = 1; g.act = kind;
    return finish(nfad::launch_product_bytes(dtype, g, static_cast<cudaStream_t>(stream)));
}

size_t nfad_i8_linear_dynamic_scratch_bytes(size_t rows, size_t in)
{
    if (in > NFAD_I8_MAX_IN || rows >= (size_t(1) << 31)) return 0;
    return ((rows * in + 15) & ~size_t(15)) + rows * sizeof(float);   // the integers, then the scales
}

int nfad_i8_linear_dynamic(int kind, int dtype, const void* x, const signed char* wq, const float* w_scale, const void* bias, void* y, void* scratch,
                           size_t scratch_bytes, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    int rc = check_product(kind, dtype, rows, in, out, 1);
    if (rc) return rc;
    if (in > NFAD_I8_MAX_IN) return NFAD_E_TOO_LARGE;
    if (rows == 0 || out == 0) return NFAD_OK;
    if ((in && (!x || !wq)) || !w_scale || !y || !scratch) return NFAD_E_NULL;
    const size_t need = nfad_i8_linear_dynamic_scratch_bytes(rows, in);
    const Span sx{x, rows * in * 2, 2}, sw{wq, out * in, 1}, sws{w_scale, out * 4, 4}, sb{bias, out * 2, 2};
    const Span oy{y, rows * out * 2, 2}, sc{scratch, need, 16};
    if ((rc = aligned({sx, sw, sws, sb, oy, sc}))) return rc;
    if (scratch_bytes < need) return NFAD_E_SCRATCH;
    if ((rc = aliasing({oy, sc}, {}, {sx, sw, sws, sb}))) return rc;
    signed char* q = static_cast<signed char*>(scratch);
    float* scale = reinterpret_cast<float*>(q + ((rows * in + 15) & ~size_t(15)));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if ((rc = finish(nfad::launch_quantize_rows(dtype, x, q, scale, rows, uint32_t(in), st)))) return rc;
    nfad::ProdArgs g = {};
    g.a = q; g.b = wq; g.bias = bias; g.a_scale = scale; g.b_scale = w_scale; g.out = y;
    g.rows = rows; g.in = uint32_t(in); g.outs = uint32_t(out); g.experts = 1; g.act = kind;
    g.b_ready = 1;                                                    // the quantiser lets its successor start only after its own wait
    return finish(nfad::launch_product_bytes(dtype, g, st));
}

int nfad_f8_quantize_rows(int dtype, const void* x, unsigned char* q, float* scale, size_t rows, size_t cols, nfad_stream_t stream)
{
    if (dtype < 0 || dtype > 2) return NFAD_E_DTYPE;
    size_t n = 0;
    int rc = element_count(rows, cols, &n);
    if (rc) return rc;
    if (n == 0) return NFAD_OK;
    if (cols > (size_t(1) << 31) - 256) return NFAD_E_TOO_LARGE;
    if (!x || !q || !scale) return NFAD_E_NULL;
    const size_t es = elem_size(dtype);
    const Span sx{x, n * es, es}, oq{q, n, 1}, os{scale, f8_blocks(cols) * rows * 4, 4};
    if ((rc = aligned({sx, oq, os}))) return rc;
    if ((rc = aliasing({oq, os}, {}, {sx}))) return rc;
    return finish(nfad::launch_f8_groups(dtype, x, q, scale, rows, uint32_t(cols), static_cast<cudaStream_t>(stream)));
}

int nfad_f8_quantize_blocks(int dtype, const void* x, unsigned char* q, float* scale, size_t matrices, size_t rows, size_t cols, nfad_stream_t stream)
{
    if (dtype < 0 || dtype > 2) return NFAD_E_DTYPE;
    size_t n = 0, all = 0;
    int rc = element_count(rows, cols, &n);
    if (rc) return rc;
    if (n == 0 || matrices == 0) return NFAD_OK;
    if (rows > (size_t(1) << 31) - 256 || cols > (size_t(1) << 31) - 256 || matrices > (~size_t(0) / 64) / n) return NFAD_E_TOO_LARGE;
    all = matrices * n;
    if (!x || !q || !scale) return NFAD_E_NULL;
    const size_t es = elem_size(dtype);
    const Span sx{x, all * es, es}, oq{q, all, 1}, os{scale, matrices * f8_blocks(rows) * f8_blocks(cols) * 4, 4};
    if ((rc = aligned({sx, oq, os}))) return rc;
    if ((rc = aliasing({oq, os}, {}, {sx}))) return rc;
    return finish(nfad::launch_f8_blocks(dtype, x, q, scale, matrices, uint32_t(rows), uint32_t(cols), static_cast<cudaStream_t>(stream)));
}

int nfad_f8_linear(int kind, int dtype, const unsigned char* xq, const float* x_scale, const unsigned char* wq, const float* w_scale, const void* bias,
                   void* y, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    return f8_product(1, kind, dtype, xq, x_scale, wq, w_scale, bias, y, rows, in, out, stream);
}

int nfad_f8_gated_linear(int kind, int dtype, const unsigned char* xq, const float* x_scale, const unsigned char* wq, const float* w_scale, const void* bias,
                         void* y, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    return f8_product(2, kind, dtype, xq, x_scale, wq, w_scale, bias, y, rows, in, out, stream);
}

size_t nfad_f8_linear_dynamic_scratch_bytes(size_t rows, size_t in)
{
    if (rows >= (size_t(1) << 31) || in >= (size_t(1) << 31)) return 0;
    return ((rows * in + 15) & ~size_t(15)) + f8_blocks(in) * rows * sizeof(float);   // the bytes, then the scales
}

int nfad_f8_linear_dynamic(int kind, int dtype, const void* x, const unsigned char* wq, const float* w_scale, const void* bias, void* y, void* scratch,
                           size_t scratch_bytes, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    return f8_dynamic(1, kind, dtype, x, wq, w_scale, bias, y, scratch, scratch_bytes, rows, in, out, stream);
}

int nfad_f8_gated_linear_dynamic(int kind, int dtype, const void* x, const unsigned char* wq, const float* w_scale, const void* bias, void* y, void* scratch,
                                 size_t scratch_bytes, size_t rows, size_t in, size_t out, nfad_stream_t stream)
{
    return f8_dynamic(2, kind, dtype, x, wq, w_scale, bias, y, scratch, scratch_bytes, rows, in, out, stream);
}

int nfad_wait_faults(void)
{
    unsigned total = 0;
    for (auto count : {nfad::wait_faults_norm, nfad::product_faults_forward, nfad::product_faults_input, nfad::product_faults_weight, nfad::product_faults_bytes,
                       nfad::product_faults_gated, nfad::product_faults_input_gated, nfad::product_faults_scaled, nfad::product_faults_scaled_gated}) {
        unsigned n = 0;
        if (int rc = finish(count(&n))) return -rc;
        total += n;
    }
    return int(total & 0x7fffffff);
}

}  // extern "C"
