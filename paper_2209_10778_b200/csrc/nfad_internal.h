// nfad_internal.h -- launchers behind the C-ABI, one set per translation unit:
// the fp32-storage kernels are built with floating-point contraction off (their
// compensated arithmetic depends on it), the 16-bit-storage kernels with it on.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <string>

namespace nfad {

enum Kind { kGeluErf = 0, kGeluTanh = 1, kSwish = 2, kMish = 3 };
enum DType { kF32 = 0, kBF16 = 1, kF16 = 2 };

// Which map to run.  Tensor order in `in` / `out` is fixed per op:
//   kOpForward        in {x}            out {y, dfdx}
//   kOpForwardInfer   in {x}            out {y}
//   kOpBackward       in {g, dfdx}      out {gin}
//   kOpConvBackward   in {g, x}         out {gin}
//   kOpRecompute1     in {x}            out {h}
//   kOpRecompute2     in {g, x, h}      out {gin}
//   kOpProbe11/12/21  in {a[, b]}       out {o0[, o1]}   (traffic probes: fp32 storage only)
//   kOpForwardStrict  in {x}            out {y, dfdx}    (fp32 storage only)
//   kOpProbe10        in {a}            out {sink}       (read-only probe; sink: one word, written only on a checksum match)
//   kOpProbe01        in {}             out {o0}         (write-only probe)
enum OpCode { kOpForward, kOpForwardInfer, kOpBackward, kOpConvBackward, kOpRecompute1, kOpRecompute2,
              kOpProbe11, kOpProbe12, kOpProbe21, kOpForwardStrict, kOpProbe10, kOpProbe01 };

cudaError_t launch_f32(OpCode op, int kind, const void* const* in, void* const* out, size_t n, cudaStream_t st);
cudaError_t launch_16(OpCode op, int kind, int dtype, const void* const* in, void* const* out, size_t n, cudaStream_t st);

// Run-time FAD sequences (nfad_seq.cuh): the program as plain arrays, so that this header
// stays free of device code.
constexpr int kSeqMaxOpsHost = 32;
struct SeqProgramHost { int n_ops; int op[kSeqMaxOpsHost], a[kSeqMaxOpsHost], b[kSeqMaxOpsHost], dst[kSeqMaxOpsHost]; float c[kSeqMaxOpsHost]; };

cudaError_t launch_seq_forward(const SeqProgramHost& p, int dtype, const void* x, void* const* y, void* const* d, int m, size_t n,
                               cudaStream_t st);
// The same sequence compiled at run time into one kernel (nfad_jit.cu).  cudaErrorNotSupported: not available here.
cudaError_t launch_seq_forward_compiled(const SeqProgramHost& p, int dtype, const void* x, void* const* y, void* const* d, int m,
                                        size_t n, cudaStream_t st);
int seq_executor_mode();                 // 0 automatic, 1 interpreter only, 2 compiled only
void seq_set_executor_mode(int mode);
int seq_last_executor();                 // of the calling thread: 0 none yet, 1 interpreter, 2 compiled
void seq_note_executor(int which);
const char* seq_jit_log();
std::string seq_generate_source(const SeqProgramHost& p, int dtype, int m);   // what the compiled executor would compile
cudaError_t launch_seq_backward(int dtype, const void* const* g, const void* const* d, int m, void* gin, size_t n, cudaStream_t st);
cudaError_t launch_ew(int op, int backward, float c, int dtype, const void* const* in, void* const* out, size_t n, cudaStream_t st);

// CTAs for a launch that takes n elements one by one with a grid-stride loop: enough to fill the current device
// (32 CTAs of `block` threads per SM at most), never more than the elements need.
unsigned edge_grid_blocks(size_t n, unsigned block);

// Records the cudaError_t behind an NFAD_E_CUDA of the calling thread (what nfad_last_cuda_error() returns).
void note_cuda_error(cudaError_t e);

// The pass fused with its producer's bias (nfad_bias.cuh).  x, y, d, g, gin: [rows, cols] row-major; bias: [cols].
cudaError_t launch_bias_forward_f32(int kind, const void* x, const void* bias, void* y, void* d, size_t rows, size_t cols,
                                    cudaStream_t st);
cudaError_t launch_bias_forward_16(int kind, int dtype, const void* x, const void* bias, void* y, void* d, size_t rows,
                                   size_t cols, cudaStream_t st);
cudaError_t launch_bias_backward(int dtype, const void* g, const void* d, void* gin, float* grad_bias, void* scratch,
                                 size_t rows, size_t cols, cudaStream_t st);
cudaError_t bias_backward_scratch(int dtype, size_t rows, size_t cols, size_t* bytes);   // on the current device

// Dropout (nfad_dropout.cuh); kind -1: no activation.
struct DropoutArgs;
cudaError_t launch_dropout_f32(int kind, const DropoutArgs& a, cudaStream_t st);
cudaError_t launch_dropout_16(int kind, int dtype, const DropoutArgs& a, cudaStream_t st);

// The norms around a block (nfad_norm.cuh).
struct NormForwardArgs;
struct NormBackwardArgs;
cudaError_t launch_norm_forward(int dtype, const NormForwardArgs& a, cudaStream_t st);
cudaError_t launch_norm_backward(int dtype, const NormBackwardArgs& a, void* scratch, cudaStream_t st);
cudaError_t norm_backward_scratch(int dtype, size_t rows, size_t cols, size_t* bytes);   // on the current device

// Matrix products (nfad_product.cuh), what stands beside them (nfad_expert.cuh, nfad_bytes.cuh), and the CTAs that gave up waiting.
struct ProdArgs;
cudaError_t launch_product_forward(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_input(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_weight(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_bytes(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_scaled(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_scaled_gated(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_gated(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t launch_product_input_gated(int dtype, const ProdArgs& g, cudaStream_t st);
cudaError_t wait_faults_norm(unsigned* n);
cudaError_t product_faults_forward(unsigned* n);
cudaError_t product_faults_input(unsigned* n);
cudaError_t product_faults_weight(unsigned* n);
cudaError_t product_faults_bytes(unsigned* n);
cudaError_t product_faults_scaled(unsigned* n);
cudaError_t product_faults_scaled_gated(unsigned* n);
cudaError_t product_faults_gated(unsigned* n);
cudaError_t product_faults_input_gated(unsigned* n);
cudaError_t launch_expert_act_backward(int dtype, const void* g, const void* d, const int* offsets, void* gz, float* grad_bias, void* scratch,
                                       size_t rows, uint32_t cols, uint32_t experts, cudaStream_t st);
cudaError_t launch_expert_gated_backward(int dtype, const void* g, const void* d, const int* offsets, void* gz, float* grad_bias, void* scratch,
                                         size_t rows, uint32_t cols, uint32_t experts, cudaStream_t st);
cudaError_t expert_act_backward_scratch(size_t rows, size_t cols, size_t* bytes);        // on the current device
cudaError_t launch_f8_groups(int dtype, const void* x, unsigned char* q, float* scale, size_t rows, uint32_t cols, cudaStream_t st);
cudaError_t launch_f8_blocks(int dtype, const void* x, unsigned char* q, float* scale, size_t matrices, uint32_t rows, uint32_t cols, cudaStream_t st);
cudaError_t launch_quantize_rows(int dtype, const void* x, signed char* q, float* scale, size_t rows, uint32_t cols, cudaStream_t st);

}  // namespace nfad
