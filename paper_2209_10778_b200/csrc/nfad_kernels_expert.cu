// What stands beside the matrix products: Eq. 4 on rows grouped by expert, and rows in 8-bit integers.  Products and
// sums are explicitly rounded intrinsics.
#include "nfad_bytes.cuh"
#include "nfad_expert.cuh"

namespace nfad {

cudaError_t launch_expert_act_backward(int dtype, const void* g, const void* d, const int* offsets, void* gz, float* grad_bias, void* scratch,
                                       size_t rows, uint32_t cols, uint32_t experts, cudaStream_t st)
{
    ExpertActArgs a = {};
    a.g = g; a.d = d; a.gz = gz; a.grad_bias = grad_bias; a.partial = static_cast<float*>(scratch);
    a.offsets = offsets; a.rows = rows; a.cols = cols; a.experts = experts;
    return dtype == kBF16 ? launch_expert_act<StoreBF16>(a, st) : launch_expert_act<StoreF16>(a, st);
}

cudaError_t expert_act_backward_scratch(size_t rows, size_t cols, size_t* bytes)
{
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    *bytes = expert_act_scratch_bytes(rows, cols, di.sm_count);
    return cudaSuccess;
}

cudaError_t launch_quantize_rows(int dtype, const void* x, signed char* q, float* scale, size_t rows, uint32_t cols, cudaStream_t st)
{
    switch (dtype) {
    case kF32:  return launch_quantize<StoreF32>(x, q, scale, rows, cols, st);
    case kBF16: return launch_quantize<StoreBF16>(x, q, scale, rows, cols, st);
    case kF16:  return launch_quantize<StoreF16>(x, q, scale, rows, cols, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace nfad
