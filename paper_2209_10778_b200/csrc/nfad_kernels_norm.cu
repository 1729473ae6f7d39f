// The norms before and after a block, every storage type.  fp32 arithmetic throughout; nothing here depends on how
// multiplies and adds contract.
#include "nfad_norm.cuh"

namespace nfad {

cudaError_t launch_norm_forward(int dtype, const NormForwardArgs& a, cudaStream_t st)
{
    switch (dtype) {
    case kF32:  return launch_norm_forward<StoreF32>(a, st);
    case kBF16: return launch_norm_forward<StoreBF16>(a, st);
    case kF16:  return launch_norm_forward<StoreF16>(a, st);
    }
    return cudaErrorInvalidValue;
}

cudaError_t launch_norm_backward(int dtype, const NormBackwardArgs& a, void* scratch, cudaStream_t st)
{
    switch (dtype) {
    case kF32:  return launch_norm_backward<StoreF32>(a, scratch, st);
    case kBF16: return launch_norm_backward<StoreBF16>(a, scratch, st);
    case kF16:  return launch_norm_backward<StoreF16>(a, scratch, st);
    }
    return cudaErrorInvalidValue;
}

cudaError_t norm_backward_scratch(int dtype, size_t rows, size_t cols, size_t* bytes)
{
    DeviceInfo di;
    cudaError_t e = device_info(&di);
    if (e != cudaSuccess) return e;
    *bytes = dtype == kF32 ? norm_backward_scratch_bytes<StoreF32>(rows, cols, di.sm_count)
                           : norm_backward_scratch_bytes<StoreBF16>(rows, cols, di.sm_count);
    return cudaSuccess;
}

cudaError_t wait_faults_norm(unsigned* n) { return cudaMemcpyFromSymbol(n, g_norm_faults, sizeof *n); }

}  // namespace nfad
