// Values to 8-bit floating point by blocks of 128.  Products and quotients are explicitly rounded intrinsics.
#include "nfad_blocks.cuh"
#include "nfad_internal.h"

namespace nfad {

cudaError_t launch_f8_groups(int dtype, const void* x, unsigned char* q, float* scale, size_t rows, uint32_t cols, cudaStream_t st)
{
    switch (dtype) {
    case kF32:  return launch_quantize_groups<StoreF32>(x, q, scale, rows, cols, st);
    case kBF16: return launch_quantize_groups<StoreBF16>(x, q, scale, rows, cols, st);
    case kF16:  return launch_quantize_groups<StoreF16>(x, q, scale, rows, cols, st);
    }
    return cudaErrorInvalidValue;
}

cudaError_t launch_f8_blocks(int dtype, const void* x, unsigned char* q, float* scale, size_t matrices, uint32_t rows, uint32_t cols, cudaStream_t st)
{
    switch (dtype) {
    case kF32:  return launch_quantize_blocks<StoreF32>(x, q, scale, matrices, rows, cols, st);
    case kBF16: return launch_quantize_blocks<StoreBF16>(x, q, scale, matrices, rows, cols, st);
    case kF16:  return launch_quantize_blocks<StoreF16>(x, q, scale, matrices, rows, cols, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace nfad
