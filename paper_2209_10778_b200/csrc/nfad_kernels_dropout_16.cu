// Dropout of 16-bit tensors, alone and behind an activation (contraction on, as in the 16-bit activation pass).
#include "nfad_dropout.cuh"
#include "nfad_internal.h"

namespace nfad {

cudaError_t launch_dropout_16(int kind, int dtype, const DropoutArgs& a, cudaStream_t st)
{
    if (dtype == kBF16) return launch_dropout_store<StoreBF16, Fast>(kind, a, st);
    if (dtype == kF16) return launch_dropout_store<StoreF16, Fast>(kind, a, st);
    return cudaErrorInvalidValue;
}

}  // namespace nfad
