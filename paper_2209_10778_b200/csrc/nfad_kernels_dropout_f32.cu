// Dropout of fp32 tensors, alone and behind an activation (contraction off, as in the fp32 activation pass).
#include "nfad_dropout.cuh"
#include "nfad_internal.h"

namespace nfad {

cudaError_t launch_dropout_f32(int kind, const DropoutArgs& a, cudaStream_t st) { return launch_dropout_store<StoreF32, Wide>(kind, a, st); }

}  // namespace nfad
