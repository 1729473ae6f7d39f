#include "nfad_scaled_launch.cuh"

namespace nfad {

cudaError_t launch_product_scaled_gated(int dtype, const ProdArgs& g, cudaStream_t st) { return launch_scaled_op<kProdScaledGated>(dtype, g, st); }
cudaError_t product_faults_scaled_gated(unsigned* n) { return product_faults_here(n); }

}  // namespace nfad
