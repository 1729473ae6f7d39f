#include "nfad_product_launch.cuh"

namespace nfad {

cudaError_t launch_product_bytes(int dtype, const ProdArgs& g, cudaStream_t st) { return launch_product_op<kProdBytes>(dtype, g, st); }
cudaError_t product_faults_bytes(unsigned* n) { return product_faults_here(n); }

}  // namespace nfad
