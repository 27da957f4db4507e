// Products with 4-bit weights: the kernels of one type.
#include "weight4_product.cuh"

namespace gn {

cudaError_t launch_product4_f32(const Product4& p, cudaStream_t st) {
  return launch_product4_x<float, float, 3>(p, st);
}

}  // namespace gn
