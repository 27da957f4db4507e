// Products with 4-bit weights: the kernels of one type.
#include "weight4_product.cuh"

namespace gn {

cudaError_t launch_product4_bf16(const Product4& p, cudaStream_t st) {
  return p.x32 ? launch_product4_x<__nv_bfloat16, float, 2>(p, st) : launch_product4_x<__nv_bfloat16, __nv_bfloat16, 1>(p, st);
}

}  // namespace gn
