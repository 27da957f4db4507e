// Products with 4-bit weights: the kernels of one type.
#include "weight4_product.cuh"

namespace gn {

cudaError_t launch_product4_bf16(const Product4& p, cudaStream_t st) {
  if (p.gate) return launch_product4_of<__nv_bfloat16, __nv_bfloat16, 1, 2>(p, st);
  return p.in_parts ? launch_product4_of<__nv_bfloat16, __nv_bfloat16, 2, 1>(p, st) : launch_product4_of<__nv_bfloat16, __nv_bfloat16, 1, 1>(p, st);
}

}  // namespace gn
