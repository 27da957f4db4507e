// Products with 4-bit weights: the kernels of one type.
#include "weight4_product.cuh"

namespace gn {

namespace {
__global__ void __launch_bounds__(256) parts_kernel(const float* x, int64_t ldx, int64_t rows, int cols, __nv_bfloat16* to, int64_t ld_out) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t work = rows * ld_out;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / ld_out, c = i - r * ld_out;
    __nv_bfloat16 o[3];
    split_parts<3>(c < cols ? x[r * ldx + c] : 0.f, o);
#pragma unroll
    for (int j = 0; j < 3; ++j) to[j * work + i] = o[j];
  }
}
}  // namespace

cudaError_t launch_parts(const float* x, int64_t ldx, int64_t rows, int cols, void* to, int64_t ld_out, cudaStream_t st) {
  const int64_t want = (rows * ld_out + 255) / 256, most = (int64_t)num_sms() * 8;
  return launch_pdl(parts_kernel, (int)(want < most ? want : most), 256, 0, st, x, ldx, rows, cols, (__nv_bfloat16*)to, ld_out);
}

cudaError_t launch_product4_f32(const Product4& p, cudaStream_t st) {
  return p.gate ? launch_product4_of<float, __nv_bfloat16, 3, 2>(p, st) : launch_product4_of<float, __nv_bfloat16, 3, 1>(p, st);
}

}  // namespace gn
