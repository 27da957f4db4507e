// Products with 4-bit weights: the kernels of one type.
#include "weight4_product.cuh"

namespace gn {

namespace {
template <class T>
__global__ void __launch_bounds__(256) operands_kernel(const T* x, int64_t ldx, int64_t rows, int cols, uint16_t* to, int64_t ld_out) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t work = rows * ld_out;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / ld_out, c = i - r * ld_out;
    const T v = c < cols ? x[r * ldx + c] : T(0);
    if constexpr (sizeof(T) == 2) {
      to[i] = v;
    } else {
      __nv_bfloat16 o[3];
      split_parts<3>(v, o);
#pragma unroll
      for (int j = 0; j < 3; ++j) to[j * work + i] = __bfloat16_as_ushort(o[j]);
    }
  }
}
}  // namespace

cudaError_t launch_operands(const void* x, int64_t ldx, int64_t rows, int cols, int bytes, void* to, cudaStream_t st) {
  const int64_t ld_out = (cols + 7) / 8 * 8, want = (rows * ld_out + 255) / 256, most = (int64_t)num_sms() * 8;
  const int grid = (int)(want < most ? want : most);
  if (bytes == 2) return launch_pdl(operands_kernel<uint16_t>, grid, 256, 0, st, (const uint16_t*)x, ldx, rows, cols, (uint16_t*)to, ld_out);
  return launch_pdl(operands_kernel<float>, grid, 256, 0, st, (const float*)x, ldx, rows, cols, (uint16_t*)to, ld_out);
}

cudaError_t launch_product4_f32(const Product4& p, cudaStream_t st) {
  return p.gate ? launch_product4_of<float, __nv_bfloat16, 3, 2>(p, st) : launch_product4_of<float, __nv_bfloat16, 3, 1>(p, st);
}

}  // namespace gn
