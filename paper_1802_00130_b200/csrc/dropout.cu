// Dropout by a counter-based generator: the mask is a function of the element's number, the key and the step, and never stored.
#include <math.h>

#include "op_common.cuh"

namespace gn {
namespace {

struct DropParams {
  int64_t rows; int cols;
  const void *x, *res; void* y; int64_t ldx, ld_res, ldy;
  float scale; uint64_t threshold;          // keep iff word >= threshold (2^32: never)
  uint32_t k0, k1; uint64_t step; const uint64_t* d_step;
};

// Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011): ten rounds of two 32 x 32 -> 64 bit products.
__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return c;
}

template <class T>
__global__ void dropout_kernel(const DropParams p) {
  const uint64_t step = p.step + (p.d_step ? *p.d_step : 0);
  const int64_t n = p.rows * p.cols, blocks = (n + 3) / 4;
  for (int64_t b = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * blockDim.x) {
    const uint4 w = philox(make_uint4((uint32_t)b, (uint32_t)(b >> 32), (uint32_t)step, (uint32_t)(step >> 32)), p.k0, p.k1);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
    for (int k = 0; k < 4 && 4 * b + k < n; ++k) {
      const int64_t r = (4 * b + k) / p.cols, c = (4 * b + k) % p.cols;
      float v = word[k] >= p.threshold ? to_f(((const T*)p.x)[r * p.ldx + c]) * p.scale : 0.f;
      if (p.res) v += to_f(((const T*)p.res)[r * p.ld_res + c]);
      ((T*)p.y)[r * p.ldy + c] = from_f<T>(v);
    }
  }
}

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" gn_status gn_dropout(gn_dtype type, int64_t rows, int32_t cols, const void* d_x, int64_t ldx, const void* d_residual,
                                int64_t ld_res, void* d_y, int64_t ldy, double p, uint64_t key, uint64_t step, const uint64_t* d_step,
                                void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = nullptr;
  if (!type_ok(type)) why = "type is not a gn_dtype";
  else if (rows < 0 || rows >= (int64_t(1) << 31)) why = "rows must be in [0, 2^31)";
  else if (cols < 1) why = "cols must be >= 1";
  else if (!(p >= 0.0 && p <= 1.0)) why = "p must be in [0, 1]";
  else if ((uintptr_t)d_step & 7) why = "d_step is not aligned to 8 bytes";
  else if (rows > 0) {
    if (!mat_ok(d_x, ldx, cols, type)) why = "x: null, misaligned, or a leading dimension below cols";
    else if (d_residual && !mat_ok(d_residual, ld_res, cols, type)) why = "residual: misaligned, or a leading dimension below cols";
    else if (!mat_ok(d_y, ldy, cols, type)) why = "y: null, misaligned, or a leading dimension below cols";
    else if ((d_y == d_x && ldy != ldx) || (d_y == d_residual && ldy != ld_res)) why = "y in the place of x or the residual needs its leading dimension";
  }
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  if (rows == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  DropParams a = {};
  a.rows = rows; a.cols = cols; a.x = d_x; a.ldx = ldx; a.res = d_residual; a.ld_res = ld_res; a.y = d_y; a.ldy = ldy;
  a.threshold = (uint64_t)nearbyint(p * 4294967296.0);
  a.scale = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.f;
  a.k0 = (uint32_t)key; a.k1 = (uint32_t)(key >> 32); a.step = step; a.d_step = d_step;
  const int64_t want = ((rows * cols + 3) / 4 + 255) / 256;
  const int grid = (int)(want < 148 * 8 ? want : 148 * 8);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (type == GN_F32) dropout_kernel<float><<<grid, 256, 0, st>>>(a);
  else if (type == GN_BF16) dropout_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
  else dropout_kernel<__half><<<grid, 256, 0, st>>>(a);
  return op_done(cudaSuccess, errbuf, errbuf_len);
}
