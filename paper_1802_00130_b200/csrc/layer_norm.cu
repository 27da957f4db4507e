// Layer norm and its backward pass.
#include <math.h>

#include "op_common.cuh"

namespace gn {
namespace {

template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N]) {
  __shared__ float part[N][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < N; ++k)
    for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  __syncthreads();
  if (lane == 0)
    for (int k = 0; k < N; ++k) part[k][warp] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = lane < (blockDim.x >> 5) ? part[k][lane] : 0.f;
    for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  }
}

template <class T, class W>
__global__ void layer_norm_kernel(int64_t rows, int cols, const T* x, int64_t ldx, const W* w, const W* b, float eps, T* y, int64_t ldy,
                                  float* mean_out, float* rstd_out) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* xr = x + r * ldx;
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < cols; c += blockDim.x) s[0] += to_f(xr[c]);
    block_sum(s);
    const float m = s[0] / cols;
    float d[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < cols; c += blockDim.x) { const float v = to_f(xr[c]) - m; d[0] += v; d[1] += v * v; }
    block_sum(d);
    const float off = d[0] / cols, rstd = 1.f / sqrtf(d[1] / cols - off * off + eps);
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
      const float v = (to_f(xr[c]) - m - off) * rstd;
      y[r * ldy + c] = from_f<T>(v * (w ? to_f(w[c]) : 1.f) + (b ? to_f(b[c]) : 0.f));
    }
    if (threadIdx.x == 0) {
      if (mean_out) mean_out[r] = m + off;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

template <class T, class W>
__global__ void layer_norm_dx_kernel(int64_t rows, int cols, const T* dy, int64_t ld_dy, const T* x, int64_t ldx, const float* mean,
                                     const float* rstd, const W* w, const T* add, int64_t ld_add, T* dx, int64_t ld_dx) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float m = mean[r], rs = rstd[r];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
      const float g = to_f(dy[r * ld_dy + c]) * (w ? to_f(w[c]) : 1.f);
      s[0] += g; s[1] += g * (to_f(x[r * ldx + c]) - m) * rs;
    }
    block_sum(s);
    const float a = s[0] / cols, q = s[1] / cols;
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
      const float g = to_f(dy[r * ld_dy + c]) * (w ? to_f(w[c]) : 1.f), xh = (to_f(x[r * ldx + c]) - m) * rs;
      dx[r * ld_dx + c] = from_f<T>(rs * (g - a - xh * q) + (add ? to_f(add[r * ld_add + c]) : 0.f));
    }
  }
}

constexpr int kChunkRows = 256;
template <class T>
__global__ void layer_norm_dw_kernel(int64_t rows, int cols, const T* dy, int64_t ld_dy, const T* x, int64_t ldx, const float* mean,
                                     const float* rstd, float* part) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= cols) return;
  const int64_t r0 = (int64_t)blockIdx.y * kChunkRows, r1 = r0 + kChunkRows < rows ? r0 + kChunkRows : rows;
  float sw = 0.f, sb = 0.f;
  for (int64_t r = r0; r < r1; ++r) {
    const float g = to_f(dy[r * ld_dy + c]);
    sb += g; sw += g * (to_f(x[r * ldx + c]) - mean[r]) * rstd[r];
  }
  part[((int64_t)blockIdx.y * 2) * cols + c] = sw;
  part[((int64_t)blockIdx.y * 2 + 1) * cols + c] = sb;
}
template <class W>
__global__ void layer_norm_dw_final_kernel(int64_t chunks, int cols, const float* part, W* dw, W* db) {
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= cols) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t k = 0; k < chunks; ++k) { sw += part[2 * k * cols + c]; sb += part[(2 * k + 1) * cols + c]; }
  if (dw) dw[c] = from_f<W>(sw);
  if (db) db[c] = from_f<W>(sb);
}

struct NormCall {
  int64_t rows; int cols;
  const void *dy, *x, *w, *b, *add; int64_t ld_dy, ldx, ld_add;
  void *y, *dw, *db; int64_t ldy;
  float *mean, *rstd; float eps;
  void* ws; cudaStream_t st;
};

template <class T, class W>
void run_norm(const NormCall& a) {
  const int grid = (int)(a.rows < 4096 ? a.rows : 4096);
  layer_norm_kernel<T, W><<<grid, 256, 0, a.st>>>(a.rows, a.cols, (const T*)a.x, a.ldx, (const W*)a.w, (const W*)a.b, a.eps, (T*)a.y, a.ldy, a.mean, a.rstd);
}
template <class T, class W>
void run_norm_grad(const NormCall& a) {
  const int64_t chunks = (a.rows + kChunkRows - 1) / kChunkRows;
  if (a.dw || a.db) {
    if (chunks) layer_norm_dw_kernel<T><<<dim3((a.cols + 127) / 128, (unsigned)chunks), 128, 0, a.st>>>(a.rows, a.cols, (const T*)a.dy, a.ld_dy, (const T*)a.x, a.ldx, a.mean, a.rstd, (float*)a.ws);
    layer_norm_dw_final_kernel<W><<<(a.cols + 127) / 128, 128, 0, a.st>>>(chunks, a.cols, (const float*)a.ws, (W*)a.dw, (W*)a.db);
  }
  if (a.y && a.rows) {
    const int grid = (int)(a.rows < 4096 ? a.rows : 4096);
    layer_norm_dx_kernel<T, W><<<grid, 256, 0, a.st>>>(a.rows, a.cols, (const T*)a.dy, a.ld_dy, (const T*)a.x, a.ldx, a.mean, a.rstd, (const W*)a.w, (const T*)a.add, a.ld_add, (T*)a.y, a.ldy);
  }
}

template <template <class, class> class F, class... A>
void by_types(int type, int wtype, const NormCall& a) {
  if (type == GN_F32) F<float, float>::run(a);
  else if (type == GN_BF16) { if (wtype == GN_F32) F<__nv_bfloat16, float>::run(a); else F<__nv_bfloat16, __nv_bfloat16>::run(a); }
  else { if (wtype == GN_F32) F<__half, float>::run(a); else F<__half, __half>::run(a); }
}
template <class T, class W> struct Norm { static void run(const NormCall& a) { run_norm<T, W>(a); } };
template <class T, class W> struct NormGrad { static void run(const NormCall& a) { run_norm_grad<T, W>(a); } };

constexpr int kMaxCols = 1 << 20;
const char* norm_sizes(int type, int wtype, int64_t rows, int cols) {
  if (!type_ok(type)) return "type is not a gn_dtype";
  if (wtype != type && wtype != GN_F32) return "the weight's type must be the matrices' or GN_F32";
  if (rows < 0 || rows >= (int64_t(1) << 31)) return "rows must be in [0, 2^31)";
  if (cols < 1 || cols > kMaxCols) return "cols must be in [1, 2^20]";
  return nullptr;
}
bool vec_ok(const void* p, int type) { return (uintptr_t)p % (uintptr_t)type_bytes(type) == 0; }

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" gn_status gn_layer_norm(gn_dtype type, gn_dtype wtype, int64_t rows, int32_t cols, const void* d_x, int64_t ldx,
                                   const void* d_weight, const void* d_bias, double eps, void* d_y, int64_t ldy, float* d_mean,
                                   float* d_rstd, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = norm_sizes(type, wtype, rows, cols);
  if (!why && !(eps >= 0.0 && eps <= 1e30)) why = "eps must be a number >= 0";
  if (!why && !vec_ok(d_weight, wtype)) why = "weight is not aligned to its type";
  if (!why && !vec_ok(d_bias, wtype)) why = "bias is not aligned to its type";
  if (!why && rows > 0 && !mat_ok(d_x, ldx, cols, type)) why = "x: null, misaligned, or a leading dimension below cols";
  if (!why && rows > 0 && !mat_ok(d_y, ldy, cols, type)) why = "y: null, misaligned, or a leading dimension below cols";
  if (!why && rows > 0 && d_x == d_y && ldx != ldy) why = "y in the place of x needs x's leading dimension";
  if (!why && (!vec_ok(d_mean, GN_F32) || !vec_ok(d_rstd, GN_F32))) why = "mean or rstd is not aligned to a float";
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  if (rows == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  NormCall a = {};
  a.rows = rows; a.cols = cols; a.x = d_x; a.ldx = ldx; a.w = d_weight; a.b = d_bias; a.eps = (float)eps;
  a.y = d_y; a.ldy = ldy; a.mean = d_mean; a.rstd = d_rstd; a.st = (cudaStream_t)cuda_stream;
  by_types<Norm>(type, wtype, a);
  return op_done(cudaSuccess, errbuf, errbuf_len);
}

extern "C" int64_t gn_layer_norm_grad_workspace(int64_t rows, int32_t cols) {
  if (rows < 0 || cols < 1 || cols > kMaxCols) return -1;
  return (rows + kChunkRows - 1) / kChunkRows * 2 * cols * 4 + 16;
}

extern "C" gn_status gn_layer_norm_grad(gn_dtype type, gn_dtype wtype, int64_t rows, int32_t cols, const void* d_dy, int64_t ld_dy,
                                        const void* d_x, int64_t ldx, const float* d_mean, const float* d_rstd, const void* d_weight,
                                        const void* d_add, int64_t ld_add, void* d_dx, int64_t ld_dx, void* d_dweight, void* d_dbias,
                                        void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = norm_sizes(type, wtype, rows, cols);
  if (!why && (!vec_ok(d_weight, wtype) || !vec_ok(d_dweight, wtype) || !vec_ok(d_dbias, wtype))) why = "a weight vector is not aligned to its type";
  if (!why && rows > 0) {
    if (!mat_ok(d_dy, ld_dy, cols, type)) why = "dy: null, misaligned, or a leading dimension below cols";
    else if (!mat_ok(d_x, ldx, cols, type)) why = "x: null, misaligned, or a leading dimension below cols";
    else if (!d_mean || !d_rstd || !vec_ok(d_mean, GN_F32) || !vec_ok(d_rstd, GN_F32)) why = "mean or rstd: null or misaligned";
    else if (d_add && !mat_ok(d_add, ld_add, cols, type)) why = "add: misaligned, or a leading dimension below cols";
    else if (d_dx && !mat_ok(d_dx, ld_dx, cols, type)) why = "dx: misaligned, or a leading dimension below cols";
    else if (d_dx && (d_dx == d_x || (d_dx == d_dy && ld_dx != ld_dy) || (d_dx == d_add && ld_dx != ld_add))) why = "dx in the place of dy or add needs its leading dimension, and x is not its place";
  }
  if (!why && (!d_ws || ((uintptr_t)d_ws & 15) || ws_bytes < gn_layer_norm_grad_workspace(rows, cols))) why = "workspace: null, not 16-byte aligned or too small";
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  NormCall a = {};
  a.rows = rows; a.cols = cols; a.dy = d_dy; a.ld_dy = ld_dy; a.x = d_x; a.ldx = ldx; a.w = d_weight; a.add = d_add; a.ld_add = ld_add;
  a.y = d_dx; a.ldy = ld_dx; a.dw = d_dweight; a.db = d_dbias; a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
  a.ws = d_ws; a.st = (cudaStream_t)cuda_stream;
  by_types<NormGrad>(type, wtype, a);
  return op_done(cudaSuccess, errbuf, errbuf_len);
}
