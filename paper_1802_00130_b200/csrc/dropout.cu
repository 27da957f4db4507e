// Dropout by a counter-based generator: the mask is a function of the element's number, the key and the step, and never stored.
//
// Bound by memory and, close behind, by the generator: ten rounds of two 32 x 32 -> 64 bit products and two three-way exclusive ors for four
// elements, 10 of the some 17 issue slots of an element, and the wide products have a pipe of their own busy for 46 us at 16384 x 4096 elements.  There, in bf16:
// 75 us with a residual (5.4 TB/s; an addition of the two alone takes 62), 66 us without (4.1 TB/s: the generator's bound).
// A thread asks for the next unit of 16 bytes (and the residual's) before it draws the numbers of one.
// Matrices without gaps are one long row, whatever their width; others go by units of a row where no unit straddles one, else by the
// generator's blocks of four elements.
#include <math.h>

#include "op_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

struct DropParams {
  int64_t rows, cols;
  const void *x, *res; void* y; int64_t ldx, ld_res, ldy;
  float scale; uint32_t last; int all;      // kept: words above `last`, or all of them; last = 2^32 - 1 keeps none
  uint32_t k0[10], k1[10];                  // the rounds' keys (as parameters they are operands of the rounds' instructions, and cost nothing)
  uint64_t step; const uint64_t* d_step;
};

// Philox4x32-10 (Salmon, Moraes, Dror and Shaw 2011).
__device__ __forceinline__ uint4 philox(uint4 c, const DropParams& p) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ p.k0[r], (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ p.k1[r], (uint32_t)a);
  }
  return c;
}
__device__ __forceinline__ bool kept(const DropParams& p, uint32_t word) { return p.all || word > p.last; }
__device__ __forceinline__ uint64_t step_of(const DropParams& p) {
  const uint64_t* const d = dep(p.d_step);
  return p.step + (d ? *d : 0);
}

// Units of 16 bytes; cols a multiple of their elements, or one row, whose last elements the first thread takes by themselves.  I: what numbers the units.
constexpr int kDropBlocks = 8;            // of an SM: 75 us where 6 take 76 and 4 80 (16384 x 4096 bf16 with a residual)
template <class T, bool ONE_ROW, class I>
__global__ void __launch_bounds__(256, kDropBlocks) dropout_units_kernel(const __grid_constant__ DropParams p) {
  constexpr int V = Pack<T>::V;
  grid_dep_wait();
  grid_dep_launch();
  const uint64_t step = step_of(p);
  const T* const x = (const T*)dep(p.x);
  const T* const res = (const T*)dep(p.res);
  T* const y = (T*)p.y;
  const I per_row = (I)(p.cols / V), units = (I)p.rows * per_row, stride = (I)gridDim.x * 256;
  const auto block = [&](I i) {
    return philox(make_uint4((uint32_t)i, sizeof(I) > 4 ? (uint32_t)((uint64_t)i >> 32) : 0u, (uint32_t)step, (uint32_t)(step >> 32)), p);
  };
  const auto at = [&](I q, int64_t ld) {
    if (ONE_ROW) return (int64_t)q * V;
    const I r = q / per_row;
    return (int64_t)r * ld + (int64_t)(q - r * per_row) * V;
  };
  const auto fetch = [&](I q, Pack<T>& v, Pack<T>& w) {
    v.w = *reinterpret_cast<const uint4*>(x + at(q, p.ldx));
    w.w = res ? *reinterpret_cast<const uint4*>(res + at(q, p.ld_res)) : make_uint4(0u, 0u, 0u, 0u);
  };
  I q = (I)blockIdx.x * 256 + threadIdx.x;
  Pack<T> v, w;
  if (q < units) fetch(q, v, w);
  while (q < units) {
    const I next = q + stride;
    Pack<T> vn, wn;
    if (next < units) fetch(next, vn, wn);
    float o[V];
#pragma unroll
    for (int b = 0; b < V / 4; ++b) {
      const uint4 r = block(q * (V / 4) + b);
      const uint32_t word[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) o[4 * b + e] = fmaf(kept(p, word[e]) ? v.get(4 * b + e) : 0.f, p.scale, w.get(4 * b + e));
    }
    v.set(o);
    *reinterpret_cast<uint4*>(y + at(q, p.ldy)) = v.w;
    v = vn; w = wn; q = next;
  }
  if (ONE_ROW && blockIdx.x == 0 && threadIdx.x == 0)
    for (int64_t c = (int64_t)units * V; c < p.cols; ++c) {
      const uint4 r = block((I)(c / 4));
      const uint32_t word[4] = {r.x, r.y, r.z, r.w};
      y[c] = from_f<T>(fmaf(kept(p, word[c & 3]) ? to_f(x[c]) : 0.f, p.scale, res ? to_f(res[c]) : 0.f));
    }
}

// Any layout: a thread takes the four elements of a block of the generator, wherever they lie.
template <class T>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropParams p) {
  grid_dep_wait();
  grid_dep_launch();
  const uint64_t step = step_of(p);
  const T* const x = (const T*)dep(p.x);
  const T* const res = (const T*)dep(p.res);
  T* const y = (T*)p.y;
  const int64_t n = p.rows * p.cols, blocks = (n + 3) / 4;
  for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * 256) {
    int64_t r = 4 * b / p.cols, c = 4 * b - r * p.cols;
    float v[4], w[4];
    int64_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool in = 4 * b + k < n;
      at[k] = in ? r * p.ldy + c : -1;
      v[k] = in ? to_f(x[r * p.ldx + c]) : 0.f;
      w[k] = in && res ? to_f(res[r * p.ld_res + c]) : 0.f;
      if (++c == p.cols) { c = 0; ++r; }
    }
    const uint4 q = philox(make_uint4((uint32_t)b, (uint32_t)((uint64_t)b >> 32), (uint32_t)step, (uint32_t)(step >> 32)), p);
    const uint32_t word[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (at[k] >= 0) y[at[k]] = from_f<T>(fmaf(kept(p, word[k]) ? v[k] : 0.f, p.scale, w[k]));
  }
}

template <class T>
cudaError_t run_dropout(DropParams a, int type, cudaStream_t st) {
  constexpr int V = Pack<T>::V;
  const bool one_row = a.rows == 1 || (a.ldx == a.cols && a.ldy == a.cols && (!a.res || a.ld_res == a.cols));
  if (one_row) { a.cols *= a.rows; a.rows = 1; a.ldx = a.ldy = a.ld_res = 0; }
  const bool wide = wide_ok(a.x, a.ldx, type) && wide_ok(a.y, a.ldy, type) && wide_ok(a.res, a.ld_res, type) && (one_row || a.cols % V == 0);
  const int64_t threads = wide ? a.rows * (a.cols / V) + 1 : (a.rows * a.cols + 3) / 4;
  const int64_t want = (threads + 255) / 256, most = 148 * (wide ? kDropBlocks : 8);
  const dim3 grid((unsigned)(want < most ? want : most));
  if (!wide) return launch_pdl_grid(dropout_kernel<T>, grid, 256, 0, st, a);
  // (below 2^30 units neither they, nor the generator's blocks in them, nor a step past the last pass 32 bits)
  if (threads < (int64_t(1) << 30)) return launch_pdl_grid(one_row ? dropout_units_kernel<T, true, uint32_t> : dropout_units_kernel<T, false, uint32_t>, grid, 256, 0, st, a);
  return launch_pdl_grid(one_row ? dropout_units_kernel<T, true, uint64_t> : dropout_units_kernel<T, false, uint64_t>, grid, 256, 0, st, a);
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
  const uint64_t threshold = (uint64_t)nearbyint(p * 4294967296.0);            // kept: words from here on
  a.all = threshold == 0; a.last = (uint32_t)(threshold - 1);
  a.scale = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.f;
  for (uint32_t r = 0; r < 10; ++r) { a.k0[r] = (uint32_t)key + r * 0x9E3779B9u; a.k1[r] = (uint32_t)(key >> 32) + r * 0xBB67AE85u; }
  a.step = step; a.d_step = d_step;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = type == GN_F32 ? run_dropout<float>(a, type, st) : type == GN_BF16 ? run_dropout<__nv_bfloat16>(a, type, st) : run_dropout<__half>(a, type, st);
  return op_done(e, errbuf, errbuf_len);
}
