// Layer norm and its backward pass, each in one pass over the data: memory bound, so a row is read once, kept in registers as it is
// stored, and written once.
//
// Forward: a thread has one or two units of 16 bytes, four of the longest rows: 8 or 32 threads a row up to 512 columns of 16 bits (no barrier), 64 to 1024 threads
// and a barrier for each sum up to 32768, a row's loads all in flight; longer rows are read three times.  The sums
// of a row are taken twice from the registers, of x for the mean m and then of x - m and its square: the first of these two
// is what m's rounding has left, which corrects the mean and the variance, so a mean far above the spread costs no accuracy (see about and variance for
// a spread of nothing or of a few steps).
//
// Backward, up to 8192 columns (longer rows: two kernels that read them once each): two units a thread.  With mean and rstd at hand a row needs one reduction, of g and g xhat; the sums
// over rows of dy xhat and dy stay with the thread that owns the column, and each block leaves one row of partial sums, which a
// second kernel adds in a fixed order.
#include <math.h>

#include "op_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

// Sum over the TPR threads of a row, known to all of them.  `part`: TPR / 32 words of shared memory for each value, which must not be written again
// before every thread has passed another barrier.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* part) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if constexpr (TPR > 32) {
    constexpr int WARPS = TPR / 32;
    const int warp = threadIdx.x % TPR / 32, lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) part[k * WARPS + warp] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = part[k * WARPS + lane % WARPS];
#pragma unroll
      for (int o = WARPS / 2; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
  }
}

// Where a row's sums are taken about: its mean, or its first element where that is as near to the mean as the mean's rounding `near` (relative) lets one
// tell.  Elements that are all equal then leave nothing at all, whatever their sum has been rounded to, or overflowed to.
constexpr float kNear = 0x1p-18f;              // 32 terms a thread, ten steps of a tree, the quotient: 44 times 2^-24 at most
// With variance() it costs FP32 rows up to 5 % (19794 x 599 24.5 us instead of 23.4, 16384 x 2048 46.2 and 45.8).
// (16-bit elements up to 8192 columns need neither: the sum of equal ones is exact, its quotient is made so, and any spread is 2^-11 of a value or more.)
__device__ __forceinline__ float about(float mean, float first, float near) { return fabsf(first - mean) <= near * fabsf(mean) ? first : mean; }
// sum t^2 / n - (sum t / n)^2 of n elements t, from their sums s, s2 and off = s / n rounded.  s^2 / n = s off + off (s - off n) but for terms of second order, and
// neither product is rounded before it is taken from s2, so where the two are almost equal little is lost (few steps of FP32 between the elements
// make their sums exact).  Never below zero; NaN stays.
__device__ __forceinline__ float variance(float s, float s2, float off, float n, float inv_n) {
  return __fmul_rn(max_nan(fmaf(-off, fmaf(-off, n, s), fmaf(-s, off, s2)), 0.f), inv_n);
}

// TPR threads a row, which hold NU units of 16 bytes each.  A block walks its rows with the next row's loads under way while it works on
// one; the weights stay in registers where they are few.
template <int TPR> constexpr int norm_block = TPR > 128 ? TPR : 128;
// Blocks of an SM.  16384 x 4096 bf16 with two units a thread: 51.3 us at 768 threads an SM (80 registers), 52.6 at 1024, 74 at 1280; a unit of FP32 has half the
// elements and needs fewer registers (16384 x 2048: 48.4 and 43.9 us), as do rows of eight threads, one unit each (10^6 x 64 bf16: 63 and 54).
template <class T, int TPR> constexpr int norm_blocks = (TPR > 256 || sizeof(T) == 4 || TPR == 8 ? 1024 : 768) / norm_block<TPR>;
template <class T, class W, int TPR, int NU, bool VEC>
__global__ void __launch_bounds__(norm_block<TPR>, norm_blocks<T, TPR>)
layer_norm_kernel(int64_t rows, int cols, const T* x, int64_t ldx, const W* w, const W* b, float eps, T* y, int64_t ldy, float* mean_out, float* rstd_out) {
  constexpr int V = Pack<T>::V, VW = Pack<W>::V, WU = sizeof(W) / sizeof(T);      // WU: units of the weights to a unit of x
  constexpr int PER = norm_block<TPR> / TPR;                     // rows of a block
  constexpr bool KEEP = NU * WU <= 2;
  constexpr bool NEAR = sizeof(T) == 4 || TPR * NU * V > 8192;     // see about
  __shared__ float part[TPR > 32 ? PER : 1][3 * (TPR > 32 ? TPR / 32 : 1) + 1];    // (the last word: the row's first element)
  const int thread = threadIdx.x % TPR;
  float* const mine = part[TPR > 32 ? threadIdx.x / TPR : 0];
  grid_dep_wait();
  grid_dep_launch();
  x = dep(x); w = dep(w); b = dep(b);
  const float n = (float)cols, inv_n = 1.f / n;
  const int64_t step = (int64_t)gridDim.x * PER;
  int64_t r = (int64_t)blockIdx.x * PER + threadIdx.x / TPR;
  // (the weights of unit u are units u WU .. u WU + WU - 1 of theirs, and lie side by side where x's elements do)
  const auto weights = [&](const W* p, int u, int q) {
    return VEC && WU > 1 ? load_pack<true>(p, 0, (u * TPR + thread) * WU + q, 1, cols) : load_pack<VEC>(p, u * WU + q, thread, TPR, cols);
  };
  Pack<W> wk[KEEP ? NU * WU : 1], bk[KEEP ? NU * WU : 1];
  if constexpr (KEEP)
#pragma unroll
    for (int q = 0; q < NU * WU; ++q) {
      if (w) wk[q] = weights(w, q / WU, q % WU);
      if (b) bk[q] = weights(b, q / WU, q % WU);
    }
  Pack<T> next[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) next[u] = load_pack<VEC>(x + (r < rows ? r : 0) * ldx, u, thread, TPR, cols);
  // (all threads of a block make the same rounds: those without a row still take part in the sums' exchanges and barriers)
  for (int64_t r0 = (int64_t)blockIdx.x * PER; r0 < rows; r0 += step, r += step) {
    const bool in = r < rows;
    Pack<T> v[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) v[u] = next[u];
    if (r0 + step < rows)
#pragma unroll
      for (int u = 0; u < NU; ++u) next[u] = load_pack<VEC>(x + (r + step < rows ? r + step : 0) * ldx, u, thread, TPR, cols);
    // (few instructions an element: at 16 bits the arithmetic alone is half of what memory takes)
    float t[NU * V], s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NU * V; ++k) { t[k] = v[k / V].get(k % V); s[0] += t[k]; }
    float first = t[0];
    if (NEAR && TPR > 32 && thread == 0) mine[3 * TPR / 32] = first;
    row_sum<TPR>(s, mine);
    float m = s[0] * inv_n;
    if constexpr (NEAR) {
      first = TPR > 32 ? mine[3 * TPR / 32] : __shfl_sync(0xffffffffu, first, 0, TPR > 32 ? 32 : TPR);
      m = about(m, first, kNear);
    } else {
      m = fmaf(fmaf(-m, n, s[0]), inv_n, m);
    }
    float d[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if (pack_col<VEC, T>(u, V - 1, thread, TPR) < cols) {
#pragma unroll
        for (int e = 0; e < V; ++e) { t[u * V + e] -= m; d[0] += t[u * V + e]; d[1] = fmaf(t[u * V + e], t[u * V + e], d[1]); }
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (pack_col<VEC, T>(u, e, thread, TPR) < cols) { t[u * V + e] -= m; d[0] += t[u * V + e]; d[1] = fmaf(t[u * V + e], t[u * V + e], d[1]); }
      }
    }
    row_sum<TPR>(d, mine + (TPR > 32 ? TPR / 32 : 0));
    const float off = d[0] * inv_n, var = NEAR ? variance(d[0], d[1], off, n, inv_n) : d[1] * inv_n - off * off;
    const float rstd = 1.f / sqrtf(var + eps), shift = -off * rstd;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if (pack_col<VEC, T>(u, 0, thread, TPR) >= cols) break;
      float o[V];
#pragma unroll
      for (int q = 0; q < WU; ++q) {
        Pack<W> pw, pb;
        if constexpr (KEEP) { pw = wk[u * WU + q]; pb = bk[u * WU + q]; }
        else {
          if (w) pw = weights(w, u, q);
          if (b) pb = weights(b, u, q);
        }
#pragma unroll
        for (int e = 0; e < VW; ++e) o[q * VW + e] = fmaf(fmaf(t[u * V + q * VW + e], rstd, shift), w ? pw.get(e) : 1.f, b ? pb.get(e) : 0.f);
      }
      Pack<T> p;
      p.set(o);
      if (in) store_pack<VEC>(y + r * ldy, p, u, thread, TPR, cols);
    }
    if (in && thread == 0) {
      if (mean_out) mean_out[r] = m + off;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

// Rows too long for the registers of a block: the row is read three times, twice of them out of L2.
template <class T, class W>
__global__ void __launch_bounds__(1024) layer_norm_long_kernel(int64_t rows, int cols, const T* x, int64_t ldx, const W* w, const W* b, float eps, T* y,
                                                               int64_t ldy, float* mean_out, float* rstd_out) {
  __shared__ float part[3 * 32];
  const float near = kNear + 0x1p-24f * (cols / 1024);     // (as many terms a thread)
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* xr = x + r * ldx;
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < cols; c += blockDim.x) s[0] += to_f(xr[c]);
    row_sum<1024>(s, part);
    const float m = about(s[0] / cols, to_f(xr[0]), near);
    float d[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < cols; c += blockDim.x) { const float v = to_f(xr[c]) - m; d[0] += v; d[1] += v * v; }
    row_sum<1024>(d, part + 32);
    const float off = d[0] / cols, rstd = 1.f / sqrtf(variance(d[0], d[1], off, (float)cols, 1.f / cols) + eps);
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

// ---- backward ----------------------------------------------------------------------------------
template <class T> constexpr int kOwn = 2 * Pack<T>::V;   // columns of a thread

struct NormGradArgs {
  int64_t rows; int cols;
  const void *dy, *x, *w, *add; void* dx;
  int64_t ld_dy, ldx, ld_add, ld_dx;
  const float *mean, *rstd;
  float* part;                       // [blocks][2][cols]
  float* stats;                      // long rows: [rows][2], the means of g and of g xhat
  int sums;                          // whether the sums over rows are wanted
};

// The kOwn elements of a row that belong to a thread.
template <bool VEC, class T>
__device__ __forceinline__ int own_col(int k, int thread, int threads) { return pack_col<VEC, T>(k / Pack<T>::V, k % Pack<T>::V, thread, threads); }
template <bool VEC, class T>
struct Own {
  Pack<T> p[2];
  __device__ __forceinline__ void load(const T* row, int thread, int threads, int cols) {
#pragma unroll
    for (int u = 0; u < 2; ++u) p[u] = load_pack<VEC>(row, u, thread, threads, cols);
  }
  __device__ __forceinline__ float get(int k) const { return p[k / Pack<T>::V].get(k % Pack<T>::V); }
  __device__ __forceinline__ void set_store(const float (&o)[kOwn<T>], T* row, int thread, int threads, int cols) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float q[Pack<T>::V];
#pragma unroll
      for (int e = 0; e < Pack<T>::V; ++e) q[e] = o[u * Pack<T>::V + e];
      p[u].set(q);
      store_pack<VEC>(row, p[u], u, thread, threads, cols);
    }
  }
};

// The columns that a thread owns, summed over the block's groups of threads, to the block's row of partial sums.
template <bool VEC, class T, int TPR, int BLOCK>
__device__ __forceinline__ void leave_sums(const NormGradArgs& a, float (&sw)[kOwn<T>], float (&sb)[kOwn<T>], float* buf, int64_t block, int first, int cols) {
  constexpr int G = BLOCK / TPR;
  const int thread = threadIdx.x % TPR, group = threadIdx.x / TPR;
  if constexpr (G > 1) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kOwn<T>; ++k) buf[k * BLOCK + threadIdx.x] = half ? sb[k] : sw[k];
      __syncthreads();
      if (group == 0)
#pragma unroll
        for (int k = 0; k < kOwn<T>; ++k) {
          float t = 0.f;
          for (int q = 0; q < G; ++q) t += buf[k * BLOCK + q * TPR + thread];
          if (half) sb[k] = t; else sw[k] = t;
        }
    }
  }
  if (group == 0)
#pragma unroll
    for (int k = 0; k < kOwn<T>; ++k) {
      const int c = own_col<VEC, T>(k, thread, TPR);
      if (c < cols) {
        a.part[(block * 2) * a.cols + first + c] = sw[k];
        a.part[(block * 2 + 1) * a.cols + first + c] = sb[k];
      }
    }
}

template <int TPR> constexpr int grad_block = TPR > 256 ? TPR : 256;
// Threads of an SM: what a thread holds of two rows, the weights and the sums takes about 110 registers at 16 bits (16 columns).
template <class T> constexpr int ring_threads = 512;
template <class T, int TPR> constexpr int ring_blocks = ring_threads<T> / grad_block<TPR> > 0 ? ring_threads<T> / grad_block<TPR> : 1;
// 16-bit rows that 16-byte accesses cannot be made to (cp.async has none of two bytes): the next row's elements in registers.
template <class T, class W, int TPR>
__global__ void __launch_bounds__(grad_block<TPR>, ring_blocks<T, TPR>) layer_norm_grad_kernel(const NormGradArgs a) {
  constexpr int BLOCK = grad_block<TPR>, G = BLOCK / TPR;
  constexpr bool VEC = false;
  __shared__ float part[2][G][TPR > 32 ? 2 * (TPR / 32) : 1];
  __shared__ float buf[G > 1 ? kOwn<T> * BLOCK : 1];
  const int thread = threadIdx.x % TPR, group = threadIdx.x / TPR;
  grid_dep_wait();
  grid_dep_launch();
  const T* const dy = (const T*)dep(a.dy);
  const T* const x = (const T*)dep(a.x);
  const T* const add = (const T*)dep(a.add);
  const W* const w = (const W*)dep(a.w);
  const float* const mean = dep(a.mean);
  const float* const rstd = dep(a.rstd);
  const int cols = a.cols;
  const float inv_n = 1.f / (float)cols;
  float wv[kOwn<T>], sw[kOwn<T>], sb[kOwn<T>];
#pragma unroll
  for (int k = 0; k < kOwn<T>; ++k) {
    const int c = own_col<VEC, T>(k, thread, TPR);
    wv[k] = w && c < cols ? to_f(w[c]) : 1.f;
    sw[k] = sb[k] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * G;
  int64_t r = (int64_t)blockIdx.x * G + group;
  int flip = 0;
  Own<VEC, T> xn, gn_;
  float mn = 0.f, rn = 0.f;
  const auto fetch = [&](int64_t q) {          // (a group without a row reads zeros: rstd 0)
    const bool in = q < a.rows;
    mn = in ? mean[q] : 0.f; rn = in ? rstd[q] : 0.f;
    xn.load(x + (in ? q : 0) * a.ldx, thread, TPR, in ? cols : 0);
    gn_.load(dy + (in ? q : 0) * a.ld_dy, thread, TPR, in ? cols : 0);
  };
  fetch(r);
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += step, r += step, flip ^= 1) {
    Own<VEC, T> xo = xn, go = gn_, ao;
    const float m = mn, rs = rn;
    const bool out = a.dx && r < a.rows;
    if (out && add) ao.load(add + r * a.ld_add, thread, TPR, cols);
    if (r0 + step < a.rows) fetch(r + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kOwn<T>; ++k) {
      const float g = go.get(k), xh = (xo.get(k) - m) * rs;
      // (columns past the row's end: dy reads as zero there)
      s[0] = fmaf(g, wv[k], s[0]);
      s[1] = fmaf(g * wv[k], xh, s[1]);
      sw[k] = fmaf(g, xh, sw[k]);
      sb[k] += g;
    }
    row_sum<TPR>(s, part[flip][group]);        // (two sets of words in turn: one barrier a round is enough)
    if (out) {
      const float p = -rs * (s[0] * inv_n), q = -rs * (s[1] * inv_n);
      float o[kOwn<T>];
#pragma unroll
      for (int k = 0; k < kOwn<T>; ++k) {
        o[k] = fmaf((xo.get(k) - m) * rs, q, fmaf(go.get(k) * wv[k], rs, p));
        if (add) o[k] += ao.get(k);
      }
      go.set_store(o, (T*)a.dx + r * a.ld_dx, thread, TPR, cols);
    }
  }
  if (a.sums) leave_sums<VEC, T, TPR, BLOCK>(a, sw, sb, buf, blockIdx.x, 0, cols);
}

// The same where 16-byte accesses can be made, and in FP32 where they cannot (4 bytes each): a thread's elements of the next rows are on their way to its own places in shared memory (cp.async, which
// nobody else reads: no barrier), so that the loads in flight are not limited by registers.  16384 x 4096 bf16 with `add`: 95 us (117 with one row
// ahead in registers), 5.7 TB/s of the 6.4 of a copy.  Rows ahead: 2 at 16 bits (3: 96 us), 3 at 32 (16384 x 2048: 84 us, 2: 89).
template <class T, int TPR> constexpr int kAhead = TPR > 512 ? 1 : sizeof(T) == 2 ? 2 : 3;       // (a block of 1024 threads has 96 KB a row)
template <class T, int TPR> constexpr int ring_bytes = (kAhead<T, TPR> + 1) * 3 * 2 * grad_block<TPR> * 16;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {       // (the rest of the 16 reads as zero)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <class T, class W, int TPR, bool VEC>
__global__ void __launch_bounds__(grad_block<TPR>, ring_blocks<T, TPR>) layer_norm_grad_ring_kernel(const NormGradArgs a) {
  constexpr int BLOCK = grad_block<TPR>, G = BLOCK / TPR, AHEAD = kAhead<T, TPR>, STAGES = AHEAD + 1;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float part[2][G][TPR > 32 ? 2 * (TPR / 32) : 1];
  const int thread = threadIdx.x % TPR, group = threadIdx.x / TPR;
  grid_dep_wait();
  grid_dep_launch();
  const T* const dy = (const T*)dep(a.dy);
  const T* const x = (const T*)dep(a.x);
  const T* const add = (const T*)dep(a.add);
  const W* const w = (const W*)dep(a.w);
  const float* const mean = dep(a.mean);
  const float* const rstd = dep(a.rstd);
  const int cols = a.cols;
  const float inv_n = 1.f / (float)cols;
  const bool adds = add != nullptr && a.dx != nullptr;
  float wv[kOwn<T>], sw[kOwn<T>], sb[kOwn<T>];
#pragma unroll
  for (int k = 0; k < kOwn<T>; ++k) {
    const int c = own_col<VEC, T>(k, thread, TPR);
    wv[k] = w && c < cols ? to_f(w[c]) : 1.f;
    sw[k] = sb[k] = 0.f;
  }
  int bytes[2], col[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int c = pack_col<VEC, T>(u, 0, thread, TPR), n = (cols - c) * (int)sizeof(T);
    bytes[u] = n < 0 ? 0 : n > 16 ? 16 : n;
    col[u] = bytes[u] ? c : 0;
  }
  // (a unit of 16 bytes to a place, or, where an access is to one element, element e of a unit BLOCK words behind element e - 1)
  const uint32_t own = smem_u32(ring) + threadIdx.x * (VEC ? 16 : 4);
  const auto place = [&](int stage, int matrix, int u) { return own + (uint32_t)(((stage * 3 + matrix) * 2 + u) * BLOCK * 16); };
  const auto copy = [&](int stage, int matrix, const T* row) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (VEC) {
        cp_async16(place(stage, matrix, u), row + col[u], bytes[u]);
      } else {
#pragma unroll
        for (int e = 0; e < Pack<T>::V; ++e) {
          const int c = pack_col<false, T>(u, e, thread, TPR);
          cp_async4(place(stage, matrix, u) + (uint32_t)(e * BLOCK * 4), row + (c < cols ? c : 0), c < cols ? 4 : 0);
        }
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * G;
  int64_t r = (int64_t)blockIdx.x * G + group;
  const auto request = [&](int64_t q, int stage) {
    if (q < a.rows) {
      copy(stage, 0, x + q * a.ldx);
      copy(stage, 1, dy + q * a.ld_dy);
      if (adds) copy(stage, 2, add + q * a.ld_add);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const auto take = [&](int stage, int matrix, Own<VEC, T>& o) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint4& w4 = o.p[u].w;
      if constexpr (VEC) {
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w4.x), "=r"(w4.y), "=r"(w4.z), "=r"(w4.w) : "r"(place(stage, matrix, u)) : "memory");
      } else {
        const uint32_t at = place(stage, matrix, u);
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w4.x) : "r"(at) : "memory");
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w4.y) : "r"(at + BLOCK * 4u) : "memory");
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w4.z) : "r"(at + BLOCK * 8u) : "memory");
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w4.w) : "r"(at + BLOCK * 12u) : "memory");
      }
    }
  };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) request(r + k * step, k);
  float mn = r < a.rows ? mean[r] : 0.f, rn = r < a.rows ? rstd[r] : 0.f;
  int flip = 0, stage = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * G; r0 < a.rows; r0 += step, r += step, flip ^= 1) {
    const bool in = r < a.rows;
    const float m = mn, rs = rn;
    request(r + AHEAD * step, stage == 0 ? STAGES - 1 : stage - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD) : "memory");
    Own<VEC, T> xo, go, ao;
    if (in) {
      take(stage, 0, xo); take(stage, 1, go);
      if (adds) take(stage, 2, ao);
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) xo.p[u].w = go.p[u].w = make_uint4(0u, 0u, 0u, 0u);
    }
    if (r + step < a.rows) { mn = mean[r + step]; rn = rstd[r + step]; }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kOwn<T>; ++k) {
      const float g = go.get(k), xh = (xo.get(k) - m) * rs;
      s[0] = fmaf(g, wv[k], s[0]);
      s[1] = fmaf(g * wv[k], xh, s[1]);
      sw[k] = fmaf(g, xh, sw[k]);
      sb[k] += g;
    }
    row_sum<TPR>(s, part[flip][group]);
    if (in && a.dx) {
      const float p = -rs * (s[0] * inv_n), q = -rs * (s[1] * inv_n);
      float o[kOwn<T>];
#pragma unroll
      for (int k = 0; k < kOwn<T>; ++k) {
        o[k] = fmaf((xo.get(k) - m) * rs, q, fmaf(go.get(k) * wv[k], rs, p));
        if (adds) o[k] += ao.get(k);
      }
      go.set_store(o, (T*)a.dx + r * a.ld_dx, thread, TPR, cols);
    }
    if (++stage == STAGES) stage = 0;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  if (a.sums) leave_sums<VEC, T, TPR, BLOCK>(a, sw, sb, (float*)ring, blockIdx.x, 0, cols);
}

// Rows of more than 8192 columns: the two means of a row by a kernel of their own, then blocks of columns that walk a share of the rows.
template <class T, class W>
__global__ void __launch_bounds__(1024) layer_norm_stats_kernel(const NormGradArgs a) {
  const T* const dy = (const T*)a.dy;
  const T* const x = (const T*)a.x;
  const W* const w = (const W*)a.w;
  __shared__ float part[2][64];
  int flip = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, flip ^= 1) {
    const float m = a.mean[r], rs = a.rstd[r];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float g = to_f(dy[r * a.ld_dy + c]) * (w ? to_f(w[c]) : 1.f);
      s[0] += g; s[1] += g * ((to_f(x[r * a.ldx + c]) - m) * rs);
    }
    row_sum<1024>(s, part[flip]);
    if (threadIdx.x == 0) { a.stats[2 * r] = s[0] / a.cols; a.stats[2 * r + 1] = s[1] / a.cols; }
  }
}
template <class T> constexpr int kLongCols = 256 * kOwn<T>;
template <class T, class W, bool VEC>
__global__ void __launch_bounds__(256) layer_norm_grad_long_kernel(const NormGradArgs a) {
  const int first = blockIdx.x * kLongCols<T>, cols = min(kLongCols<T>, a.cols - first), thread = threadIdx.x;
  const T* const dy = (const T*)a.dy + first;
  const T* const x = (const T*)a.x + first;
  const T* const add = a.add ? (const T*)a.add + first : nullptr;
  const W* const w = a.w ? (const W*)a.w + first : nullptr;
  float wv[kOwn<T>], sw[kOwn<T>], sb[kOwn<T>];
#pragma unroll
  for (int k = 0; k < kOwn<T>; ++k) {
    const int c = own_col<VEC, T>(k, thread, 256);
    wv[k] = w && c < cols ? to_f(w[c]) : 1.f;
    sw[k] = sb[k] = 0.f;
  }
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const float m = a.mean[r], rs = a.rstd[r], p = a.dx ? a.stats[2 * r] : 0.f, q = a.dx ? a.stats[2 * r + 1] : 0.f;
    Own<VEC, T> xo, go, ao;
    xo.load(x + r * a.ldx, thread, 256, cols);
    go.load(dy + r * a.ld_dy, thread, 256, cols);
    if (add) ao.load(add + r * a.ld_add, thread, 256, cols);
    float o[kOwn<T>];
#pragma unroll
    for (int k = 0; k < kOwn<T>; ++k) {
      const float g = go.get(k), xh = (xo.get(k) - m) * rs;
      sw[k] = fmaf(g, xh, sw[k]); sb[k] += g;
      o[k] = rs * (g * wv[k] - p - xh * q) + (add ? ao.get(k) : 0.f);
    }
    if (a.dx) go.set_store(o, (T*)a.dx + first + r * a.ld_dx, thread, 256, cols);
  }
  if (a.sums) leave_sums<VEC, T, 256, 256>(a, sw, sb, nullptr, blockIdx.y, first, cols);
}

// dw, db = sums of the blocks' partial sums, in order of the blocks: 32 columns of either a block, a warp for every 32nd partial row.
template <class W>
__global__ void __launch_bounds__(1024) layer_norm_sums_kernel(int blocks, int cols, const float* part, W* dw, W* db) {
  __shared__ float buf[32][33];
  grid_dep_wait();
  grid_dep_launch();
  part = dep(part);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols)
    for (int k = warp; k < blocks; k += 32) s += part[((int64_t)k * 2 + blockIdx.y) * cols + c];
  buf[warp][lane] = s;
  __syncthreads();
  s = buf[lane][warp];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  W* const out = blockIdx.y ? db : dw;
  if (lane == 0 && out && blockIdx.x * 32 + warp < cols) out[blockIdx.x * 32 + warp] = from_f<W>(s);
}

// How a backward pass is cut: threads a row (0: long rows), and the blocks that leave partial sums.
struct NormGradPlan { int tpr; int64_t blocks; };
template <class T>
NormGradPlan norm_grad_plan(int64_t rows, int cols) {
  NormGradPlan p{0, 0};
  for (int t = 8; t <= 8192 / kOwn<T>; t *= 2)
    if (cols <= t * kOwn<T>) { p.tpr = t; break; }
  if (p.tpr) {
    const int block = p.tpr > 256 ? p.tpr : 256, per = block / p.tpr, threads = ring_threads<T>;
    const int resident = threads / block > 0 ? threads / block : 1;
    const int64_t want = (rows + per - 1) / per, most = 148LL * resident;
    p.blocks = want < most ? want : most;
  } else {
    const int64_t strips = (cols + kLongCols<T> - 1) / kLongCols<T>, most = (148 * 4 + strips - 1) / strips;
    p.blocks = rows < most ? rows : most;
  }
  return p;
}
template <class T>
int64_t norm_grad_floats(int64_t rows, int cols) {
  const NormGradPlan p = norm_grad_plan<T>(rows, cols);
  return p.blocks * 2 * cols + (p.tpr ? 0 : 2 * rows);
}

struct NormCall {
  int type;
  int64_t rows; int cols;
  const void *dy, *x, *w, *b, *add; int64_t ld_dy, ldx, ld_add;
  void *y, *dw, *db; int64_t ldy;
  float *mean, *rstd; float eps;
  void* ws; cudaStream_t st;
};

template <class T, class W, int TPR, int NU>
cudaError_t norm_as(const NormCall& a, bool vec) {
  constexpr int BLOCK = norm_block<TPR>, PER = BLOCK / TPR;
  const int64_t want = (a.rows + PER - 1) / PER, most = 148LL * norm_blocks<T, TPR>, blocks = want < most ? want : most;
  auto* const k = vec ? layer_norm_kernel<T, W, TPR, NU, true> : layer_norm_kernel<T, W, TPR, NU, false>;
  return launch_pdl_grid(k, dim3((unsigned)blocks), BLOCK, 0, a.st, a.rows, a.cols, (const T*)a.x, a.ldx, (const W*)a.w, (const W*)a.b, a.eps,
                         (T*)a.y, a.ldy, a.mean, a.rstd);
}
template <class T, class W>
cudaError_t run_norm(const NormCall& a) {
  const bool vec = wide_ok(a.x, a.ldx, a.type) && wide_ok(a.y, a.ldy, a.type) && wide_ok(a.w, 0, GN_F32) && wide_ok(a.b, 0, GN_F32);
  const int units = (a.cols + Pack<T>::V - 1) / Pack<T>::V;
  if (units <= 8) return norm_as<T, W, 8, 1>(a, vec);
  if (units <= 32) return norm_as<T, W, 32, 1>(a, vec);
  if (units <= 64) return norm_as<T, W, 32, 2>(a, vec);
  if (units <= 128) return norm_as<T, W, 64, 2>(a, vec);
  if (units <= 256) return norm_as<T, W, 128, 2>(a, vec);
  if (units <= 512) return norm_as<T, W, 256, 2>(a, vec);
  if (units <= 1024) return norm_as<T, W, 512, 2>(a, vec);
  if (units <= 2048) return norm_as<T, W, 1024, 2>(a, vec);
  if (units <= 4096) return norm_as<T, W, 1024, 4>(a, vec);
  const int64_t most = 148 * 2;
  layer_norm_long_kernel<T, W><<<(unsigned)(a.rows < most ? a.rows : most), 1024, 0, a.st>>>(
      a.rows, a.cols, (const T*)a.x, a.ldx, (const W*)a.w, (const W*)a.b, a.eps, (T*)a.y, a.ldy, a.mean, a.rstd);
  return cudaGetLastError();
}

template <class T, class W, int TPR>
cudaError_t norm_grad_as(const NormGradArgs& g, bool vec, int64_t blocks, cudaStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (!vec) return launch_pdl_grid(layer_norm_grad_kernel<T, W, TPR>, dim3((unsigned)blocks), grad_block<TPR>, 0, st, g);
  auto* const k = vec ? layer_norm_grad_ring_kernel<T, W, TPR, true> : layer_norm_grad_ring_kernel<T, W, TPR, sizeof(T) == 2>;
  static std::atomic<signed char> ready[2][64];
  if (!once_per_device(ready[vec], [&] { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes<T, TPR>) == cudaSuccess; })) return cudaErrorInvalidDevice;
  return launch_pdl_grid(k, dim3((unsigned)blocks), grad_block<TPR>, ring_bytes<T, TPR>, st, g);
}
template <class T, class W>
cudaError_t run_norm_grad(const NormCall& a) {
  NormGradArgs g{a.rows, a.cols, a.dy, a.x, a.w, a.add, a.y, a.ld_dy, a.ldx, a.ld_add, a.ldy, a.mean, a.rstd, (float*)a.ws, nullptr, a.dw || a.db};
  const bool vec = wide_ok(a.dy, a.ld_dy, a.type) && wide_ok(a.x, a.ldx, a.type) && wide_ok(a.add, a.ld_add, a.type) && wide_ok(a.y, a.ldy, a.type);
  const NormGradPlan plan = norm_grad_plan<T>(a.rows, a.cols);
  cudaError_t e = cudaSuccess;
  if (a.rows > 0 && (g.sums || g.dx)) {
    switch (plan.tpr) {
      case 8: e = norm_grad_as<T, W, 8>(g, vec, plan.blocks, a.st); break;
      case 16: e = norm_grad_as<T, W, 16>(g, vec, plan.blocks, a.st); break;
      case 32: e = norm_grad_as<T, W, 32>(g, vec, plan.blocks, a.st); break;
      case 64: e = norm_grad_as<T, W, 64>(g, vec, plan.blocks, a.st); break;
      case 128: e = norm_grad_as<T, W, 128>(g, vec, plan.blocks, a.st); break;
      case 256: e = norm_grad_as<T, W, 256>(g, vec, plan.blocks, a.st); break;
      case 512: e = norm_grad_as<T, W, 512>(g, vec, plan.blocks, a.st); break;
      case 1024:
        if constexpr (sizeof(T) == 4) e = norm_grad_as<T, W, 1024>(g, vec, plan.blocks, a.st);
        break;
      default: {
        g.stats = g.part + plan.blocks * 2 * a.cols;
        if (g.dx) layer_norm_stats_kernel<T, W><<<(unsigned)(a.rows < 296 ? a.rows : 296), 1024, 0, a.st>>>(g);
        const dim3 grid((unsigned)((a.cols + kLongCols<T> - 1) / kLongCols<T>), (unsigned)plan.blocks);
        if (vec) layer_norm_grad_long_kernel<T, W, true><<<grid, 256, 0, a.st>>>(g);
        else layer_norm_grad_long_kernel<T, W, false><<<grid, 256, 0, a.st>>>(g);
        e = cudaGetLastError();
      }
    }
  }
  if (e != cudaSuccess || !g.sums) return e;
  return launch_pdl_grid(layer_norm_sums_kernel<W>, dim3((unsigned)((a.cols + 31) / 32), 2), 1024, 0, a.st, (int)plan.blocks, a.cols, (const float*)g.part,
                         (W*)a.dw, (W*)a.db);
}

template <template <class, class> class F>
cudaError_t by_types(int type, int wtype, const NormCall& a) {
  if (type == GN_F32) return F<float, float>::run(a);
  if (type == GN_BF16) return wtype == GN_F32 ? F<__nv_bfloat16, float>::run(a) : F<__nv_bfloat16, __nv_bfloat16>::run(a);
  return wtype == GN_F32 ? F<__half, float>::run(a) : F<__half, __half>::run(a);
}
template <class T, class W> struct Norm { static cudaError_t run(const NormCall& a) { return run_norm<T, W>(a); } };
template <class T, class W> struct NormGrad { static cudaError_t run(const NormCall& a) { return run_norm_grad<T, W>(a); } };

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
  a.type = type; a.rows = rows; a.cols = cols; a.x = d_x; a.ldx = ldx; a.w = d_weight; a.b = d_bias; a.eps = (float)eps;
  a.y = d_y; a.ldy = ldy; a.mean = d_mean; a.rstd = d_rstd; a.st = (cudaStream_t)cuda_stream;
  return op_done(by_types<Norm>(type, wtype, a), errbuf, errbuf_len);
}

extern "C" int64_t gn_layer_norm_grad_workspace(int64_t rows, int32_t cols) {
  if (rows < 0 || cols < 1 || cols > kMaxCols) return -1;
  const int64_t a = norm_grad_floats<float>(rows, cols), b = norm_grad_floats<__half>(rows, cols);
  return (a > b ? a : b) * 4 + 16;
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
  a.type = type; a.rows = rows; a.cols = cols; a.dy = d_dy; a.ld_dy = ld_dy; a.x = d_x; a.ldx = ldx; a.w = d_weight; a.add = d_add; a.ld_add = ld_add;
  a.y = d_dx; a.ldy = ld_dx; a.dw = d_dweight; a.db = d_dbias; a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
  a.ws = d_ws; a.st = (cudaStream_t)cuda_stream;
  return op_done(by_types<NormGrad>(type, wtype, a), errbuf, errbuf_len);
}
