// Gated feed-forward block and its backward pass: the calls, their workspaces and the order of their products.
#include <math.h>

#include "op_common.cuh"

namespace gn {
namespace {

// 1 / (1 + exp(-v)) and 1 / (1 + exp(v)), each to full relative accuracy: one minus the other would lose it where it is small.
__device__ __forceinline__ void sigmoids(float v, float& z, float& nz) {
  const float e = expf(-fabsf(v)), r = 1.f / (1.f + e);
  z = v < 0.f ? e * r : r; nz = v < 0.f ? r : e * r;
}
// act(v) and its derivative.  A NaN stays one: comparisons with it fall to the branch that computes with it.
__device__ __forceinline__ void activation(int act, float v, float& a, float& da) {
  float z, nz;
  switch (act) {
    case GN_ACT_RELU: a = v < 0.f ? 0.f : v; da = v > 0.f ? 1.f : 0.f; break;
    case GN_ACT_GELU: {
      const float cdf = 0.5f * erfcf(-0.70710678118654752f * v);
      a = v * cdf; da = cdf + v * 0.39894228040143268f * expf(-0.5f * v * v);
      break;
    }
    case GN_ACT_GELU_TANH: {                   // (1 + tanh q) / 2 = 1 / (1 + exp(-2 q))
      const float k = 1.5957691216057308f;     // 2 sqrt(2 / pi)
      sigmoids(k * (v + 0.044715f * v * v * v), z, nz);
      a = v * z; da = z + v * z * nz * k * (1.f + 0.134145f * v * v);
      break;
    }
    case GN_ACT_SIGMOID: sigmoids(v, z, nz); a = z; da = z * nz; break;
    default: sigmoids(v, z, nz); a = v * z; da = z + v * z * nz;
  }
}

// D(m, n) = sum over the operand pairs of sum_k A(m, k) B(k, n), element (i, j) of an operand at i s0 + j s1.
struct Operand { const void* p; int64_t s0, s1; };
struct PlainGemm { int64_t M, N, K; int pairs; Operand a[2], b[2]; void* d; int64_t ldd; };
template <class T, class D>
__global__ void plain_gemm_kernel(const PlainGemm g) {
  __shared__ float sa[16][65], sb[16][65];
  const int64_t m0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int q = 0; q < g.pairs; ++q)
    for (int64_t k0 = 0; k0 < g.K; k0 += 16) {
      for (int e = threadIdx.x; e < 1024; e += 256) {
        const int i = e >> 4, k = e & 15;
        sa[k][i] = m0 + i < g.M && k0 + k < g.K ? to_f(((const T*)g.a[q].p)[(m0 + i) * g.a[q].s0 + (k0 + k) * g.a[q].s1]) : 0.f;
        sb[k][i] = n0 + i < g.N && k0 + k < g.K ? to_f(((const T*)g.b[q].p)[(k0 + k) * g.b[q].s0 + (n0 + i) * g.b[q].s1]) : 0.f;
      }
      __syncthreads();
      for (int k = 0; k < 16; ++k)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
      __syncthreads();
    }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m < g.M && n < g.N) ((D*)g.d)[m * g.ldd + n] = from_f<D>(acc[i][j]);
    }
}

// h = act(gate) * up, and with dh the two gradients.
struct Gates { int64_t rows; int cols, act; const void *gate, *up; int64_t ld_gate, ld_up; const float* dh; void *h, *dgate, *dup; };
template <class T>
__global__ void gate_kernel(const Gates g) {
  const int64_t n = g.rows * g.cols;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t r = i / g.cols, c = i % g.cols;
    float a, da;
    const float u = to_f(((const T*)g.up)[r * g.ld_up + c]);
    activation(g.act, to_f(((const T*)g.gate)[r * g.ld_gate + c]), a, da);
    if (g.h) ((T*)g.h)[i] = from_f<T>(a * u);
    if (g.dh) {
      ((T*)g.dup)[i] = from_f<T>(g.dh[i] * a);
      ((T*)g.dgate)[i] = from_f<T>(g.dh[i] * u * da);
    }
  }
}
template <class T, class D = T>
cudaError_t plain_gemm(const PlainGemm& g, cudaStream_t st) {
  if (g.M == 0 || g.N == 0) return cudaSuccess;
  plain_gemm_kernel<T, D><<<dim3((unsigned)((g.M + 63) / 64), (unsigned)((g.N + 63) / 64)), 256, 0, st>>>(g);
  return cudaGetLastError();
}

const char* ffn_args(const gn_ffn* f, bool backward) {
  if (!f) return "no arguments";
  if (!type_ok(f->type)) return "type is not a gn_dtype";
  if (f->act < GN_ACT_SIGMOID || f->act > GN_ACT_RELU) return "act is not a gn_act";
  if (f->rows < 0 || f->rows >= (int64_t(1) << 31)) return "rows must be in [0, 2^31)";
  if (f->cols < 1 || f->inner < 1 || f->cols > (1 << 24) || f->inner > (1 << 24) || (int64_t)f->cols * f->inner >= (int64_t(1) << 31))
    return "cols and inner must be in [1, 2^24] with a product below 2^31";
  const struct { const gn_mat* m; int64_t cols; bool needed, rows; const char* why; } list[] = {
      {&f->x, f->cols, true, true, "x: null, misaligned, or a leading dimension below cols"},
      {&f->w_gate, f->cols, true, false, "w_gate: null, misaligned, or a leading dimension below cols"},
      {&f->w_up, f->cols, true, false, "w_up: null, misaligned, or a leading dimension below cols"},
      {&f->w_down, f->inner, true, false, "w_down: null, misaligned, or a leading dimension below inner"},
      {&f->gate, f->inner, backward, true, "gate: null, misaligned, or a leading dimension below inner"},
      {&f->up, f->inner, backward, true, "up: null, misaligned, or a leading dimension below inner"},
      {&f->y, f->cols, !backward, true, "y: null, misaligned, or a leading dimension below cols"},
      {&f->dy, f->cols, backward, true, "dy: null, misaligned, or a leading dimension below cols"},
      {&f->dx, f->cols, false, true, "dx: misaligned, or a leading dimension below cols"},
      {&f->dw_gate, f->cols, false, false, "dw_gate: misaligned, or a leading dimension below cols"},
      {&f->dw_up, f->cols, false, false, "dw_up: misaligned, or a leading dimension below cols"},
      {&f->dw_down, f->inner, false, false, "dw_down: misaligned, or a leading dimension below inner"},
  };
  for (int i = 0; i < 12; ++i) {
    if ((list[i].m == &f->y && backward) || (i >= 7 && !backward)) continue;
    if (list[i].rows && f->rows == 0) continue;
    if ((list[i].needed || list[i].m->p) && !mat_ok(list[i].m->p, list[i].m->ld, list[i].cols, f->type)) return list[i].why;
  }
  return nullptr;
}

struct Workspace {               // hands out 256-byte aligned pieces, or only counts them
  char* p; int64_t used = 0;
  void* take(int64_t bytes) { void* r = p ? p + used : nullptr; used += (bytes + 255) / 256 * 256; return r; }
};
struct Pieces { void *gate, *up, *h, *dgate, *dup; float* dh; };
int64_t lay_out(const gn_ffn& f, bool backward, char* base, Pieces& w) {
  Workspace ws{base};
  const int64_t hidden = f.rows * f.inner * type_bytes(f.type);
  w = Pieces{};
  w.h = ws.take(hidden);
  if (backward) { w.dgate = ws.take(hidden); w.dup = ws.take(hidden); w.dh = (float*)ws.take(f.rows * f.inner * 4); }
  else { w.gate = ws.take(f.gate.p ? 0 : hidden); w.up = ws.take(f.up.p ? 0 : hidden); }
  return ws.used + 256;
}

template <class T>
cudaError_t forward(const gn_ffn& f, const Pieces& w, cudaStream_t st) {
  const int64_t R = f.rows, C = f.cols, F = f.inner;
  const gn_mat gate = f.gate.p ? f.gate : gn_mat{w.gate, F}, up = f.up.p ? f.up : gn_mat{w.up, F};
  cudaError_t e = plain_gemm<T>({R, F, C, 1, {{f.x.p, f.x.ld, 1}}, {{f.w_gate.p, 1, f.w_gate.ld}}, gate.p, gate.ld}, st);
  if (e == cudaSuccess) e = plain_gemm<T>({R, F, C, 1, {{f.x.p, f.x.ld, 1}}, {{f.w_up.p, 1, f.w_up.ld}}, up.p, up.ld}, st);
  if (e == cudaSuccess) gate_kernel<T><<<1184, 256, 0, st>>>({R, f.inner, f.act, gate.p, up.p, gate.ld, up.ld, nullptr, w.h, nullptr, nullptr});
  if (e == cudaSuccess) e = plain_gemm<T>({R, C, F, 1, {{w.h, F, 1}}, {{f.w_down.p, 1, f.w_down.ld}}, f.y.p, f.y.ld}, st);
  return e;
}

template <class T>
cudaError_t backward(const gn_ffn& f, const Pieces& w, cudaStream_t st) {
  const int64_t R = f.rows, C = f.cols, F = f.inner;
  cudaError_t e = plain_gemm<T, float>({R, F, C, 1, {{f.dy.p, f.dy.ld, 1}}, {{f.w_down.p, f.w_down.ld, 1}}, w.dh, F}, st);
  if (e == cudaSuccess && R) gate_kernel<T><<<1184, 256, 0, st>>>({R, f.inner, f.act, f.gate.p, f.up.p, f.gate.ld, f.up.ld, w.dh, w.h, w.dgate, w.dup});
  if (e == cudaSuccess && f.dx.p) e = plain_gemm<T>({R, C, F, 2, {{w.dgate, F, 1}, {w.dup, F, 1}}, {{f.w_gate.p, f.w_gate.ld, 1}, {f.w_up.p, f.w_up.ld, 1}}, f.dx.p, f.dx.ld}, st);
  if (e == cudaSuccess && f.dw_gate.p) e = plain_gemm<T>({F, C, R, 1, {{w.dgate, 1, F}}, {{f.x.p, f.x.ld, 1}}, f.dw_gate.p, f.dw_gate.ld}, st);
  if (e == cudaSuccess && f.dw_up.p) e = plain_gemm<T>({F, C, R, 1, {{w.dup, 1, F}}, {{f.x.p, f.x.ld, 1}}, f.dw_up.p, f.dw_up.ld}, st);
  if (e == cudaSuccess && f.dw_down.p) e = plain_gemm<T>({C, F, R, 1, {{f.dy.p, 1, f.dy.ld}}, {{w.h, F, 1}}, f.dw_down.p, f.dw_down.ld}, st);
  return e;
}

gn_status run(const gn_ffn* f, bool back, void* d_ws, int64_t ws_bytes, void* stream, char* errbuf, int64_t errbuf_len) {
  const char* why = ffn_args(f, back);
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  Pieces w;
  if (!d_ws || ((uintptr_t)d_ws & 15) || ws_bytes < lay_out(*f, back, nullptr, w))
    return op_fail(GN_EINVAL, "workspace: null, not 16-byte aligned or too small", errbuf, errbuf_len);
  if (f->rows == 0 && !back) return op_done(cudaSuccess, errbuf, errbuf_len);
  lay_out(*f, back, (char*)(((uintptr_t)d_ws + 255) & ~(uintptr_t)255), w);
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (f->type == GN_F32) e = back ? backward<float>(*f, w, st) : forward<float>(*f, w, st);
  else if (f->type == GN_BF16) e = back ? backward<__nv_bfloat16>(*f, w, st) : forward<__nv_bfloat16>(*f, w, st);
  else e = back ? backward<__half>(*f, w, st) : forward<__half>(*f, w, st);
  return op_done(e, errbuf, errbuf_len);
}

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" int64_t gn_gated_ffn_workspace(const gn_ffn* args, int32_t backward) {
  Pieces w;
  return ffn_args(args, backward != 0) ? -1 : lay_out(*args, backward != 0, nullptr, w);
}
extern "C" gn_status gn_gated_ffn(const gn_ffn* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return run(args, false, d_ws, ws_bytes, cuda_stream, errbuf, errbuf_len);
}
extern "C" gn_status gn_gated_ffn_grad(const gn_ffn* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return run(args, true, d_ws, ws_bytes, cuda_stream, errbuf, errbuf_len);
}
