// Gated feed-forward block and its backward pass: the calls, their workspaces and the order of their products.
//
// 16-bit types: two tensor-core launches forward (both projections with the gate, then the product with Wd), two backward (dh with the
// gate's gradient, then dx and the three weight gradients as one launch; with few tokens dx is one of its own).  TMA reads the operands, so one with a base or a leading
// dimension that is no multiple of 16 bytes is copied to the workspace first.
// FP32, few tokens forward or a small backward pass: on FMAs (ffn_dot.cu, ffn_small.cu).
// FP32: the FP32-accurate products of the rest of the library (gemm_f16x3.cu, gemm_ffma.cu), with the gate as a pass of its own.
#include <math.h>

#include <atomic>

#include "ffn_act.cuh"
#include "ffn_kernels.h"
#include "gn_kernels.h"
#include "tc_common.cuh"

namespace gn {
namespace {
__device__ int ffn_error;        // code of a bounded wait that ran out
}

int* ffn_error_word() {
  static std::atomic<void*> at[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  void* p = at[dev].load(std::memory_order_acquire);
  if (!p) {
    if (cudaGetSymbolAddress(&p, ffn_error) != cudaSuccess) return nullptr;
    at[dev].store(p, std::memory_order_release);
  }
  return static_cast<int*>(p);
}

namespace {

// h = act(gate) * up, and with dh the two gradients, in FP32: a thread takes four columns, 64 threads neighbouring ones, a block four rows at a time.
struct Gates { int64_t rows; int cols, act; const float *gate, *up; int64_t ld_gate, ld_up; const float* dh; float *h, *dgate, *dup; int64_t ld; };
template <bool VEC>
__global__ void __launch_bounds__(256, VEC ? 5 : 4) gate_kernel(const Gates g) {
  const int unit = blockIdx.x * 64 + threadIdx.x, units = (g.cols + 3) / 4;
  if (unit >= units) return;
  with_activation(g.act, [&](auto act) {
    for (int64_t r = (int64_t)blockIdx.y * 4 + threadIdx.y; r < g.rows; r += (int64_t)gridDim.y * 4) {
      const auto get = [&](const float* p, int64_t ld) { return load_pack<VEC>(p + r * ld, 0, unit, units, g.cols); };
      const Pack<float> gate = get(g.gate, g.ld_gate), up = get(g.up, g.ld_up);
      Pack<float> dh = {};
      if (g.dh) dh = get(g.dh, g.ld);
      float h[4], dg[4], du[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float a, da;
        activation<decltype(act)::value, false>(gate.get(e), a, da);
        h[e] = a * up.get(e); du[e] = dh.get(e) * a; dg[e] = dh.get(e) * up.get(e) * da;
      }
      const auto put = [&](const float (&x)[4], float* p) {
        Pack<float> o;
        o.set(x);
        store_pack<VEC>(p + r * g.ld, o, 0, unit, units, g.cols);
      };
      put(h, g.h);
      if (g.dh) { put(dg, g.dgate); put(du, g.dup); }
    }
  });
}
cudaError_t launch_gate(const Gates& g, cudaStream_t st) {
  const int64_t groups = (g.rows + 3) / 4;
  const unsigned gx = (unsigned)((g.cols + 255) / 256), most = 148 * 8 / gx + 1;
  const dim3 grid(gx, (unsigned)(groups < most ? groups : most)), block(64, 4);
  if (wide_ok(g.gate, g.ld_gate, GN_F32) && wide_ok(g.up, g.ld_up, GN_F32)) gate_kernel<true><<<grid, block, 0, st>>>(g);
  else gate_kernel<false><<<grid, block, 0, st>>>(g);
  return cudaGetLastError();
}

// Copies of 16-bit matrices with rows that TMA can address: a warp per 256 columns of a row.
constexpr int kPackMax = 7;
struct PackJob { const uint16_t* src; uint16_t* dst; int64_t rows, ld, ld_out; int cols; };
struct PackList { PackJob j[kPackMax]; };
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackList list) {
  grid_dep_wait();
  grid_dep_launch();
  const PackJob& j = list.j[blockIdx.y];
  const uint16_t* const src = dep(j.src);
  const int64_t per_row = (j.cols + 255) / 256, n = j.rows * per_row, step = (int64_t)gridDim.x * 8;
  int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), r = i / per_row;
  int part = (int)(i - r * per_row);
  const int64_t step_r = step / per_row;
  const int step_part = (int)(step - step_r * per_row);
  for (; i < n; i += step) {
    const int c = part * 256 + (threadIdx.x & 31) * 8, left = j.cols - c;
    if (left > 0) {
      const uint16_t* const s = src + r * j.ld + c;
      uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) w[e >> 1] |= (uint32_t)__ldg(s + e) << (16 * (e & 1));
      *reinterpret_cast<uint4*>(j.dst + r * j.ld_out + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    r += step_r; part += step_part;
    if (part >= per_row) { part -= (int)per_row; ++r; }
  }
}

const char* ffn_args(const gn_ffn* f, bool backward) {
  if (!f) return "no arguments";
  if (!type_ok(f->type)) return "type is not a gn_dtype";
  if (f->act < GN_ACT_SIGMOID || f->act > GN_ACT_RELU) return "act is not a gn_act";
  if (f->rows < 0 || f->rows >= (int64_t(1) << 30)) return "rows must be in [0, 2^30)";
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


inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

struct Workspace {               // hands out 256-byte aligned pieces (of no memory at all where a call is only measured)
  char* p; int64_t used = 0;
  void* take(int64_t bytes) { void* r = p + used; used += (bytes + 255) / 256 * 256; return r; }
};
char* const kNowhere = reinterpret_cast<char*>(256);

// ---- 16-bit types ------------------------------------------------------------------------------
struct Half {
  Mat16 x, w_gate, w_up, w_down, dy, gate, up;      // with rows of 16-byte units, as TMA and the gate's gradient read them
  PackList packs; int n_packs; int64_t pack_warps;
  Out16 h, low, dgate, dup;               // low: see two_parts
  void* sums;                             // of slices of K
};
Mat16 addressable(const gn_mat& m, int64_t rows, int cols, Workspace& ws, Half& w) {
  if (((uintptr_t)m.p & 15) == 0 && m.ld % 8 == 0) return {m.p, m.ld};
  const int64_t ld = up8(cols);
  void* const dst = ws.take(rows * ld * 2);
  w.packs.j[w.n_packs++] = {(const uint16_t*)m.p, (uint16_t*)dst, rows, m.ld, ld, cols};
  const int64_t warps = rows * ((cols + 255) / 256);
  if (warps > w.pack_warps) w.pack_warps = warps;
  return {dst, ld};
}
inline Mat16 in16(const Out16& m) { return {m.p, m.ld}; }
inline Out16 out16(const gn_mat& m) { return {m.p, m.ld}; }
// Whether h goes to the product with Wd in two parts, rounded and what that has left.  Its rounding makes y's error sqrt 2 times that of y's own, and more where
// few values make it up (1.6, one token and 25 hidden units).  The second pass over Wd, 2 MB of it at most, takes 0.2 to 0.9 us (1 x 64 x 128 6.0 and 6.9, 128 x 1024 x
// 1024 13.0 and 13.7); with more hidden units, whose roundings average, it would take more (1 x 512 x 2048 8.4 and 10.0, 128 x 128 x 8192 19 and 26).
bool two_parts(const gn_ffn& f, bool backward) {
  return !backward && f.rows <= kFfnNarrow && f.inner <= 1024 && (int64_t)f.cols * f.inner <= (1 << 20);
}
// The plain products of a call, in the order they run: forward the one with Wd, backward dx and the weights' gradients.
int plain_products(const gn_ffn& f, bool backward, const Half& w, FfnGemm (&list)[kFfnGroup]) {
  const int R = (int)f.rows;
  int n = 0;
  if (!backward) {
    FfnGemm& q = list[n++];
    q.M = R; q.N = f.cols; q.K[0] = f.inner;
    q.A[0] = in16(w.h); q.B[0] = w.w_down; q.d[0] = out16(f.y);
    if (two_parts(f, backward)) { q.K[1] = f.inner; q.A[1] = in16(w.low); q.B[1] = w.w_down; }
    return n;
  }
  if (f.dx.p) {
    FfnGemm& q = list[n++];
    q.M = R; q.N = f.cols; q.K[0] = q.K[1] = f.inner; q.b_mn = true;
    q.A[0] = in16(w.dgate); q.B[0] = w.w_gate; q.A[1] = in16(w.dup); q.B[1] = w.w_up; q.d[0] = out16(f.dx);
  }
  auto weights = [&](int M, int N, const Mat16& A, const Mat16& B, const gn_mat& d) {
    if (!d.p) return;
    FfnGemm& q = list[n++];
    q.M = M; q.N = N; q.K[0] = R; q.a_mn = q.b_mn = true; q.A[0] = A; q.B[0] = B; q.d[0] = out16(d);
  };
  weights(f.inner, f.cols, in16(w.dgate), w.x, f.dw_gate);
  weights(f.inner, f.cols, in16(w.dup), w.x, f.dw_up);
  weights(f.cols, f.inner, w.dy, in16(w.h), f.dw_down);
  return n;
}
// Which products go to the kernel for few tokens: the call's first one, and the first of the list above (y, or dx).  By sizes alone.
struct Few { bool first; int listed; };
Few few_tokens(const gn_ffn& f, bool backward, const FfnGemm* list, int n) {
  const FfnKind kind = backward ? FFN_GRAD : FFN_GATE;
  const bool candidate = !backward || f.dx.p;              // (a weight's gradient has a long K and many rows: never)
  if (f.rows <= kFfnNarrow) return {true, candidate ? 1 : 0};
  if (f.rows > 4096) return {false, 0};
  const int R = (int)f.rows;
  Few c{ffn_narrow_us(kind, R, f.inner, f.cols) < ffn_pair_us(kind, R, f.inner, f.cols), 0};
  if (candidate && n > 0)
    c.listed = ffn_narrow_us(FFN_STORE, R, f.cols, list[0].K[0] + list[0].K[1]) + ffn_pair_list_us(list + 1, n - 1) < ffn_pair_list_us(list, n) ? 1 : 0;
  return c;
}

int64_t lay_out_half(const gn_ffn& f, bool backward, char* base, Half& w) {
  Workspace ws{base};
  w = Half{};
  const int64_t ld = up8(f.inner);
  w.x = addressable(f.x, f.rows, f.cols, ws, w);
  w.w_gate = addressable(f.w_gate, f.inner, f.cols, ws, w);
  w.w_up = addressable(f.w_up, f.inner, f.cols, ws, w);
  w.w_down = addressable(f.w_down, f.cols, f.inner, ws, w);
  if (backward) {
    w.dy = addressable(f.dy, f.rows, f.cols, ws, w);
    w.gate = addressable(f.gate, f.rows, f.inner, ws, w);
    w.up = addressable(f.up, f.rows, f.inner, ws, w);
  }
  for (Out16* o : {&w.h, &w.low, &w.dgate, &w.dup}) {
    if (o == &w.low ? !two_parts(f, backward) : o != &w.h && !backward) continue;
    *o = {ws.take(f.rows * ld * 2), ld};
  }
  FfnGemm list[kFfnGroup];
  const int n = plain_products(f, backward, w, list), few = f.rows > 0 ? few_tokens(f, backward, list, n).listed : 0;
  w.sums = f.rows > 0 && n > few ? ws.take(ffn_pair_workspace(list + few, n - few)) : nullptr;
  return ws.used;
}
cudaError_t pack(const Half& w, cudaStream_t st) {
  if (w.n_packs == 0) return cudaSuccess;
  const int64_t blocks = (w.pack_warps + 7) / 8;
  return launch_pdl_grid(pack_kernel, dim3((unsigned)(blocks < 1184 ? blocks : 1184), (unsigned)w.n_packs), 256, 0, st, w.packs);
}

cudaError_t run_half(const gn_ffn& f, bool backward, const Half& w, int* err, cudaStream_t st) {
  const bool bf16 = f.type == GN_BF16;
  FfnGemm list[kFfnGroup], a;
  const int n = plain_products(f, backward, w, list);
  if (n == 0) return cudaSuccess;
  a.M = (int)f.rows; a.N = f.inner; a.K[0] = f.cols;
  a.d[0] = w.h; a.low = w.low;
  if (backward) {
    a.b_mn = true;
    a.A[0] = w.dy; a.B[0] = w.w_down; a.d[1] = w.dgate; a.d[2] = w.dup;
    a.gate = w.gate; a.up = w.up;
  } else {
    a.A[0] = w.x; a.B[0] = w.w_gate; a.B[1] = w.w_up; a.d[1] = out16(f.gate); a.d[2] = out16(f.up);
  }
  const FfnKind first = backward ? FFN_GRAD : FFN_GATE;
  const Few choice = few_tokens(f, backward, list, n);
  const bool narrow = choice.first;
  const int few = choice.listed;
  cudaError_t e = pack(w, st);
  if (e == cudaSuccess) e = narrow ? launch_ffn_narrow(first, bf16, f.act, a, false, err, st) : launch_ffn_pair(first, bf16, f.act, &a, 1, nullptr, err, st);
  if (e == cudaSuccess && few) e = launch_ffn_narrow(FFN_STORE, bf16, f.act, list[0], true, err, st);
  if (e == cudaSuccess && n > few) e = launch_ffn_pair(FFN_STORE, bf16, f.act, list + few, n - few, w.sums, err, st);
  return e;
}

// ---- FP32 --------------------------------------------------------------------------------------
struct Stored { const float* p; int64_t rows; int cols; int64_t ld; };
// The two FP16 parts of a call's operands, each split once however many products read it: what the caller gives in one launch at the start (phase
// 0), what the gate has written in one after it.
struct Parts {
  int n;
  Stored m[8];
  int phase[8];
  SplitJob job[8];
  SplitOperand op[8];
};
struct Single { float *gate, *up, *h, *dgate, *dup, *dh; int64_t ld; Parts parts; float* sums; };

// Whether the tensor-core form is the faster way to FP32 accuracy (the rule of the contexts' contractions, see gn_context.cu).
bool on_tensor_cores(const GemmArgs& g) {
  if (!gemm_f16x3_usable()) return false;
  const double K = (double)g.K1 + (g.A2 ? g.K2 : 0);
  const double blocks = ((g.M + 127) / 128) * (double)((g.N + 127) / 128);
  const double fma_us = 10.0 + (blocks <= 148.0 ? 1.0 : blocks / 148.0) * K * 0.12;
  return gemm_f16x3_estimate_us(g) + 14.0 + (g.M + (double)g.N) * K * 8.0 / 4.0e6 * 0.5 < fma_us;
}

// One product: its operands as stored.
GemmArgs product(int64_t M, int64_t N, const Stored& A, bool a_k, const Stored& B, bool b_k, float* D, int64_t ldd) {
  GemmArgs g;
  g.M = (int)M; g.N = (int)N;
  g.A1 = A.p; g.lda1 = A.ld; g.B1 = B.p; g.ldb1 = B.ld; g.K1 = a_k ? A.cols : (int)A.rows;
  g.a_kmajor = a_k; g.b_kmajor = b_k; g.D = D; g.ldd = ldd;
  g.chunk_kb = M > 128 && N >= 128 ? 2 : 1;
  return g;
}
// Operand k of A1, B1, A2, B2.
Stored stored(const GemmArgs& g, int k) {
  const int s = k / 2, K = s ? g.K2 : g.K1;
  if (k % 2 == 0) {
    const float* p = s ? g.A2 : g.A1; const int64_t ld = s ? g.lda2 : g.lda1;
    return g.a_kmajor ? Stored{p, g.M, K, ld} : Stored{p, K, g.M, ld};
  }
  const float* p = s ? g.B2 : g.B1; const int64_t ld = s ? g.ldb2 : g.ldb1;
  return g.b_kmajor ? Stored{p, g.N, K, ld} : Stored{p, K, g.N, ld};
}
int find_parts(const Parts& t, const Stored& m) {
  for (int i = 0; i < t.n; ++i)
    if (t.m[i].p == m.p && t.m[i].rows == m.rows && t.m[i].cols == m.cols && t.m[i].ld == m.ld) return i;
  return -1;
}

struct SingleCall { GemmArgs g[6]; int n, gate_after; };   // products, the gate's pass after the first gate_after of them
SingleCall single_products(const gn_ffn& f, bool backward, const Single& w) {
  SingleCall c{};
  const int64_t R = f.rows;
  const int C = f.cols, F = f.inner;
  const Stored x{(const float*)f.x.p, R, C, f.x.ld}, wg{(const float*)f.w_gate.p, F, C, f.w_gate.ld}, wu{(const float*)f.w_up.p, F, C, f.w_up.ld};
  const Stored wd{(const float*)f.w_down.p, C, F, f.w_down.ld}, h{w.h, R, F, w.ld};
  if (!backward) {
    c.g[c.n++] = product(R, F, x, true, wg, true, w.gate, f.gate.p ? f.gate.ld : w.ld);
    c.g[c.n++] = product(R, F, x, true, wu, true, w.up, f.up.p ? f.up.ld : w.ld);
    c.gate_after = c.n;
    c.g[c.n++] = product(R, C, h, true, wd, true, (float*)f.y.p, f.y.ld);
    return c;
  }
  const Stored dy{(const float*)f.dy.p, R, C, f.dy.ld}, dg{w.dgate, R, F, w.ld}, du{w.dup, R, F, w.ld};
  c.g[c.n++] = product(R, F, dy, true, wd, false, w.dh, w.ld);
  c.gate_after = c.n;
  if (f.dx.p) {
    GemmArgs& g = c.g[c.n++] = product(R, C, dg, true, wg, false, (float*)f.dx.p, f.dx.ld);
    g.A2 = du.p; g.lda2 = du.ld; g.B2 = wu.p; g.ldb2 = wu.ld; g.K2 = F;
  }
  if (f.dw_gate.p) c.g[c.n++] = product(F, C, dg, false, x, false, (float*)f.dw_gate.p, f.dw_gate.ld);
  if (f.dw_up.p) c.g[c.n++] = product(F, C, du, false, x, false, (float*)f.dw_up.p, f.dw_up.ld);
  if (f.dw_down.p) c.g[c.n++] = product(C, F, dy, false, h, false, (float*)f.dw_down.p, f.dw_down.ld);
  return c;
}
int64_t lay_out_single(const gn_ffn& f, bool backward, char* base, Single& w) {
  Workspace ws{base};
  w = Single{};
  w.ld = up8(f.inner);
  const int64_t hidden = f.rows * w.ld * 4;
  w.h = (float*)ws.take(hidden);
  if (backward) {
    w.dgate = (float*)ws.take(hidden); w.dup = (float*)ws.take(hidden); w.dh = (float*)ws.take(hidden);
  } else {
    w.gate = f.gate.p ? (float*)f.gate.p : (float*)ws.take(hidden);
    w.up = f.up.p ? (float*)f.up.p : (float*)ws.take(hidden);
  }
  const SingleCall c = single_products(f, backward, w);
  int64_t sums = 0;
  Parts& t = w.parts;
  for (int i = 0; i < c.n && f.rows > 0; ++i) {
    const GemmArgs& g = c.g[i];
    if (!on_tensor_cores(g)) continue;
    const int64_t b = gemm_f16x3_workspace_floats(g) * 4;
    sums = b > sums ? b : sums;
    for (int k = 0; k < (g.A2 ? 4 : 2); ++k) {
      const Stored m = stored(g, k);
      if (find_parts(t, m) >= 0) continue;
      const int64_t ld = up8(m.cols), cells = (m.rows + 127) / 128 * ((m.cols + 127) / 128);
      t.m[t.n] = m;
      t.phase[t.n] = m.p == w.h || m.p == w.dgate || m.p == w.dup;
      t.job[t.n] = {m.p, m.rows, m.cols, m.ld, ws.take(m.rows * ld * 2), ws.take(m.rows * ld * 2), ld, (int8_t*)ws.take(cells)};
      SplitOperand& o = t.op[t.n];
      o.hi = t.job[t.n].hi; o.lo = t.job[t.n].lo; o.ld = ld; o.cells = t.job[t.n].cells; o.cells_ld = (m.cols + 127) / 128;
      ++t.n;
    }
  }
  w.sums = (float*)ws.take(sums);
  return ws.used;
}
cudaError_t own_error() {             // what a launch of the library's that says -1 has left
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? cudaErrorInvalidValue : e;
}
cudaError_t split_phase(const Parts& t, int phase, cudaStream_t st) {
  SplitJob jobs[8];
  int n = 0;
  for (int i = 0; i < t.n; ++i)
    if (t.phase[i] == phase) jobs[n++] = t.job[i];
  return n > 0 && launch_split_f16(jobs, n, st) < 0 ? own_error() : cudaSuccess;
}
cudaError_t run_product(const GemmArgs& g, const Single& w, int* err, cudaStream_t st) {
  if (!on_tensor_cores(g)) { launch_gemm_ffma(g, st); return cudaGetLastError(); }
  SplitOperand ops[4];
  for (int k = 0; k < (g.A2 ? 4 : 2); ++k) ops[k] = w.parts.op[find_parts(w.parts, stored(g, k))];
  return launch_gemm_f16x3(g, ops, w.sums, err, st) < 0 ? own_error() : cudaSuccess;
}
cudaError_t run_single(const gn_ffn& f, bool backward, const Single& w, int* err, cudaStream_t st) {
  const SingleCall c = single_products(f, backward, w);
  if (backward && c.n == 1) return cudaSuccess;
  cudaError_t e = split_phase(w.parts, 0, st);
  for (int i = 0; i < c.n && e == cudaSuccess; ++i) {
    if (i == c.gate_after) {
      e = launch_gate(backward ? Gates{f.rows, f.inner, f.act, (const float*)f.gate.p, (const float*)f.up.p, f.gate.ld, f.up.ld, w.dh, w.h, w.dgate, w.dup, w.ld}
                               : Gates{f.rows, f.inner, f.act, w.gate, w.up, f.gate.p ? f.gate.ld : w.ld, f.up.p ? f.up.ld : w.ld, nullptr, w.h, nullptr, nullptr, w.ld}, st);
      if (e == cudaSuccess) e = split_phase(w.parts, 1, st);
    }
    if (e == cudaSuccess) e = run_product(c.g[i], w, err, st);
  }
  return e;
}

cudaError_t clear(const gn_mat& m, int64_t rows, int64_t cols, int type, cudaStream_t st) {
  const size_t b = (size_t)type_bytes(type);
  return m.p ? cudaMemset2DAsync(m.p, (size_t)m.ld * b, 0, (size_t)cols * b, (size_t)rows, st) : cudaSuccess;
}

// ---- few FP32 tokens ---------------------------------------------------------------------------
// Forward by ffn_dot.cu where its estimated time, in us, is the smaller one: its sums end in shuffles (0.085 a thousand of them), its FMAs run at 33 TFLOP/s;
// the three products at FP32 accuracy take six launches, their k-blocks and the weights' parts.  Measured, here and there: 9 x 64 x 128 5.3 and 33,
// 64 x 256 x 512 14 and 31, 64 x 617 x 1201 46 and 56, 128 x 617 x 1201 75 and 57, 16 x 2048 x 4096 102 and 137, 64 x 2048 x 4096 263 and 139.
bool on_fmas(const gn_ffn& f, bool backward) {
  if (backward || f.type != GN_F32) return false;
  if (f.rows <= kFfnDot) return true;
  const double R = (double)((f.rows + 7) / 8 * 8), C = f.cols, F = f.inner, C128 = (f.cols + 127) / 128 * 128.0, F128 = (f.inner + 127) / 128 * 128.0;
  const double fmas = 5.0 + 85e-6 * R * (2 * F + C) + 60e-9 * R * (2 * F * C128 + C * F128) * 2;
  const double products = 27.0 + 0.011 * (C + F) + 5.5e-6 * C * F + R * C * F * 18 / 1.2e9;
  return fmas < products;
}
cudaError_t run_fmas(const gn_ffn& f, float* h, cudaStream_t st) {
  const int64_t ld = up8(f.inner);
  const auto in = [](const gn_mat& m) { return FfnMat{(const float*)m.p, m.ld}; };
  const auto out = [](const gn_mat& m) { return FfnOut{(float*)m.p, m.ld}; };
  const FfnDot a{(int)f.rows, f.inner, f.cols, f.act, in(f.x), {in(f.w_gate), in(f.w_up)}, {{h, ld}, out(f.gate), out(f.up)}};
  const FfnDot b{(int)f.rows, f.cols, f.inner, f.act, {h, ld}, {in(f.w_down), {}}, {out(f.y), {}, {}}};
  const cudaError_t e = launch_ffn_dot(a, st);
  return e == cudaSuccess ? launch_ffn_dot(b, st) : e;
}

// ---- a small FP32 backward pass ----------------------------------------------------------------
struct Small { FfnSmall dh, list[kFfnGroup]; int n; FfnSmallGrad grad; int64_t bytes; };
Small lay_out_small(const gn_ffn& f, char* base) {
  const auto in = [](const gn_mat& m) { return FfnMat{(const float*)m.p, m.ld}; };
  const auto out = [](const gn_mat& m) { return FfnOut{(float*)m.p, m.ld}; };
  Workspace ws{base};
  Small w{};
  const int R = (int)f.rows, C = f.cols, F = f.inner;
  FfnMat part[3];
  for (int k = 0; k < 3; ++k) {
    w.grad.out[k] = {(float*)ws.take(f.rows * up8(F) * 4), up8(F)};
    part[k] = {w.grad.out[k].p, w.grad.out[k].ld};
  }
  w.grad.act = f.act; w.grad.gate = in(f.gate); w.grad.up = in(f.up);
  w.dh.M = R; w.dh.N = F; w.dh.K[0] = C; w.dh.A[0] = in(f.dy); w.dh.B[0] = in(f.w_down);
  if (f.dx.p) {
    FfnSmall& q = w.list[w.n++];
    q.M = R; q.N = C; q.K[0] = q.K[1] = F; q.A[0] = part[1]; q.B[0] = in(f.w_gate); q.A[1] = part[2]; q.B[1] = in(f.w_up); q.d = out(f.dx);
  }
  const auto weights = [&](int M, int N, const FfnMat& A, const FfnMat& B, const gn_mat& d) {
    if (!d.p) return;
    FfnSmall& q = w.list[w.n++];
    q.M = M; q.N = N; q.K[0] = R; q.a_mn = true; q.A[0] = A; q.B[0] = B; q.d = out(d);
  };
  weights(F, C, part[1], in(f.x), f.dw_gate);
  weights(F, C, part[2], in(f.x), f.dw_up);
  weights(C, F, in(f.dy), part[0], f.dw_down);
  w.bytes = ws.used;
  return w;
}
// Where its estimated time, in us, is the smaller one; the products at FP32 accuracy and what goes with them take 40 to 60 whatever the size, of which the wanted ones
// their share.  Measured, here and there: 32 x 64 x 128 9.3 and 50, 1000 x 64 x 512 41 and 68, 32 x 617 x 1201 55 and 77, 300 x 300 x 784 64 and 56.
bool is_small(const gn_ffn& f, bool backward) {
  if (!backward || f.type != GN_F32 || f.rows > (1 << 20)) return false;
  const Small w = lay_out_small(f, kNowhere);
  const double R = (double)f.rows, C = f.cols, F = f.inner;
  const double products = (40.0 + 0.011 * (C + F) + 8e-6 * C * F + 0.005 * R + R * C * F * 36 / 1.2e9) * (1 + w.n) / 5.0;
  return ffn_small_us(&w.dh, 1) + ffn_small_us(w.list, w.n) < products;
}
cudaError_t run_small(const Small& w, cudaStream_t st) {
  if (w.n == 0) return cudaSuccess;
  const cudaError_t e = launch_ffn_small(&w.dh, 1, &w.grad, st);
  return e == cudaSuccess ? launch_ffn_small(w.list, w.n, nullptr, st) : e;
}

int64_t needed(const gn_ffn& f, bool backward, char* base, Half& h, Single& s) {
  if (is_small(f, backward)) return lay_out_small(f, base).bytes + 256;
  if (on_fmas(f, backward)) return f.rows * up8(f.inner) * 4 + 256;
  return (f.type == GN_F32 ? lay_out_single(f, backward, base, s) : lay_out_half(f, backward, base, h)) + 256;
}

gn_status run(const gn_ffn* f, bool back, void* d_ws, int64_t ws_bytes, void* stream, char* errbuf, int64_t errbuf_len) {
  const char* why = ffn_args(f, back);
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  Half h;
  Single s;
  char* const base = (char*)(((uintptr_t)d_ws + 255) & ~(uintptr_t)255);
  if (!d_ws || ((uintptr_t)d_ws & 15) || ws_bytes < needed(*f, back, base, h, s))
    return op_fail(GN_EINVAL, "workspace: null, not 16-byte aligned or too small", errbuf, errbuf_len);
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  if (f->rows == 0) {
    if (back) {
      e = clear(f->dw_gate, f->inner, f->cols, f->type, st);
      if (e == cudaSuccess) e = clear(f->dw_up, f->inner, f->cols, f->type, st);
      if (e == cudaSuccess) e = clear(f->dw_down, f->cols, f->inner, f->type, st);
    }
    return op_done(e, errbuf, errbuf_len);
  }
  int* const err = ffn_error_word();
  if (!err) return op_done(cudaErrorNoDevice, errbuf, errbuf_len);
  if (on_fmas(*f, back)) e = run_fmas(*f, (float*)base, st);
  else if (is_small(*f, back)) e = run_small(lay_out_small(*f, base), st);
  else if (f->type == GN_F32) e = run_single(*f, back, s, err, st);
  else e = run_half(*f, back, h, err, st);
  return op_done(e, errbuf, errbuf_len);
}

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" int64_t gn_gated_ffn_workspace(const gn_ffn* args, int32_t backward) {
  Half h;
  Single s;
  return ffn_args(args, backward != 0) ? -1 : needed(*args, backward != 0, kNowhere, h, s);
}
extern "C" gn_status gn_gated_ffn(const gn_ffn* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return run(args, false, d_ws, ws_bytes, cuda_stream, errbuf, errbuf_len);
}
extern "C" gn_status gn_gated_ffn_grad(const gn_ffn* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return run(args, true, d_ws, ws_bytes, cuda_stream, errbuf, errbuf_len);
}
extern "C" gn_status gn_gated_ffn_status(void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  int* const err = ffn_error_word();
  if (!err) return op_done(cudaErrorNoDevice, errbuf, errbuf_len);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  int code = 0;
  cudaError_t e = cudaMemcpyAsync(&code, err, sizeof code, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess || code == 0) return op_done(e, errbuf, errbuf_len);
  e = cudaMemsetAsync(err, 0, sizeof code, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return op_done(e, errbuf, errbuf_len);
  return op_fail(GN_ETIMEOUT, "a bounded wait of a tensor-core kernel ran out: results since the last look are invalid", errbuf, errbuf_len);
}
