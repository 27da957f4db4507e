// A mixture's experts and their backward pass: the calls, their workspaces and the order of their products.
//
// 16-bit types, forward: the plan (which pairs of token and choice are whose), the tokens to the experts' slots, both projections with the gate, the product
// with Wd, the weighted sums of each token's results.  Backward: the plan again (it is cheaper than to keep it), x and dy to the slots, q = dy Wd with the gate's
// gradient, dx's two products, the three weight gradients as one launch, and each token's sums.
// FP32: the same products on the tensor cores, operands in three parts, or on FMAs, rows read where they lie.
// Nothing is read by the host: how many tokens an expert has only the device knows, and grids are for what there can be.
#include <math.h>

#include "expert_kernels.h"
#include "op_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

struct Workspace {               // hands out 256-byte aligned pieces (of no memory at all where a call is only measured)
  char* p; int64_t used = 0;
  void* take(int64_t bytes) { void* r = p + used; used += (bytes + 255) / 256 * 256; return r; }
};
char* const kNowhere = reinterpret_cast<char*>(256);
inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

const char* mixture_args(const gn_mixture* f, bool backward) {
  if (!f) return "no arguments";
  if (!type_ok(f->type)) return "type is not a gn_dtype";
  if (f->act < GN_ACT_SIGMOID || f->act > GN_ACT_RELU) return "act is not a gn_act";
  if (f->experts < 1 || f->experts > kMostExperts) return "experts must be in [1, 1024]";
  if (f->k < 1 || f->k > 32) return "k must be in [1, 32]";
  if (f->tokens < 0 || f->tokens >= (int64_t(1) << 28) || f->tokens * f->k >= (int64_t(1) << 28)) return "tokens times k must be in [0, 2^28)";
  if (f->cols < 1 || f->inner < 1 || f->cols > (1 << 20) || f->inner > (1 << 20) || (int64_t)f->cols * f->inner >= (int64_t(1) << 31))
    return "cols and inner must be in [1, 2^20] with a product below 2^31";
  const int64_t C = f->cols, F = f->inner;
  const struct { const gn_stack* m; int64_t rows, cols; bool needed, used; const char* why; } stacks[] = {
      {&f->w_gate, F, C, true, true, "w_gate: null, misaligned, or a leading dimension or stride too small"},
      {&f->w_up, F, C, true, true, "w_up: null, misaligned, or a leading dimension or stride too small"},
      {&f->w_down, C, F, true, true, "w_down: null, misaligned, or a leading dimension or stride too small"},
      {&f->dw_gate, F, C, false, backward, "dw_gate: misaligned, or a leading dimension or stride too small"},
      {&f->dw_up, F, C, false, backward, "dw_up: misaligned, or a leading dimension or stride too small"},
      {&f->dw_down, C, F, false, backward, "dw_down: misaligned, or a leading dimension or stride too small"},
  };
  for (const auto& s : stacks) {
    if (!s.used || (!s.needed && !s.m->p)) continue;
    if (!mat_ok(s.m->p, s.m->ld, s.cols, f->type)) return s.why;
    if (f->experts > 1 && (s.m->stride < (s.rows - 1) * s.m->ld + s.cols || s.m->stride >= (int64_t(1) << 40))) return s.why;
  }
  if (f->tokens == 0) return nullptr;
  const struct { const gn_mat* m; int64_t cols; bool needed, used; const char* why; } mats[] = {
      {&f->x, C, true, true, "x: null, misaligned, or a leading dimension below cols"},
      {&f->y, C, true, !backward, "y: null, misaligned, or a leading dimension below cols"},
      {&f->gate, F, backward, true, "gate: null, misaligned, or a leading dimension below inner"},
      {&f->up, F, backward, true, "up: null, misaligned, or a leading dimension below inner"},
      {&f->dy, C, true, backward, "dy: null, misaligned, or a leading dimension below cols"},
      {&f->dx, C, false, backward, "dx: misaligned, or a leading dimension below cols"},
  };
  for (const auto& m : mats)
    if (m.used && (m.needed || m.m->p) && !mat_ok(m.m->p, m.m->ld, m.cols, f->type)) return m.why;
  if (!f->index || ((uintptr_t)f->index & 3)) return "index: null or misaligned";
  if (!f->weight || ((uintptr_t)f->weight & 3)) return "weight: null or misaligned";
  if (backward && ((uintptr_t)f->dweight & 3)) return "dweight: misaligned";
  return nullptr;
}

// ---- 16-bit types ------------------------------------------------------------------------------
struct Half {
  ExpertPlan plan;
  Mat16 x, dy, gate, up;         // x, dy: in slots
  Weights16 w_gate, w_up, w_down;
  PackMats packs[kPackMats]; int n_packs;
  Out16 h, dgate, dup;           // in slots
  float* parts;
  FfnOut out;                    // of the pairs
  int64_t slots;
};
Weights16 addressable(const gn_stack& m, int experts, int64_t rows, int cols, Workspace& ws, Half& w) {
  if (((uintptr_t)m.p & 15) == 0 && m.ld % 8 == 0 && (experts == 1 || m.stride % 8 == 0)) return {m.p, m.ld, experts == 1 ? rows * m.ld : m.stride};
  const int64_t ld = up8(cols);
  void* const dst = ws.take(experts * rows * ld * 2);
  w.packs[w.n_packs++] = {m.p, dst, m.ld, experts == 1 ? 0 : m.stride, ld, rows, experts, cols};
  return {dst, ld, rows * ld};
}
Mat16 addressable(const gn_mat& m, int64_t rows, int cols, Workspace& ws, Half& w) {
  const Weights16 a = addressable(gn_stack{m.p, m.ld, 0}, 1, rows, cols, ws, w);
  return {a.p, a.ld};
}
bool any_weights(const gn_mixture& f) { return f.dw_gate.p || f.dw_up.p || f.dw_down.p; }

int64_t lay_out_half(const gn_mixture& f, bool backward, char* base, Half& w) {
  Workspace ws{base};
  w = Half{};
  const int64_t pairs = f.tokens * f.k, lc = up8(f.cols), lf = up8(f.inner);
  w.slots = plan_slots(pairs, f.experts);
  w.plan = plan_at((int*)ws.take(plan_ints(pairs, f.experts, kGroupHeight) * 4), pairs, f.experts, kGroupHeight);
  if (!backward || f.dx.p) {
    w.w_gate = addressable(f.w_gate, f.experts, f.inner, f.cols, ws, w);
    w.w_up = addressable(f.w_up, f.experts, f.inner, f.cols, ws, w);
  }
  w.w_down = addressable(f.w_down, f.experts, f.cols, f.inner, ws, w);
  if (!backward || any_weights(f)) w.x = {ws.take(w.slots * lc * 2), lc};
  w.h = {ws.take(w.slots * lf * 2), lf};
  if (backward) {
    w.dy = {ws.take(w.slots * lc * 2), lc};
    w.gate = addressable(f.gate, pairs, f.inner, ws, w);
    w.up = addressable(f.up, pairs, f.inner, ws, w);
    w.dgate = {ws.take(w.slots * lf * 2), lf};
    w.dup = {ws.take(w.slots * lf * 2), lf};
    w.parts = (float*)ws.take(w.slots * group_parts(f.inner) * 4);
  }
  if (!backward || f.dx.p) w.out = {(float*)ws.take(pairs * lc * 4), lc};
  return ws.used;
}

Mat16 in16(const Out16& m) { return {m.p, m.ld}; }

cudaError_t run_half(const gn_mixture& f, bool backward, const Half& w, int* err, cudaStream_t st) {
  const bool bf16 = f.type == GN_BF16;
  cudaError_t e = launch_pack_mats(w.packs, w.n_packs, st);
  if (e == cudaSuccess) e = launch_plan(f.index, w.plan, kGroupHeight, st);
  RowCopy rows[2];
  int n = 0;
  if (w.x.p) rows[n++] = {f.x.p, f.x.ld, const_cast<void*>(w.x.p), w.x.ld};
  if (backward) rows[n++] = {f.dy.p, f.dy.ld, const_cast<void*>(w.dy.p), w.dy.ld};
  if (e == cudaSuccess) e = launch_to_slots(rows, n, f.tokens, f.k, f.cols, backward, w.plan, st);
  GroupGemm g;
  g.act = f.act; g.slots = w.slots;
  Combine c = {};
  c.tokens = f.tokens; c.k = f.k; c.cols = f.cols; c.experts = f.experts; c.index = f.index; c.src = w.out.p; c.ld = w.out.ld;
  if (!backward) {
    g.N = f.inner; g.K = f.cols; g.A[0] = w.x; g.B[0] = w.w_gate; g.B[1] = w.w_up; g.d = w.h; g.gate_out = {f.gate.p, f.gate.ld}; g.up_out = {f.up.p, f.up.ld};
    if (e == cudaSuccess) e = launch_group(GROUP_GATE, bf16, g, w.plan, err, st);
    GroupGemm q;
    q.slots = w.slots; q.N = f.cols; q.K = f.inner; q.A[0] = in16(w.h); q.B[0] = w.w_down; q.rows = w.out;
    if (e == cudaSuccess) e = launch_group(GROUP_DOWN, bf16, q, w.plan, err, st);
    c.weight = f.weight; c.d = f.y.p; c.ld_d = f.y.ld;
    return e == cudaSuccess ? launch_combine(f.type, c, st) : e;
  }
  g.N = f.inner; g.K = f.cols; g.A[0] = w.dy; g.B[0] = w.w_down; g.d = w.h; g.dgate = w.dgate; g.dup = w.dup; g.gate = w.gate; g.up = w.up;
  g.weight = f.weight; g.parts = w.parts;
  if (e == cudaSuccess) e = launch_group(GROUP_GRAD, bf16, g, w.plan, err, st);
  if (f.dx.p) {
    GroupGemm q;
    q.slots = w.slots; q.N = f.cols; q.K = f.inner; q.A[0] = in16(w.dgate); q.A[1] = in16(w.dup); q.B[0] = w.w_gate; q.B[1] = w.w_up; q.rows = w.out;
    if (e == cudaSuccess) e = launch_group(GROUP_DX, bf16, q, w.plan, err, st);
  }
  if (any_weights(f)) {
    GroupGemm q;
    q.slots = w.slots;
    const auto add = [&](int M, int N, const Mat16& left, const Mat16& right, const gn_stack& d) {
      if (!d.p) return;
      auto& t = q.grads[q.n_grads++];
      t.M = M; t.N = N; t.left = left; t.right = right; t.d = {d.p, d.ld, d.stride};
    };
    add(f.inner, f.cols, in16(w.dgate), w.x, f.dw_gate);
    add(f.inner, f.cols, in16(w.dup), w.x, f.dw_up);
    add(f.cols, f.inner, w.dy, in16(w.h), f.dw_down);
    if (e == cudaSuccess) e = launch_group(GROUP_WEIGHT, bf16, q, w.plan, err, st);
  }
  c.d = f.dx.p; c.ld_d = f.dx.ld;
  if (f.dweight) { c.parts = w.parts; c.n_parts = group_parts(f.inner); c.slot_of = w.plan.slot_of; c.dweight = f.dweight; }
  return e == cudaSuccess && (c.d || c.parts) ? launch_combine(f.type, c, st) : e;
}

// ---- FP32 --------------------------------------------------------------------------------------
struct Single { ExpertPlan plan; bool small; int height; FfnOut h, dgate, dup, out; float* parts; };
int64_t lay_out_single(const gn_mixture& f, bool backward, char* base, Single& w) {
  Workspace ws{base};
  w = Single{};
  const int64_t pairs = f.tokens * f.k, lc = up8(f.cols), lf = up8(f.inner);
  w.small = fma_small(pairs, f.experts, f.cols, f.inner);
  w.height = w.small ? kFmaSmall : kFmaHeight;
  w.plan = plan_at((int*)ws.take(plan_ints(pairs, f.experts, w.height) * 4), pairs, f.experts, w.height);
  w.h = {(float*)ws.take(pairs * lf * 4), lf};
  if (backward) {
    w.dgate = {(float*)ws.take(pairs * lf * 4), lf};
    w.dup = {(float*)ws.take(pairs * lf * 4), lf};
    w.parts = (float*)ws.take(plan_slots(pairs, f.experts) * fma_parts(f.inner, w.small) * 4);
  }
  if (!backward || f.dx.p) w.out = {(float*)ws.take(pairs * lc * 4), lc};
  return ws.used;
}
cudaError_t run_single(const gn_mixture& f, bool backward, const Single& w, cudaStream_t st) {
  const auto in = [](const gn_mat& m) { return FfnMat{(const float*)m.p, m.ld}; };
  const auto of = [](const FfnOut& m) { return FfnMat{m.p, m.ld}; };
  const auto weights = [](const gn_stack& m) { return Weights32{(const float*)m.p, m.ld, m.stride}; };
  cudaError_t e = launch_plan(f.index, w.plan, w.height, st);
  FmaGroup g, q;
  g.act = f.act; g.k = q.k = f.k; g.N = f.inner; g.K = f.cols; g.token_rows = true; g.d = w.h;
  q.N = f.cols; q.K = f.inner; q.d = w.out;
  Combine c = {};
  c.tokens = f.tokens; c.k = f.k; c.cols = f.cols; c.experts = f.experts; c.index = f.index; c.src = w.out.p; c.ld = w.out.ld;
  if (!backward) {
    g.A[0] = in(f.x); g.B[0] = weights(f.w_gate); g.B[1] = weights(f.w_up);
    g.gate_out = {(float*)f.gate.p, f.gate.ld}; g.up_out = {(float*)f.up.p, f.up.ld};
    if (e == cudaSuccess) e = launch_group_fma(GROUP_GATE, g, w.small, w.plan, st);
    q.A[0] = of(w.h); q.B[0] = weights(f.w_down);
    if (e == cudaSuccess) e = launch_group_fma(GROUP_DOWN, q, w.small, w.plan, st);
    c.weight = f.weight; c.d = f.y.p; c.ld_d = f.y.ld;
    return e == cudaSuccess ? launch_combine(GN_F32, c, st) : e;
  }
  g.A[0] = in(f.dy); g.B[0] = weights(f.w_down); g.dgate = w.dgate; g.dup = w.dup; g.gate = in(f.gate); g.up = in(f.up); g.weight = f.weight; g.parts = w.parts;
  if (e == cudaSuccess) e = launch_group_fma(GROUP_GRAD, g, w.small, w.plan, st);
  if (f.dx.p) {
    q.A[0] = of(w.dgate); q.A[1] = of(w.dup); q.B[0] = weights(f.w_gate); q.B[1] = weights(f.w_up);
    if (e == cudaSuccess) e = launch_group_fma(GROUP_DX, q, w.small, w.plan, st);
  }
  if (any_weights(f)) {
    FmaGroup r;
    r.k = f.k;
    const auto add = [&](int M, int N, const FfnMat& left, bool left_tokens, const FfnMat& right, bool right_tokens, const gn_stack& d) {
      if (!d.p) return;
      auto& t = r.grads[r.n_grads++];
      t.M = M; t.N = N; t.left = left; t.left_tokens = left_tokens; t.right = right; t.right_tokens = right_tokens; t.d = {(float*)d.p, d.ld, d.stride};
    };
    add(f.inner, f.cols, of(w.dgate), false, in(f.x), true, f.dw_gate);
    add(f.inner, f.cols, of(w.dup), false, in(f.x), true, f.dw_up);
    add(f.cols, f.inner, in(f.dy), true, of(w.h), false, f.dw_down);
    if (e == cudaSuccess) e = launch_group_fma(GROUP_WEIGHT, r, w.small, w.plan, st);
  }
  c.d = f.dx.p; c.ld_d = f.dx.ld;
  if (f.dweight) { c.parts = w.parts; c.n_parts = fma_parts(f.inner, w.small); c.slot_of = w.plan.slot_of; c.dweight = f.dweight; }
  return e == cudaSuccess && (c.d || c.parts) ? launch_combine(GN_F32, c, st) : e;
}

// ---- FP32 on the tensor cores --------------------------------------------------------------------
struct Tensor { ExpertPlan plan; Parts x, dy, w_gate, w_up, w_down, h, dgate, dup; FfnOut out; float* parts; };
// Where its estimated time, in us, is the smaller one.  FMAs: 26 TFLOP/s of tiles that are half empty at an expert's end, or the weights' bytes (backward their gradients'
// too), and the chain of an expert's rows in its gradients.  Tensor cores: more launches, the parts of the weights (30 bytes for three), six products a term of tiles of 256 rows.
// Measured, forward and backward, tensor cores and FMAs: 16 tokens, 2 of 8 experts, 512 x 512 65, 116 and 45, 92; 500, 2 of 8, 784 x 300 65, 131 and 98, 193; 2000, 4 of 32,
// 1024 x 1024 592, 1048 and 1499, 3172; 64, 2 of 32, 1024 x 2048 893, 1202 and 394, 1557.
bool on_tensor_cores(const gn_mixture& f, bool backward) {
  const double pairs = (double)f.tokens * f.k, E = f.experts, used = pairs < E ? pairs : E, terms = (double)f.cols * f.inner * (backward ? 12 : 6);
  const double flops = (pairs + 24.0 * used) * terms / 26e6, bytes = E * f.cols * f.inner * (backward ? 36 : 12) / 2.2e6;
  const double fmas = (flops > bytes ? flops : bytes) + (backward ? 45.0 + 0.03 * pairs / E : 32.0);
  const double tensor = (backward ? 80.0 : 50.0) + E * f.cols * f.inner * 30 / 5e6 + 6 * (pairs + 128.0 * used) * terms / 0.95e9;
  return tensor < fmas;
}
int64_t lay_out_tensor(const gn_mixture& f, bool backward, char* base, Tensor& w) {
  Workspace ws{base};
  w = Tensor{};
  const int64_t pairs = f.tokens * f.k, slots = plan_slots(pairs, f.experts), lc = up8(f.cols), lf = up8(f.inner);
  w.plan = plan_at((int*)ws.take(plan_ints(pairs, f.experts, kGroupHeight) * 4), pairs, f.experts, kGroupHeight);
  const auto parts = [&](int64_t rows, int64_t ld) { return Parts{ws.take(3 * rows * ld * 2), ld, rows}; };
  if (!backward || any_weights(f)) w.x = parts(slots, lc);
  if (backward) w.dy = parts(slots, lc);
  if (!backward || f.dx.p) {
    w.w_gate = parts((int64_t)f.experts * f.inner, lc);
    w.w_up = parts((int64_t)f.experts * f.inner, lc);
  }
  w.w_down = parts((int64_t)f.experts * f.cols, lf);
  w.h = parts(slots, lf);
  if (backward) {
    w.dgate = parts(slots, lf); w.dup = parts(slots, lf);
    w.parts = (float*)ws.take(slots * tensor_parts(f.inner) * 4);
  }
  if (!backward || f.dx.p) w.out = {(float*)ws.take(pairs * lc * 4), lc};
  return ws.used;
}
cudaError_t run_tensor(const gn_mixture& f, bool backward, const Tensor& w, int* err, cudaStream_t st) {
  const auto in = [](const gn_mat& m) { return FfnMat{(const float*)m.p, m.ld}; };
  SplitMats mats[3];
  int n = 0;
  const auto split = [&](const gn_stack& m, int64_t rows, int cols, const Parts& to) {
    if (to.p) mats[n++] = {(const float*)m.p, m.ld, f.experts == 1 ? 0 : m.stride, to, rows, f.experts, cols};
  };
  split(f.w_gate, f.inner, f.cols, w.w_gate);
  split(f.w_up, f.inner, f.cols, w.w_up);
  split(f.w_down, f.cols, f.inner, w.w_down);
  cudaError_t e = launch_split_mats(mats, n, st);
  if (e == cudaSuccess) e = launch_plan(f.index, w.plan, kGroupHeight, st);
  SplitRows rows[2];
  n = 0;
  if (w.x.p) rows[n++] = {(const float*)f.x.p, f.x.ld, w.x};
  if (backward) rows[n++] = {(const float*)f.dy.p, f.dy.ld, w.dy};
  if (e == cudaSuccess) e = launch_split_to_slots(rows, n, f.tokens, f.k, f.cols, backward, w.plan, st);
  TensorGroup g, q;
  g.act = f.act; g.N = f.inner; g.K = f.cols; g.d = w.h;
  q.N = f.cols; q.K = f.inner; q.rows = w.out;
  Combine c = {};
  c.tokens = f.tokens; c.k = f.k; c.cols = f.cols; c.experts = f.experts; c.index = f.index; c.src = w.out.p; c.ld = w.out.ld;
  if (!backward) {
    g.A[0] = w.x; g.B[0] = w.w_gate; g.B[1] = w.w_up; g.gate_out = {(float*)f.gate.p, f.gate.ld}; g.up_out = {(float*)f.up.p, f.up.ld};
    if (e == cudaSuccess) e = launch_group32(GROUP_GATE, g, w.plan, err, st);
    q.A[0] = w.h; q.B[0] = w.w_down;
    if (e == cudaSuccess) e = launch_group32(GROUP_DOWN, q, w.plan, err, st);
    c.weight = f.weight; c.d = f.y.p; c.ld_d = f.y.ld;
    return e == cudaSuccess ? launch_combine(GN_F32, c, st) : e;
  }
  g.A[0] = w.dy; g.B[0] = w.w_down; g.dgate = w.dgate; g.dup = w.dup; g.gate = in(f.gate); g.up = in(f.up); g.weight = f.weight; g.parts = w.parts;
  if (e == cudaSuccess) e = launch_group32(GROUP_GRAD, g, w.plan, err, st);
  if (f.dx.p) {
    q.A[0] = w.dgate; q.A[1] = w.dup; q.B[0] = w.w_gate; q.B[1] = w.w_up;
    if (e == cudaSuccess) e = launch_group32(GROUP_DX, q, w.plan, err, st);
  }
  if (any_weights(f)) {
    TensorGroup r;
    const auto add = [&](int M, int N, const Parts& left, const Parts& right, const gn_stack& d) {
      if (!d.p) return;
      auto& t = r.grads[r.n_grads++];
      t.M = M; t.N = N; t.left = left; t.right = right; t.d = {(float*)d.p, d.ld, d.stride};
    };
    add(f.inner, f.cols, w.dgate, w.x, f.dw_gate);
    add(f.inner, f.cols, w.dup, w.x, f.dw_up);
    add(f.cols, f.inner, w.dy, w.h, f.dw_down);
    if (e == cudaSuccess) e = launch_group32(GROUP_WEIGHT, r, w.plan, err, st);
  }
  c.d = f.dx.p; c.ld_d = f.dx.ld;
  if (f.dweight) { c.parts = w.parts; c.n_parts = tensor_parts(f.inner); c.slot_of = w.plan.slot_of; c.dweight = f.dweight; }
  return e == cudaSuccess && (c.d || c.parts) ? launch_combine(GN_F32, c, st) : e;
}

cudaError_t clear(const gn_stack& m, int experts, int64_t rows, int64_t cols, int type, cudaStream_t st) {
  const size_t b = (size_t)type_bytes(type);
  cudaError_t e = cudaSuccess;
  for (int i = 0; m.p && i < experts && e == cudaSuccess; ++i)
    e = cudaMemset2DAsync((char*)m.p + i * m.stride * b, (size_t)m.ld * b, 0, (size_t)cols * b, (size_t)rows, st);
  return e;
}

struct Layouts { Half half; Single single; Tensor tensor; };
int64_t needed(const gn_mixture& f, bool backward, char* base, Layouts& w) {
  if (f.type != GN_F32) return lay_out_half(f, backward, base, w.half) + 256;
  return (on_tensor_cores(f, backward) ? lay_out_tensor(f, backward, base, w.tensor) : lay_out_single(f, backward, base, w.single)) + 256;
}

gn_status run(const gn_mixture* f, bool back, void* d_ws, int64_t ws_bytes, void* stream, char* errbuf, int64_t errbuf_len) {
  const char* why = mixture_args(f, back);
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  Layouts w;
  char* const base = (char*)(((uintptr_t)d_ws + 255) & ~(uintptr_t)255);
  if (!d_ws || ((uintptr_t)d_ws & 15) || ws_bytes < needed(*f, back, base, w))
    return op_fail(GN_EINVAL, "workspace: null, not 16-byte aligned or too small", errbuf, errbuf_len);
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  if (f->tokens == 0) {
    if (back) {
      e = clear(f->dw_gate, f->experts, f->inner, f->cols, f->type, st);
      if (e == cudaSuccess) e = clear(f->dw_up, f->experts, f->inner, f->cols, f->type, st);
      if (e == cudaSuccess) e = clear(f->dw_down, f->experts, f->cols, f->inner, f->type, st);
    }
    return op_done(e, errbuf, errbuf_len);
  }
  int* const err = ffn_error_word();
  if (!err) return op_done(cudaErrorNoDevice, errbuf, errbuf_len);
  if (f->type != GN_F32) e = run_half(*f, back, w.half, err, st);
  else if (on_tensor_cores(*f, back)) e = run_tensor(*f, back, w.tensor, err, st);
  else e = run_single(*f, back, w.single, st);
  return op_done(e, errbuf, errbuf_len);
}

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" int64_t gn_experts_workspace(const gn_mixture* args, int32_t backward) {
  Layouts w;
  return mixture_args(args, backward != 0) ? -1 : needed(*args, backward != 0, kNowhere, w);
}
extern "C" gn_status gn_experts(const gn_mixture* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return run(args, false, d_ws, ws_bytes, cuda_stream, errbuf, errbuf_len);
}
extern "C" gn_status gn_experts_grad(const gn_mixture* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return run(args, true, d_ws, ws_bytes, cuda_stream, errbuf, errbuf_len);
}
