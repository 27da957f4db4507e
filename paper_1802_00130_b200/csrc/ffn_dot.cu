// Products of the gated feed-forward block's forward pass in FP32 with few tokens, on FMAs.
//
// One token is bound by reading the weights once (two FP16 parts of them would be written and read again): 3584 x 15232 133 us, 4.9 TB/s, 2048 x 4096 33; up to four
// 188 and 38.  With five to eight the loads of the tokens' values from L1, twice the weights' bytes at four rows a warp, take longer (370 and 56; the
// weights ahead in shared memory did not help: 377 and 60).  More tokens go eight to a block; what it saves there is launches.
// A warp takes R rows of the weights at a time and walks K with 16
// bytes a lane from each (single elements, as many to a step, where rows are not 16-byte aligned), the tokens' values from L1, all of a step's loads
// before its first product.  Each lane's sums are added across the warp at the end.
#include "ffn_act.cuh"
#include "ffn_kernels.h"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int D_WARPS = 4;
struct DotParams {
  int tokens, features, K, act;
  const void *x, *w[2]; int64_t ldx, ldw[2];
  void *d[3]; int64_t ldd[3];
};

// GATE: R / 2 hidden units, a row of either weight matrix each.
template <bool GATE, int R, int TOK, bool VEC>
__global__ void __launch_bounds__(32 * D_WARPS) ffn_dot_kernel(const __grid_constant__ DotParams p) {
  constexpr int V = Pack<float>::V, F = GATE ? R / 2 : R;            // F: features of a warp
  const int lane = threadIdx.x & 31, f0 = (blockIdx.x * D_WARPS + (threadIdx.x >> 5)) * F;
  grid_dep_wait();
  grid_dep_launch();
  if (f0 >= p.features) return;
  const int t0 = blockIdx.y * TOK, tokens = min(TOK, p.tokens - t0);
  const float* const x = (const float*)dep(p.x) + t0 * p.ldx;
  const float* row[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int f = min(f0 + (GATE ? r / 2 : r), p.features - 1), m = GATE ? r % 2 : 0;
    row[r] = (const float*)dep(p.w[m]) + f * p.ldw[m];
  }
  float s[R][TOK];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < TOK; ++t) s[r][t] = 0.f;
  const int steps = (p.K + 32 * V - 1) / (32 * V);
#pragma unroll 2
  for (int k = 0; k < steps; ++k) {
    // (a warp's 32 units of this step as a row of their own: `left` elements of them exist, the others read as zero on both sides)
    const int at = k * 32 * V, left = p.K - at;
    Pack<float> w[R], v[TOK];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = load_pack<VEC>(row[r] + at, 0, lane, 32, left);
#pragma unroll
    for (int t = 0; t < TOK; ++t) v[t] = load_pack<VEC>(x + min(t, tokens - 1) * p.ldx + at, 0, lane, 32, left);
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
      for (int e = 0; e < V; ++e)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][t] = fmaf(w[r].get(e), v[t].get(e), s[r][t]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
      for (int o = 16; o; o >>= 1) s[r][t] += __shfl_xor_sync(0xffffffffu, s[r][t], o);
  // lane t finishes token t
  with_activation(p.act, [&](auto act) {
#pragma unroll
    for (int f = 0; f < F; ++f) {
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int t = 0; t < TOK; ++t)
        if (lane == t) { a = s[GATE ? 2 * f : f][t]; b = GATE ? s[2 * f + (GATE ? 1 : 0)][t] : 0.f; }
      if (lane >= tokens || f0 + f >= p.features) continue;
      const auto put = [&](int k, float v) { ((float*)p.d[k])[(t0 + lane) * p.ldd[k] + f0 + f] = v; };
      if (GATE) {
        float h, unused;
        activation<decltype(act)::value, false>(a, h, unused);
        put(0, h * b);
        if (p.d[1]) put(1, a);
        if (p.d[2]) put(2, b);
      } else {
        put(0, a);
      }
    }
  });
}

template <bool GATE, int R, int TOK>
cudaError_t launch_dot_as(const DotParams& p, bool vec, cudaStream_t st) {
  const int each = D_WARPS * (GATE ? R / 2 : R);
  return launch_pdl_grid(vec ? ffn_dot_kernel<GATE, R, TOK, true> : ffn_dot_kernel<GATE, R, TOK, false>,
                         dim3((unsigned)((p.features + each - 1) / each), (unsigned)((p.tokens + TOK - 1) / TOK)), 32 * D_WARPS, 0, st, p);
}
template <bool GATE>
cudaError_t launch_dot(const DotParams& p, cudaStream_t st) {
  const bool vec = wide_ok(p.x, p.ldx, GN_F32) && wide_ok(p.w[0], p.ldw[0], GN_F32) && (!GATE || wide_ok(p.w[1], p.ldw[1], GN_F32));
  // (four rows of the weights a warp share the tokens' loads, where that leaves every SM eight warps)
  constexpr int FEW = GATE ? 2 : 1;
  const bool few = (int64_t)p.features * FEW * ((p.tokens + 7) / 8) < 4LL * 8 * num_sms();
  const auto launch = [&](auto tok) {
    constexpr int TOK = decltype(tok)::value;
    return few ? launch_dot_as<GATE, FEW, TOK>(p, vec, st) : launch_dot_as<GATE, 4, TOK>(p, vec, st);
  };
  return p.tokens == 1 ? launch(ActIs<1>{}) : p.tokens <= 4 ? launch(ActIs<4>{}) : launch(ActIs<8>{});
}

}  // namespace

cudaError_t launch_ffn_dot(const FfnDot& g, cudaStream_t st) {
  DotParams p = {};
  p.tokens = g.tokens; p.features = g.features; p.K = g.K; p.act = g.act;
  p.x = g.x.p; p.ldx = g.x.ld;
  for (int k = 0; k < 2; ++k) { p.w[k] = g.w[k].p; p.ldw[k] = g.w[k].ld; }
  for (int k = 0; k < 3; ++k) { p.d[k] = g.d[k].p; p.ldd[k] = g.d[k].ld; }
  return g.w[1].p ? launch_dot<true>(p, st) : launch_dot<false>(p, st);
}

}  // namespace gn
