// Products of FP32 matrices over a mixture's experts, on FMAs: tiles of 64 rows by 128 columns (GROUP_GATE: 64 hidden units, both projections of each), four rows by
// eight columns of sums to a thread, chunks of 16 terms in shared memory, the next chunk's loads under way in registers.
//
// Rows are read where they lie: a tile's rows are an expert's pairs, whose tokens' or pairs' rows are looked up once for the tile (GROUP_WEIGHT, whose terms
// they are: for each chunk).  So there are no copies in the experts' order, and no alignment is asked for.  Sums are in the order of the terms.
#include "expert_kernels.h"
#include "ffn_act.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int F_BM = kFmaHeight, F_BN = 128, F_KC = 16, F_THREADS = 256, F_A_PITCH = F_BM + 4, F_B_PITCH = F_BN + 4;
static_assert(F_A_PITCH % 4 == 0 && F_B_PITCH % 4 == 0, "rows start on 16 bytes");

struct FmaGrad { int M, N, tiles_m, tiles_n, first, left_tokens, right_tokens, vec; FfnMat left, right; Grads32 d; };
struct FmaParams {
  int N, K, tiles_n, act, k, token_rows, vec_a, vec_b, vec;
  const ExpertTile* tiles; const int* n_tiles;
  const int *start, *count, *pair_of;
  FfnMat A[2]; Weights32 B[2];
  FfnOut d, dgate, dup, gate_out, up_out;
  FfnMat gate, up;
  const float* weight; float* parts; int n_parts;
  FmaGrad grad[3]; int n_grads;
};

// Four neighbouring elements from column c on of a row of n; zeros past its end, or without a row.
__device__ __forceinline__ float4 four(const float* row, int c, int n, bool vec) {
  if (!row || c >= n) return make_float4(0.f, 0.f, 0.f, 0.f);
  if (vec && c + 4 <= n) return *reinterpret_cast<const float4*>(row + c);
  float4 v = make_float4(row[c], 0.f, 0.f, 0.f);
  if (c + 1 < n) v.y = row[c + 1];
  if (c + 2 < n) v.z = row[c + 2];
  if (c + 3 < n) v.w = row[c + 3];
  return v;
}
__device__ __forceinline__ void put_four(float* row, int c, int n, bool vec, const float* v) {
  if (vec && c + 4 <= n) {
    *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < n) row[c + e] = v[e];
  }
}

template <int KIND>
__global__ void __launch_bounds__(F_THREADS, 2) group_fma_kernel(const __grid_constant__ FmaParams p) {
  constexpr bool A_MN = KIND == GROUP_WEIGHT, B_MN = KIND == GROUP_GRAD || KIND == GROUP_DX || KIND == GROUP_WEIGHT;
  __shared__ __align__(16) float As[2][F_KC][F_A_PITCH], Bs[2][F_KC][F_B_PITCH];
  __shared__ int pairs[F_BM];
  grid_dep_wait();
  grid_dep_launch();
  const int* const pair_of = dep(p.pair_of);
  const int tid = threadIdx.x;
  int expert, slot, rows, n0, m0 = 0, N, K, grad = 0;
  if constexpr (KIND == GROUP_WEIGHT) {
    int i = blockIdx.x;
    while (grad + 1 < p.n_grads && i >= p.grad[grad + 1].first) ++grad;
    const FmaGrad& g = p.grad[grad];
    i -= g.first;
    const int each = g.tiles_m * g.tiles_n;
    expert = i / each; i -= expert * each;
    m0 = i / g.tiles_n * F_BM; n0 = i % g.tiles_n * F_BN;
    N = g.N; rows = g.M - m0; slot = p.start[expert]; K = p.count[expert];
  } else {
    const int t = blockIdx.x / p.tiles_n;
    if (t >= *p.n_tiles) return;
    const int4 e = *reinterpret_cast<const int4*>(p.tiles + t);
    expert = e.x; slot = e.y; rows = e.z;
    n0 = (blockIdx.x - t * p.tiles_n) * (KIND == GROUP_GATE ? F_BN / 2 : F_BN);
    N = p.N; K = p.K;
    if (tid < F_BM) pairs[tid] = tid < rows ? pair_of[slot + tid] : -1;
    __syncthreads();
  }
  const int chunks_each = (K + F_KC - 1) / F_KC, chunks = KIND == GROUP_DX ? 2 * chunks_each : chunks_each;
  // K-major operands: thread = row tid / 4 (and 64 further), four terms; others: term tid / 16, four columns (and 64 further).
  const int kr = tid >> 2, kc = (tid & 3) * 4, mr = tid >> 4, mc = (tid & 15) * 4;
  const float *a_row = nullptr, *a_row2 = nullptr;
  if constexpr (!A_MN) {
    const int pair = pairs[kr];
    if (pair >= 0) {
      a_row = dep(p.A[0].p) + (int64_t)(p.token_rows ? pair / p.k : pair) * p.A[0].ld;
      if (KIND == GROUP_DX) a_row2 = dep(p.A[1].p) + (int64_t)pair * p.A[1].ld;
    }
  }
  float4 a, b[2];
  const auto fetch = [&](int c) {
    const int part = KIND == GROUP_DX && c >= chunks_each ? 1 : 0, k0 = (part ? c - chunks_each : c) * F_KC;
    if constexpr (KIND == GROUP_WEIGHT) {
      const FmaGrad& g = p.grad[grad];
      const int pair = k0 + mr < K ? pair_of[slot + k0 + mr] : -1;
      const float* const left = pair < 0 ? nullptr : dep(g.left.p) + (int64_t)(g.left_tokens ? pair / p.k : pair) * g.left.ld;
      const float* const right = pair < 0 ? nullptr : dep(g.right.p) + (int64_t)(g.right_tokens ? pair / p.k : pair) * g.right.ld;
      a = four(left, m0 + mc, g.M, p.vec_a);
      b[0] = four(right, n0 + mc, N, p.vec_b);
      b[1] = four(right, n0 + 64 + mc, N, p.vec_b);
    } else {
      a = four(part ? a_row2 : a_row, k0 + kc, K, p.vec_a);
      const Weights32& w0 = p.B[part];
      const float* const w = dep(w0.p) + expert * w0.stride;
      if constexpr (B_MN) {
        const float* const row = k0 + mr < K ? w + (int64_t)(k0 + mr) * w0.ld : nullptr;
        b[0] = four(row, n0 + mc, N, p.vec_b);
        b[1] = four(row, n0 + 64 + mc, N, p.vec_b);
      } else if constexpr (KIND == GROUP_GATE) {
        const bool in = n0 + kr < N;
        b[0] = four(in ? w + (int64_t)(n0 + kr) * w0.ld : nullptr, k0 + kc, K, p.vec_b);
        b[1] = four(in ? dep(p.B[1].p) + expert * p.B[1].stride + (int64_t)(n0 + kr) * p.B[1].ld : nullptr, k0 + kc, K, p.vec_b);
      } else {
        b[0] = four(n0 + kr < N ? w + (int64_t)(n0 + kr) * w0.ld : nullptr, k0 + kc, K, p.vec_b);
        b[1] = four(n0 + 64 + kr < N ? w + (int64_t)(n0 + 64 + kr) * w0.ld : nullptr, k0 + kc, K, p.vec_b);
      }
    }
  };
  const auto stage = [&](int s) {
    if constexpr (A_MN) {
      *reinterpret_cast<float4*>(&As[s][mr][mc]) = a;
    } else {
      As[s][kc][kr] = a.x; As[s][kc + 1][kr] = a.y; As[s][kc + 2][kr] = a.z; As[s][kc + 3][kr] = a.w;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (B_MN) {
        *reinterpret_cast<float4*>(&Bs[s][mr][64 * h + mc]) = b[h];
      } else {
        Bs[s][kc][64 * h + kr] = b[h].x; Bs[s][kc + 1][64 * h + kr] = b[h].y; Bs[s][kc + 2][64 * h + kr] = b[h].z; Bs[s][kc + 3][64 * h + kr] = b[h].w;
      }
    }
  };
  // sums: rows 4 (tid / 16) .., columns 4 (tid % 16) .. and 64 further
  const int m = (tid >> 4) * 4, n = (tid & 15) * 4;
  float v[4][8] = {};
  if (chunks > 0) { fetch(0); stage(0); }
  __syncthreads();
  for (int c = 0; c < chunks; ++c) {
    const int s = c & 1;
    if (c + 1 < chunks) fetch(c + 1);
#pragma unroll
    for (int q = 0; q < F_KC; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(&As[s][q][m]);
      const float4 y = *reinterpret_cast<const float4*>(&Bs[s][q][n]), z = *reinterpret_cast<const float4*>(&Bs[s][q][64 + n]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf(xs[i], ys[j], v[i][j]);
    }
    if (c + 1 < chunks) stage(s ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (KIND == GROUP_WEIGHT) {
      const FmaGrad& g = p.grad[grad];
      if (m + i >= rows) continue;
      float* const row = g.d.p + expert * g.d.stride + (int64_t)(m0 + m + i) * g.d.ld;
      put_four(row, n0 + n, N, g.vec, v[i]);
      put_four(row, n0 + 64 + n, N, g.vec, v[i] + 4);
    } else {
      const int pair = m + i < rows ? pairs[m + i] : -1;
      if constexpr (KIND == GROUP_GATE) {
        if (pair < 0) continue;
        float h[4];
        with_activation(p.act, [&](auto act) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float f, unused;
            activation<decltype(act)::value, false>(v[i][e], f, unused);
            h[e] = f * v[i][4 + e];
          }
        });
        put_four(p.d.p + pair * p.d.ld, n0 + n, N, p.vec, h);
        if (p.gate_out.p) put_four(p.gate_out.p + pair * p.gate_out.ld, n0 + n, N, p.vec, v[i]);
        if (p.up_out.p) put_four(p.up_out.p + pair * p.up_out.ld, n0 + n, N, p.vec, v[i] + 4);
      } else if constexpr (KIND == GROUP_GRAD) {
        float sum = 0.f;
        if (pair >= 0) {
          const float share = dep(p.weight)[pair];
          const float* const gate = dep(p.gate.p) + pair * p.gate.ld;
          const float* const up = dep(p.up.p) + pair * p.up.ld;
#pragma unroll
          for (int h2 = 0; h2 < 2; ++h2) {
            const int col = n0 + 64 * h2 + n;
            const float4 g4 = four(gate, col, N, p.vec), u4 = four(up, col, N, p.vec);
            const float gs[4] = {g4.x, g4.y, g4.z, g4.w}, us[4] = {u4.x, u4.y, u4.z, u4.w};
            float h[4], dg[4], du[4];
            with_activation(p.act, [&](auto act) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float q = v[i][4 * h2 + e];
                float f, df;
                activation<decltype(act)::value, false>(gs[e], f, df);
                const float plain = f * us[e];
                if (col + e < N) sum = fmaf(q, plain, sum);
                h[e] = share * plain; dg[e] = share * q * us[e] * df; du[e] = share * q * f;
              }
            });
            put_four(p.d.p + pair * p.d.ld, col, N, p.vec, h);
            put_four(p.dgate.p + pair * p.dgate.ld, col, N, p.vec, dg);
            put_four(p.dup.p + pair * p.dup.ld, col, N, p.vec, du);
          }
        }
#pragma unroll
        for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);       // (16 neighbouring threads share a row)
        if (pair >= 0 && (tid & 15) == 0) p.parts[(int64_t)(slot + m + i) * p.n_parts + n0 / F_BN] = sum;
      } else {
        if (pair < 0) continue;
        put_four(p.d.p + pair * p.d.ld, n0 + n, N, p.vec, v[i]);
        put_four(p.d.p + pair * p.d.ld, n0 + 64 + n, N, p.vec, v[i] + 4);
      }
    }
  }
}

bool vec4(const void* p, int64_t ld, int64_t stride = 0) { return !p || (((uintptr_t)p & 15) == 0 && ld % 4 == 0 && stride % 4 == 0); }

template <int KIND>
cudaError_t launch_fma_as(const FmaGroup& g, const ExpertPlan& plan, cudaStream_t st) {
  FmaParams p = {};
  p.act = g.act; p.k = g.k; p.tiles = plan.tiles; p.n_tiles = plan.n_tiles; p.start = plan.start; p.count = plan.count; p.pair_of = plan.pair_of;
  long long blocks;
  if constexpr (KIND == GROUP_WEIGHT) {
    blocks = 0;
    p.n_grads = g.n_grads; p.vec_a = p.vec_b = 1;
    for (int i = 0; i < g.n_grads; ++i) {
      const auto& q = g.grads[i];
      FmaGrad& to = p.grad[i];
      to.M = q.M; to.N = q.N; to.tiles_m = (q.M + F_BM - 1) / F_BM; to.tiles_n = (q.N + F_BN - 1) / F_BN; to.first = (int)blocks;
      to.left = q.left; to.right = q.right; to.left_tokens = q.left_tokens; to.right_tokens = q.right_tokens; to.d = q.d;
      to.vec = vec4(q.d.p, q.d.ld, q.d.stride);
      p.vec_a = p.vec_a && vec4(q.left.p, q.left.ld); p.vec_b = p.vec_b && vec4(q.right.p, q.right.ld);
      blocks += (long long)plan.experts * to.tiles_m * to.tiles_n;
      if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    }
  } else {
    constexpr int WIDTH = KIND == GROUP_GATE ? F_BN / 2 : F_BN;
    p.N = g.N; p.K = g.K; p.tiles_n = (g.N + WIDTH - 1) / WIDTH; p.token_rows = g.token_rows;
    for (int s = 0; s < 2; ++s) { p.A[s] = g.A[s]; p.B[s] = g.B[s]; }
    p.vec_a = vec4(g.A[0].p, g.A[0].ld) && vec4(g.A[1].p, g.A[1].ld);
    p.vec_b = vec4(g.B[0].p, g.B[0].ld, g.B[0].stride) && vec4(g.B[1].p, g.B[1].ld, g.B[1].stride);
    p.d = g.d; p.dgate = g.dgate; p.dup = g.dup; p.gate_out = g.gate_out; p.up_out = g.up_out; p.gate = g.gate; p.up = g.up;
    p.vec = vec4(p.d.p, p.d.ld) && vec4(p.dgate.p, p.dgate.ld) && vec4(p.dup.p, p.dup.ld) && vec4(p.gate_out.p, p.gate_out.ld) && vec4(p.up_out.p, p.up_out.ld) &&
            vec4(p.gate.p, p.gate.ld) && vec4(p.up.p, p.up.ld);
    p.weight = g.weight; p.parts = g.parts; p.n_parts = fma_parts(g.N);
    blocks = plan_tiles(plan.pairs, plan.experts, kFmaHeight) * p.tiles_n;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  }
  return launch_pdl(group_fma_kernel<KIND>, (int)blocks, F_THREADS, 0, st, p);
}

}  // namespace

int fma_parts(int N) { return (N + F_BN - 1) / F_BN; }

cudaError_t launch_group_fma(GroupKind kind, const FmaGroup& g, const ExpertPlan& plan, cudaStream_t st) {
  switch (kind) {
    case GROUP_GATE: return launch_fma_as<GROUP_GATE>(g, plan, st);
    case GROUP_DOWN: return launch_fma_as<GROUP_DOWN>(g, plan, st);
    case GROUP_GRAD: return launch_fma_as<GROUP_GRAD>(g, plan, st);
    case GROUP_DX: return launch_fma_as<GROUP_DX>(g, plan, st);
    default: return launch_fma_as<GROUP_WEIGHT>(g, plan, st);
  }
}

}  // namespace gn
