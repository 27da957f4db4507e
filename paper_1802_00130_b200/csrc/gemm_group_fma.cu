// Products of FP32 matrices over a mixture's experts, on FMAs: four rows by eight columns of sums to a thread, chunks of 16 terms in shared memory, the next chunk's loads
// under way in registers.
//
// Tiles of 64 rows by 128 columns (GROUP_GATE: 64 hidden units, both projections of each) where they are enough for every SM, else of 32 by 64 that four groups of 64 threads
// share, each with every fourth chunk: the chain of chunks bounds a small problem (500 tokens, 2 of 8 experts, 784 x 300 backward: 222 us with the large tiles alone).  The
// groups' sums are added in order.
//
// Rows are read where they lie: a tile's rows are an expert's pairs, whose tokens' or pairs' rows are looked up once for the tile (GROUP_WEIGHT, whose terms
// they are: for each chunk).  So there are no copies in the experts' order, and no alignment is asked for.  At most 34 of the 74 TFLOP/s of FP32, reached at 8000 tokens: the
// tensor cores take over well below that.
#include "expert_kernels.h"
#include "ffn_act.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int F_KC = 16, F_THREADS = 256;
template <bool SMALL> struct FmaTile {
  static constexpr int BM = SMALL ? kFmaSmall : kFmaHeight, BN = SMALL ? 64 : 128, GROUPS = SMALL ? 4 : 1, TG = F_THREADS / GROUPS;
  static constexpr int AP = BM + 4, BP = BN + 4;                 // pitches: rows start on 16 bytes
  static constexpr int NA = BM * F_KC / 4 / TG, NB = BN * F_KC / 4 / TG;         // units of four that a thread loads for a chunk
  static constexpr int STAGE = F_KC * (AP + BP);                 // floats
  static constexpr int SMEM = GROUPS * 2 * STAGE * 4;
  static_assert((BM / 4) * (BN / 8) == TG, "four rows by eight columns to a thread");
  static_assert((GROUPS - 1) * TG * 32 <= GROUPS * 2 * STAGE, "the groups' sums fit the chunks' place");
};

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

template <int KIND, bool SMALL>
__global__ void __launch_bounds__(F_THREADS, 2) group_fma_kernel(const __grid_constant__ FmaParams p) {
  using Tile = FmaTile<SMALL>;
  constexpr bool A_MN = KIND == GROUP_WEIGHT, B_MN = KIND == GROUP_GRAD || KIND == GROUP_DX || KIND == GROUP_WEIGHT;
  constexpr int BM = Tile::BM, BN = Tile::BN, TG = Tile::TG, NA = Tile::NA, NB = Tile::NB;
  extern __shared__ __align__(16) float ring[];
  __shared__ int pairs[BM];
  grid_dep_wait();
  grid_dep_launch();
  const int* const pair_of = dep(p.pair_of);
  const int group = threadIdx.x / TG, tid = threadIdx.x % TG;
  int expert, slot, rows, n0, m0 = 0, N, K, grad = 0;
  if constexpr (KIND == GROUP_WEIGHT) {
    int i = blockIdx.x;
    while (grad + 1 < p.n_grads && i >= p.grad[grad + 1].first) ++grad;
    const FmaGrad& g = p.grad[grad];
    i -= g.first;
    const int each = g.tiles_m * g.tiles_n;
    expert = i / each; i -= expert * each;
    m0 = i / g.tiles_n * BM; n0 = i % g.tiles_n * BN;
    N = g.N; rows = g.M - m0; slot = p.start[expert]; K = p.count[expert];
  } else {
    const int t = blockIdx.x / p.tiles_n;
    if (t >= *p.n_tiles) return;
    const int4 e = *reinterpret_cast<const int4*>(p.tiles + t);
    expert = e.x; slot = e.y; rows = e.z;
    n0 = (blockIdx.x - t * p.tiles_n) * (KIND == GROUP_GATE ? BN / 2 : BN);
    N = p.N; K = p.K;
    if (threadIdx.x < BM) pairs[threadIdx.x] = threadIdx.x < rows ? pair_of[slot + threadIdx.x] : -1;
    __syncthreads();
  }
  const int chunks_each = (K + F_KC - 1) / F_KC, chunks = KIND == GROUP_DX ? 2 * chunks_each : chunks_each;
  // Unit i of a thread, x = i TG + tid: row x / 4 and four terms of a K-major operand, term x / (columns / 4) and four columns of another.
  const float *a_row[NA], *a_row2[NA];
  if constexpr (!A_MN) {
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int pair = pairs[(i * TG + tid) >> 2];
      a_row[i] = a_row2[i] = nullptr;
      if (pair >= 0) {
        a_row[i] = dep(p.A[0].p) + (int64_t)(p.token_rows ? pair / p.k : pair) * p.A[0].ld;
        if (KIND == GROUP_DX) a_row2[i] = dep(p.A[1].p) + (int64_t)pair * p.A[1].ld;
      }
    }
  }
  float4 a[NA], b[NB];
  const auto fetch = [&](int c) {
    const int part = KIND == GROUP_DX && c >= chunks_each ? 1 : 0, k0 = (part ? c - chunks_each : c) * F_KC;
    const int kc = (tid & 3) * 4;
    if constexpr (KIND == GROUP_WEIGHT) {
      const FmaGrad& g = p.grad[grad];
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        const int x = i * TG + tid, k = k0 + x / (BM / 4);
        const int pair = k < K ? pair_of[slot + k] : -1;
        a[i] = four(pair < 0 ? nullptr : dep(g.left.p) + (int64_t)(g.left_tokens ? pair / p.k : pair) * g.left.ld, m0 + x % (BM / 4) * 4, g.M, p.vec_a);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int x = i * TG + tid, k = k0 + x / (BN / 4);
        const int pair = k < K ? pair_of[slot + k] : -1;
        b[i] = four(pair < 0 ? nullptr : dep(g.right.p) + (int64_t)(g.right_tokens ? pair / p.k : pair) * g.right.ld, n0 + x % (BN / 4) * 4, N, p.vec_b);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NA; ++i) a[i] = four(part ? a_row2[i] : a_row[i], k0 + kc, K, p.vec_a);
      const Weights32& w0 = p.B[part];
      const float* const w = dep(w0.p) + expert * w0.stride;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int x = i * TG + tid;
        if constexpr (B_MN) {
          const int k = k0 + x / (BN / 4);
          b[i] = four(k < K ? w + (int64_t)k * w0.ld : nullptr, n0 + x % (BN / 4) * 4, N, p.vec_b);
        } else if constexpr (KIND == GROUP_GATE) {       // the first half of the tile's columns the gate's, the other the up projection's
          const int r = x >> 2, h = r >= BN / 2 ? 1 : 0, n = n0 + r - h * (BN / 2);
          const Weights32& wh = p.B[h];
          b[i] = four(n < N ? dep(wh.p) + expert * wh.stride + (int64_t)n * wh.ld : nullptr, k0 + kc, K, p.vec_b);
        } else {
          const int n = n0 + (x >> 2);
          b[i] = four(n < N ? w + (int64_t)n * w0.ld : nullptr, k0 + kc, K, p.vec_b);
        }
      }
    }
  };
  float* const mine = ring + group * 2 * Tile::STAGE;
  const auto stage = [&](int s) {
    float* const As = mine + s * Tile::STAGE;
    float* const Bs = As + F_KC * Tile::AP;
    const int kc = (tid & 3) * 4;
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int x = i * TG + tid;
      if constexpr (A_MN) {
        *reinterpret_cast<float4*>(As + x / (BM / 4) * Tile::AP + x % (BM / 4) * 4) = a[i];
      } else {
        float* const q = As + kc * Tile::AP + (x >> 2);
        q[0] = a[i].x; q[Tile::AP] = a[i].y; q[2 * Tile::AP] = a[i].z; q[3 * Tile::AP] = a[i].w;
      }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int x = i * TG + tid;
      if constexpr (B_MN) {
        *reinterpret_cast<float4*>(Bs + x / (BN / 4) * Tile::BP + x % (BN / 4) * 4) = b[i];
      } else {
        float* const q = Bs + kc * Tile::BP + (x >> 2);
        q[0] = b[i].x; q[Tile::BP] = b[i].y; q[2 * Tile::BP] = b[i].z; q[3 * Tile::BP] = b[i].w;
      }
    }
  };
  const auto together = [&] {
    if constexpr (Tile::GROUPS == 1) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TG) : "memory");
  };
  // sums: four rows from m, four columns from n and four half a tile further
  const int m = tid / (BN / 8) * 4, n = tid % (BN / 8) * 4;
  float v[4][8] = {};
  if (group < chunks) { fetch(group); stage(0); }
  together();
  int s = 0;
  for (int c = group; c < chunks; c += Tile::GROUPS, s ^= 1) {
    if (c + Tile::GROUPS < chunks) fetch(c + Tile::GROUPS);
    const float* const As = mine + s * Tile::STAGE + m;
    const float* const Bs = mine + s * Tile::STAGE + F_KC * Tile::AP + n;
#pragma unroll
    for (int q = 0; q < F_KC; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(As + q * Tile::AP);
      const float4 y = *reinterpret_cast<const float4*>(Bs + q * Tile::BP), z = *reinterpret_cast<const float4*>(Bs + q * Tile::BP + BN / 2);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf(xs[i], ys[j], v[i][j]);
    }
    if (c + Tile::GROUPS < chunks) stage(s ^ 1);
    together();
  }
  if constexpr (Tile::GROUPS > 1) {
    __syncthreads();                 // (the chunks' place is free)
    float4* const sums = reinterpret_cast<float4*>(ring);
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[((group - 1) * 8 + i) * TG + tid] = make_float4(v[i / 2][i % 2 * 4], v[i / 2][i % 2 * 4 + 1], v[i / 2][i % 2 * 4 + 2], v[i / 2][i % 2 * 4 + 3]);
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 0; g < Tile::GROUPS - 1; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 x = sums[(g * 8 + i) * TG + tid];
        float* const q = &v[i / 2][i % 2 * 4];
        q[0] += x.x; q[1] += x.y; q[2] += x.z; q[3] += x.w;
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (KIND == GROUP_WEIGHT) {
      const FmaGrad& g = p.grad[grad];
      if (m + i >= rows) continue;
      float* const row = g.d.p + expert * g.d.stride + (int64_t)(m0 + m + i) * g.d.ld;
      put_four(row, n0 + n, N, g.vec, v[i]);
      put_four(row, n0 + BN / 2 + n, N, g.vec, v[i] + 4);
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
            const int col = n0 + BN / 2 * h2 + n;
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
        for (int o = BN / 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);       // (BN / 8 neighbouring threads share a row)
        if (pair >= 0 && tid % (BN / 8) == 0) p.parts[(int64_t)(slot + m + i) * p.n_parts + n0 / BN] = sum;
      } else {
        if (pair < 0) continue;
        put_four(p.d.p + pair * p.d.ld, n0 + n, N, p.vec, v[i]);
        put_four(p.d.p + pair * p.d.ld, n0 + BN / 2 + n, N, p.vec, v[i] + 4);
      }
    }
  }
}

bool vec4(const void* p, int64_t ld, int64_t stride = 0) { return !p || (((uintptr_t)p & 15) == 0 && ld % 4 == 0 && stride % 4 == 0); }

template <int KIND, bool SMALL>
cudaError_t launch_fma_as(const FmaGroup& g, const ExpertPlan& plan, cudaStream_t st) {
  using Tile = FmaTile<SMALL>;
  FmaParams p = {};
  p.act = g.act; p.k = g.k; p.tiles = plan.tiles; p.n_tiles = plan.n_tiles; p.start = plan.start; p.count = plan.count; p.pair_of = plan.pair_of;
  long long blocks;
  if constexpr (KIND == GROUP_WEIGHT) {
    blocks = 0;
    p.n_grads = g.n_grads; p.vec_a = p.vec_b = 1;
    for (int i = 0; i < g.n_grads; ++i) {
      const auto& q = g.grads[i];
      FmaGrad& to = p.grad[i];
      to.M = q.M; to.N = q.N; to.tiles_m = (q.M + Tile::BM - 1) / Tile::BM; to.tiles_n = (q.N + Tile::BN - 1) / Tile::BN; to.first = (int)blocks;
      to.left = q.left; to.right = q.right; to.left_tokens = q.left_tokens; to.right_tokens = q.right_tokens; to.d = q.d;
      to.vec = vec4(q.d.p, q.d.ld, q.d.stride);
      p.vec_a = p.vec_a && vec4(q.left.p, q.left.ld); p.vec_b = p.vec_b && vec4(q.right.p, q.right.ld);
      blocks += (long long)plan.experts * to.tiles_m * to.tiles_n;
      if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    }
  } else {
    constexpr int WIDTH = KIND == GROUP_GATE ? Tile::BN / 2 : Tile::BN;
    p.N = g.N; p.K = g.K; p.tiles_n = (g.N + WIDTH - 1) / WIDTH; p.token_rows = g.token_rows;
    for (int s = 0; s < 2; ++s) { p.A[s] = g.A[s]; p.B[s] = g.B[s]; }
    p.vec_a = vec4(g.A[0].p, g.A[0].ld) && vec4(g.A[1].p, g.A[1].ld);
    p.vec_b = vec4(g.B[0].p, g.B[0].ld, g.B[0].stride) && vec4(g.B[1].p, g.B[1].ld, g.B[1].stride);
    p.d = g.d; p.dgate = g.dgate; p.dup = g.dup; p.gate_out = g.gate_out; p.up_out = g.up_out; p.gate = g.gate; p.up = g.up;
    p.vec = vec4(p.d.p, p.d.ld) && vec4(p.dgate.p, p.dgate.ld) && vec4(p.dup.p, p.dup.ld) && vec4(p.gate_out.p, p.gate_out.ld) && vec4(p.up_out.p, p.up_out.ld) &&
            vec4(p.gate.p, p.gate.ld) && vec4(p.up.p, p.up.ld);
    p.weight = g.weight; p.parts = g.parts; p.n_parts = fma_parts(g.N, SMALL);
    blocks = plan_tiles(plan.pairs, plan.experts, Tile::BM) * p.tiles_n;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  }
  static std::atomic<signed char> ready[64];
  auto* const kernel = group_fma_kernel<KIND, SMALL>;
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Tile::SMEM) == cudaSuccess; })) return cudaErrorInvalidDevice;
  return launch_pdl(kernel, (int)blocks, F_THREADS, Tile::SMEM, st, p);
}
template <bool SMALL>
cudaError_t launch_fma_of(GroupKind kind, const FmaGroup& g, const ExpertPlan& plan, cudaStream_t st) {
  switch (kind) {
    case GROUP_GATE: return launch_fma_as<GROUP_GATE, SMALL>(g, plan, st);
    case GROUP_DOWN: return launch_fma_as<GROUP_DOWN, SMALL>(g, plan, st);
    case GROUP_GRAD: return launch_fma_as<GROUP_GRAD, SMALL>(g, plan, st);
    case GROUP_DX: return launch_fma_as<GROUP_DX, SMALL>(g, plan, st);
    default: return launch_fma_as<GROUP_WEIGHT, SMALL>(g, plan, st);
  }
}

}  // namespace

int fma_parts(int N, bool small) { return small ? (N + FmaTile<true>::BN - 1) / FmaTile<true>::BN : (N + FmaTile<false>::BN - 1) / FmaTile<false>::BN; }

// The large tiles where those of the product with the fewest columns are two to an SM.
bool fma_small(int64_t pairs, int experts, int cols, int inner) {
  const int64_t rows = pairs / kFmaHeight + (pairs < experts ? pairs : (int64_t)experts) / 2;
  return rows * (((cols < inner ? cols : inner) + 127) / 128) < 2LL * num_sms();
}

cudaError_t launch_group_fma(GroupKind kind, const FmaGroup& g, bool small, const ExpertPlan& plan, cudaStream_t st) {
  return small ? launch_fma_of<true>(kind, g, plan, st) : launch_fma_of<false>(kind, g, plan, st);
}

}  // namespace gn
