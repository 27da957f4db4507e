// The backward pass of the gated feed-forward block in FP32 where it is small: two launches on FMAs, where the products at FP32 accuracy take nine.
//
// The first computes dh = dy Wd and, in its epilogue, h, dgate and dup; the second all of dx = dgate Wg + dup Wu and the weights' gradients.  A block has a tile of
// 32 x 32 sums, two rows by four columns of them to a thread of each of four groups, which take the chunks of K in turn (the chain of chunks bounds a small problem:
// 1000 tokens, 64 columns, 128 hidden units took 46 us with one group, 21 with four) and whose sums are added in order at the end.  cp.async brings the chunks, two ahead, element by element
// (any alignment, zeros past an edge).
#include <atomic>

#include "ffn_act.cuh"
#include "ffn_kernels.h"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int S_T = 32, S_KC = 32, S_STAGES = 3, S_GROUPS = 4, S_GROUP = 128, S_THREADS = S_GROUPS * S_GROUP, S_A_PITCH = S_T + 2;
struct SmallStage { float a[S_KC][S_A_PITCH], b[S_KC][S_T]; };
constexpr int S_SMEM = S_GROUPS * S_STAGES * (int)sizeof(SmallStage);
static_assert(sizeof(SmallStage) % 16 == 0 && S_KC * S_A_PITCH % 4 == 0, "rows of b start on 16 bytes");
struct SmallProblem { int M, N, K[2], a_mn, vec, tiles_n, tiles; FfnMat A[2], B[2]; FfnOut d; };
struct SmallParams {
  SmallProblem p[kFfnGroup];
  int n, act;
  FfnMat gate, up;                   // GRAD: as stored; its results go to out (h, dgate, dup) instead of p[0].d
  FfnOut out[3];
};

__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void put4(const FfnOut& d, int m, int n, int N, bool vec, const float (&v)[4]) {
  float* const q = d.p + m * d.ld + n;
  if (vec && n + 4 <= N) {
    *reinterpret_cast<float4*>(q) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) q[e] = v[e];
  }
}

template <bool GRAD>
__global__ void __launch_bounds__(S_THREADS) ffn_small_kernel(const __grid_constant__ SmallParams g) {
  extern __shared__ __align__(16) SmallStage ring[];       // [S_GROUPS][S_STAGES]
  grid_dep_wait();
  grid_dep_launch();
  int t = blockIdx.x, k = 0;
  while (k + 1 < g.n && t >= g.p[k].tiles) t -= g.p[k++].tiles;
  const SmallProblem& p = g.p[k];
  const int m0 = t / p.tiles_n * S_T, n0 = t % p.tiles_n * S_T;
  const int group = threadIdx.x / S_GROUP, thread = threadIdx.x % S_GROUP, lane = thread & 31, row0 = (thread >> 5) * (S_KC / 4);
  const int chunks0 = (p.K[0] + S_KC - 1) / S_KC, chunks = chunks0 + (p.K[1] + S_KC - 1) / S_KC;
  SmallStage* const mine = ring + group * S_STAGES;
  const auto request = [&](int c, int stage) {
    if (c < chunks) {
      const int s = c >= chunks0 ? 1 : 0, k0 = (s ? c - chunks0 : c) * S_KC, K = p.K[s];
      const float* const a = dep(p.A[s].p);
      const float* const b = dep(p.B[s].p);
      const int64_t lda = p.A[s].ld, ldb = p.B[s].ld;
      // row i of this thread's eight: k0 + row0 + i of B, and of A where it is stored as B is; else m0 + row0 + i of A
      const float* pb = b + (k0 + row0) * ldb + n0 + lane;
      const float* pa = a + ((p.a_mn ? k0 : m0) + row0) * lda + (p.a_mn ? m0 : k0) + lane;
      const int rows_b = n0 + lane < p.N ? K - k0 - row0 : 0;
      const int rows_a = p.a_mn ? (m0 + lane < p.M ? K - k0 - row0 : 0) : (k0 + lane < K ? p.M - m0 - row0 : 0);
      const uint32_t to_b = smem_u32(&mine[stage].b[row0][lane]);
      const uint32_t to_a = smem_u32(p.a_mn ? &mine[stage].a[row0][lane] : &mine[stage].a[lane][row0]), step_a = p.a_mn ? S_A_PITCH * 4 : 4;
#pragma unroll
      for (int i = 0; i < S_KC / 4; ++i) {
        cp_async4(to_b + i * S_T * 4, i < rows_b ? pb : b, i < rows_b);
        cp_async4(to_a + i * step_a, i < rows_a ? pa : a, i < rows_a);
        pb += ldb; pa += lda;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int c = 0; c < S_STAGES - 1; ++c) request(group + c * S_GROUPS, c);
  const int n = (thread & 7) * 4, m = (thread >> 3) * 2;
  float v[2][4] = {};
  int stage = 0;
  for (int c = group; c < chunks; c += S_GROUPS) {
    asm volatile("cp.async.wait_group %0;" ::"n"(S_STAGES - 2) : "memory");
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(S_GROUP) : "memory");     // the chunk is there for the group, and nobody reads the one before it any more
    request(c + (S_STAGES - 1) * S_GROUPS, stage == 0 ? S_STAGES - 1 : stage - 1);
#pragma unroll
    for (int q = 0; q < S_KC; ++q) {
      const float2 a = *reinterpret_cast<const float2*>(&mine[stage].a[q][m]);
      const float4 b = *reinterpret_cast<const float4*>(&mine[stage].b[q][n]);
      v[0][0] = fmaf(a.x, b.x, v[0][0]); v[0][1] = fmaf(a.x, b.y, v[0][1]); v[0][2] = fmaf(a.x, b.z, v[0][2]); v[0][3] = fmaf(a.x, b.w, v[0][3]);
      v[1][0] = fmaf(a.y, b.x, v[1][0]); v[1][1] = fmaf(a.y, b.y, v[1][1]); v[1][2] = fmaf(a.y, b.z, v[1][2]); v[1][3] = fmaf(a.y, b.w, v[1][3]);
    }
    if (++stage == S_STAGES) stage = 0;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();                   // (the ring is free)
  float4* const sums = reinterpret_cast<float4*>(ring);
  if (group > 0) {
#pragma unroll
    for (int r = 0; r < 2; ++r) sums[((group - 1) * 2 + r) * S_GROUP + thread] = make_float4(v[r][0], v[r][1], v[r][2], v[r][3]);
  }
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int q = 0; q < S_GROUPS - 1; ++q)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float4 x = sums[(q * 2 + r) * S_GROUP + thread];
      v[r][0] += x.x; v[r][1] += x.y; v[r][2] += x.z; v[r][3] += x.w;
    }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = m0 + m + r, col = n0 + n;
    if (row >= p.M || col >= p.N) continue;
    if constexpr (!GRAD) {
      put4(p.d, row, col, p.N, p.vec, v[r]);
    } else {
      const float* const gate = dep(g.gate.p) + row * g.gate.ld + col;
      const float* const up = dep(g.up.p) + row * g.up.ld + col;
      float gt[4], u[4], h[4], dg[4], du[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) { const bool in = col + e < p.N; gt[e] = in ? gate[e] : 0.f; u[e] = in ? up[e] : 0.f; }
      with_activation(g.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float a, da;
          activation<decltype(act)::value, false>(gt[e], a, da);
          h[e] = a * u[e]; dg[e] = v[r][e] * u[e] * da; du[e] = v[r][e] * a;
        }
      });
      put4(g.out[0], row, col, p.N, p.vec, h);
      put4(g.out[1], row, col, p.N, p.vec, dg);
      put4(g.out[2], row, col, p.N, p.vec, du);
    }
  }
}

bool vec4(const FfnOut& d) { return ((uintptr_t)d.p & 15) == 0 && d.ld % 4 == 0; }
long long tiles_of(const FfnSmall& g) { return (long long)((g.M + S_T - 1) / S_T) * ((g.N + S_T - 1) / S_T); }
int chunks_of(const FfnSmall& g) { return (g.K[0] + S_KC - 1) / S_KC + (g.K[1] + S_KC - 1) / S_KC; }

}  // namespace

// 2.5 us a launch, its longest chain of chunks at 1.5 for four of them, and all tiles' shares of an SM, 0.9 each and 0.45 a chunk: measured at 1 to 4000 tokens, 16 to
// 2048 columns and 16 to 4096 hidden units, from a third below to a third above.
double ffn_small_us(const FfnSmall* g, int n) {
  double work = 0.0;
  int longest = 0;
  for (int i = 0; i < n; ++i) {
    const int c = chunks_of(g[i]);
    longest = c > longest ? c : longest;
    work += (double)tiles_of(g[i]) * (0.9 + 0.45 * c);
  }
  return 2.5 + 1.5 * ((longest + S_GROUPS - 1) / S_GROUPS) + work / num_sms();
}

cudaError_t launch_ffn_small(const FfnSmall* g, int n, const FfnSmallGrad* grad, cudaStream_t st) {
  static std::atomic<signed char> ready[2][64];
  auto* const kernel = grad ? ffn_small_kernel<true> : ffn_small_kernel<false>;
  if (!once_per_device(ready[grad != nullptr], [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S_SMEM) == cudaSuccess; }))
    return cudaErrorInvalidDevice;
  SmallParams q = {};
  q.n = n;
  long long tiles = 0;
  int order[kFfnGroup];              // the longest chains first
  for (int i = 0; i < n; ++i) {
    int at = i;
    for (; at > 0 && chunks_of(g[order[at - 1]]) < chunks_of(g[i]); --at) order[at] = order[at - 1];
    order[at] = i;
  }
  for (int k = 0; k < n; ++k) {
    const int i = order[k];
    SmallProblem& p = q.p[k];
    p.M = g[i].M; p.N = g[i].N; p.a_mn = g[i].a_mn; p.d = g[i].d; p.vec = vec4(p.d);
    for (int s = 0; s < 2; ++s) { p.K[s] = g[i].K[s]; p.A[s] = g[i].A[s]; p.B[s] = g[i].B[s]; }
    p.tiles_n = (p.N + S_T - 1) / S_T;
    tiles += tiles_of(g[i]);
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    p.tiles = (int)tiles_of(g[i]);
  }
  if (!grad) return launch_pdl(kernel, (int)tiles, S_THREADS, S_SMEM, st, q);
  q.act = grad->act; q.gate = grad->gate; q.up = grad->up;
  for (int k = 0; k < 3; ++k) q.out[k] = grad->out[k];
  q.p[0].vec = vec4(q.out[0]) && vec4(q.out[1]) && vec4(q.out[2]);
  return launch_pdl(kernel, (int)tiles, S_THREADS, S_SMEM, st, q);
}

}  // namespace gn
