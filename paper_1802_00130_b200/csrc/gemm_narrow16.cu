// Products of 16-bit matrices for the gated feed-forward block with few tokens (one and upwards): bound by reading the weights, so the weights are
// the rows of the tensor core's tile, 128 of them to a CTA, and the tokens its 16 to 128 columns.  Some hundred tokens take several columns of tiles,
// where the pairs' 256 x 256 tiles would be too few to fill the GPU.
//
// FFN_GATE takes 64 rows of the gate's weights and the same 64 of the up projection's, so that both sums of a hidden unit are in one CTA.
// Where the tiles are fewer than the SMs, a cluster of up to eight CTAs shares a tile, each with a part of K: the partial sums stay in
// shared memory, and each CTA adds, over the cluster in order of rank, those of its share of the tokens (no workspace, no atomics, no waiting on
// another cluster).  Roles: warp 0 TMA producer, warp 1 MMA issuer, warps 2..5 move the sums from tensor memory to shared memory; then every
// warp takes tokens of the epilogue.
//
// The second product of a call reads weights that the first does not write, and that nothing before the first can still be writing (the
// first has waited for it before it let this one start): its first slots are filled before it waits for the first.
// Half of an SM's shared memory to a CTA: with a third (more of the next kernel's CTAs find room early) one token took 38.1 us instead of 37.2 (4096 x
// 8192 bf16), and weights brought to L2 before the wait cost more than they hid (40.7).
// Bound by the weights' bytes, 5.4 TB/s there, and by 8 us of two dependent launches: 48 tokens, 2048 x 8192 fp16, 27.6 us, of which the stream is 15.
// Tiles of tokens: 256 tokens, 768 x 2048, 14.7 us (29.7 on the pairs' kernel), 256 x 4096 x 8192 60 (76).
#include <math.h>

#include "ffn_act.cuh"
#include "ffn_kernels.h"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int N_BM = 128, N_BK = 64, N_WARPS = 6, N_THREADS = 32 * N_WARPS;
constexpr int N_A_BYTES = N_BM * N_BK * 2;
constexpr int N_RING_BYTES = 108 * 1024;        // of stages: two CTAs on an SM
constexpr int N_STAGES_MAX = 8;
constexpr int N_SLICES = 8;                     // CTAs of a cluster at most
constexpr int N_TOKENS = 128;                   // tokens of a tile at most

struct NarrowParams {
  int tokens, features;              // of the result: d[0] [tokens][features]
  int n_pad, stages, cols_tmem;
  int kb0, kb;                       // k-blocks of the first operand pair, of both
  // early: the weights may be loaded before the kernel before this one is done
  int a_mn, act, early, vec;         // vec: every matrix of the epilogue takes accesses to four (FFN_GATE: two) elements
  Out16 d[3], low;
  Mat16 gate, up;
  int* err;
};
struct NarrowMaps { CUtensorMap m[4]; };         // weights and tokens of the first operand pair, of the second (FFN_GATE: gate, tokens, up, -)

template <bool BF16>
__device__ __forceinline__ void narrow_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accum) : "memory");
}
// (local: the address is one of this CTA's)
__device__ __forceinline__ float4 lds_cluster16(uint32_t addr, bool local) {
  float4 v;
  if (local) {
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
  }
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float2 lds_cluster8(uint32_t addr, bool local) {
  float2 v;
  if (local) {
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
  }
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}

// N elements (2 or 4) of row t from column f to a matrix, and the other way.
template <class T, int N>
__device__ __forceinline__ void put(const Out16& m, int t, int f, int features, int vec, const float (&x)[N]) {
  T* const p = reinterpret_cast<T*>(m.p) + (int64_t)t * m.ld + f;
  if (vec && f + N <= features) {
    if constexpr (N == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    else *reinterpret_cast<uint32_t*>(p) = pack2<T>(x[0], x[1]);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (f + e < features) p[e] = from_f<T>(x[e]);
  }
}
template <class T>
__device__ __forceinline__ void get4(const Mat16& m, int t, int f, int features, int vec, float (&x)[4]) {
  const T* const p = reinterpret_cast<const T*>(dep(m.p)) + (int64_t)t * m.ld + f;
  if (vec && f + 4 <= features) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = f + e < features ? to_f(p[e]) : 0.f;
  }
}

template <int KIND, class T>
__global__ void __launch_bounds__(N_THREADS, 2) ffn_narrow_kernel(const __grid_constant__ NarrowMaps maps, const __grid_constant__ NarrowParams p) {
  constexpr bool BF16 = !__is_same(T, __half);
  constexpr int WIDTH = KIND == FFN_GATE ? 64 : 128;             // features of a tile
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[N_STAGES_MAX], empty[N_STAGES_MAX], acc_full;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* const sums = reinterpret_cast<float*>(smem);            // [n_pad][128], in the ring's place once the products are done
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t slices, rank;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(slices));
  asm volatile("mov.u32 %0, %%cluster_ctaid.x;" : "=r"(rank));
  const int f0 = (int)(blockIdx.x / slices) * WIDTH, t0 = (int)blockIdx.y * N_TOKENS;
  const int tokens_here = min(N_TOKENS, p.tokens - t0);
  const int kb0 = (int)((long long)p.kb * rank / slices), kb1 = (int)((long long)p.kb * (rank + 1) / slices);
  const int stage_bytes = N_A_BYTES + p.n_pad * 128;

  if (threadIdx.x == 0) {
    for (int s = 0; s < N_STAGES_MAX; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    mbar_init(&acc_full, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(p.cols_tmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  if (warp != 0) {
    grid_dep_wait();
    grid_dep_launch();
  }

  if (warp == 0) {
    if (lane == 0) {
      const auto weights = [&](int kb, int s) {
        uint8_t* const sa = smem + s * stage_bytes;
        const int second = kb >= p.kb0 ? 1 : 0, k0 = (second ? kb - p.kb0 : kb) * N_BK;
        if (KIND == FFN_GATE) {
          tma_load_2d(sa, &maps.m[0], k0, f0, &full[s]);
          tma_load_2d(sa + 8192, &maps.m[2], k0, f0, &full[s]);
        } else if (!p.a_mn) {
          tma_load_2d(sa, &maps.m[2 * second], k0, f0, &full[s]);
        } else {
          tma_load_2d(sa, &maps.m[2 * second], f0, k0, &full[s]);
          tma_load_2d(sa + 8192, &maps.m[2 * second], f0 + 64, k0, &full[s]);
        }
      };
      const auto tokens = [&](int kb, int s) {
        const int second = kb >= p.kb0 ? 1 : 0, k0 = (second ? kb - p.kb0 : kb) * N_BK;
        tma_load_2d(smem + s * stage_bytes + N_A_BYTES, &maps.m[KIND == FFN_GATE ? 1 : 2 * second + 1], k0, t0, &full[s]);
      };
      const int head = p.early ? min(p.stages, kb1 - kb0) : 0;   // slots whose weights do not wait for the kernel before
      for (int i = 0; i < head; ++i) {
        mbar_expect_tx(&full[i], (uint32_t)stage_bytes);
        weights(kb0 + i, i);
      }
      grid_dep_wait();
      grid_dep_launch();
      for (int i = 0; i < head; ++i) tokens(kb0 + i, i);
      int s = head == p.stages ? 0 : head;
      uint32_t ph = head == p.stages ? 1u : 0u;
      for (int kb = kb0 + head; kb < kb1; ++kb) {
        if (!wait_or_abort(&empty[s], ph ^ 1, &abort_flag, p.err, 11)) break;
        mbar_expect_tx(&full[s], (uint32_t)stage_bytes);
        weights(kb, s);
        tokens(kb, s);
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)p.a_mn << 15) | ((uint32_t)(p.n_pad >> 3) << 17) |
                             ((uint32_t)(N_BM >> 4) << 24);
      const uint32_t base = smem_u32(smem);
      const uint64_t a_step = (p.a_mn ? 2048 : 32) >> 4;
      const uint64_t a0 = make_desc(base, p.a_mn ? 8192 : 16, 1024, 2), b0 = make_desc(base + N_A_BYTES, 16, 1024, 2);
      int s = 0;
      uint32_t ph = 0, acc = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!wait_or_abort(&full[s], ph, &abort_flag, p.err, 12)) { ok = false; break; }
        tc_fence_after();
        const uint64_t at = (uint64_t)(s * (stage_bytes >> 4));
#pragma unroll
        for (int k = 0; k < 4; ++k) { narrow_mma<BF16>(tmem, a0 + at + k * a_step, b0 + at + k * 2, idesc, acc); acc = 1u; }
        mma_commit(&empty[s]);
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (ok) mma_commit(&acc_full);
    }
    __syncwarp();
  } else {
    const int quad = warp & 3;
    int good = 1;
    if (lane == 0) good = wait_or_abort(&acc_full, 0, &abort_flag, p.err, 13) ? 1 : 0;
    good = __shfl_sync(0xffffffffu, good, 0);
    if (good && kb1 > kb0) {
      tc_fence_after();
      for (int c = 0; c < p.n_pad; c += 32) {
        float v[32];
        tmem_ld32(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)c, v);
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (c + i < p.n_pad) sums[(c + i) * N_BM + quad * 32 + lane] = v[i];
      }
    }
  }
  tc_fence_before();
  cluster_sync_all();                // every CTA's partial sums are in its shared memory

  // Tokens rank, rank + slices, ... are this CTA's, dealt to its warps; a token's sums are requested while the one before it is computed.
  constexpr int EACH = KIND == FFN_GATE ? 2 : 4;                 // columns of a thread
  const uint32_t mine = smem_u32(sums) + (uint32_t)(EACH * lane) * 4;
  const int first = (int)rank + (int)slices * warp, step = (int)slices * N_WARPS;
  const auto finish = [&](auto n_slices, auto act) {
    constexpr int S = decltype(n_slices)::value, ACT = decltype(act)::value;
    float4 v[S];                                                 // FFN_GATE: two sums of the gate, two of the up projection
    const auto request = [&](int t) {
#pragma unroll
      for (int q = 0; q < S; ++q) {
        const uint32_t here = mine + (uint32_t)t * (N_BM * 4), at = S == 1 ? here : map_to_cta(here, (uint32_t)q);
        if constexpr (KIND == FFN_GATE) {
          const float2 a = lds_cluster8(at, S == 1), b = lds_cluster8(at + 256, S == 1);
          v[q] = make_float4(a.x, a.y, b.x, b.y);
        } else {
          v[q] = lds_cluster16(at, S == 1);
        }
      }
    };
    if (first < tokens_here) request(first);
    for (int t = first; t < tokens_here; t += step) {
      float x[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int q = 1; q < S; ++q) { x[0] += v[q].x; x[1] += v[q].y; x[2] += v[q].z; x[3] += v[q].w; }
      if (t + step < tokens_here) request(t + step);
      const int f = f0 + EACH * lane;
      if (f >= p.features) continue;
      if constexpr (KIND == FFN_GATE) {
        float g[2] = {x[0], x[1]}, u[2] = {x[2], x[3]}, h[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float a, unused;
          activation<ACT, true>(g[e], a, unused);
          h[e] = a * u[e];
        }
        put<T>(p.d[0], t0 + t, f, p.features, p.vec, h);
        if (p.low.p) {               // (nothing is left of infinities and NaN, the rounding's own among them)
          float low[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float high = to_f(from_f<T>(h[e]));
            low[e] = fabsf(high) < __int_as_float(0x7f800000) ? h[e] - high : 0.f;
          }
          put<T>(p.low, t0 + t, f, p.features, p.vec, low);
        }
        if (p.d[1].p) put<T>(p.d[1], t0 + t, f, p.features, p.vec, g);
        if (p.d[2].p) put<T>(p.d[2], t0 + t, f, p.features, p.vec, u);
      } else if constexpr (KIND == FFN_STORE) {
        put<T>(p.d[0], t0 + t, f, p.features, p.vec, x);
      } else {
        float g[4], u[4], h[4], dg[4], du[4];
        get4<T>(p.gate, t0 + t, f, p.features, p.vec, g);
        get4<T>(p.up, t0 + t, f, p.features, p.vec, u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float a, da;
          activation<ACT, true>(g[e], a, da);
          h[e] = a * u[e]; dg[e] = x[e] * u[e] * da; du[e] = x[e] * a;
        }
        put<T>(p.d[0], t0 + t, f, p.features, p.vec, h);
        put<T>(p.d[1], t0 + t, f, p.features, p.vec, dg);
        put<T>(p.d[2], t0 + t, f, p.features, p.vec, du);
      }
    }
  };
  const auto by_slices = [&](auto act) {
    switch (slices) {
      case 1: finish(ActIs<1>{}, act); break;
      case 2: finish(ActIs<2>{}, act); break;
      case 4: finish(ActIs<4>{}, act); break;
      default: finish(ActIs<N_SLICES>{}, act);
    }
  };
  if constexpr (KIND == FFN_STORE) by_slices(ActIs<GN_ACT_RELU>{});
  else with_activation(p.act, by_slices);
  cluster_sync_all();                // nobody leaves while others read its sums
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.cols_tmem) : "memory");
  }
}

// ---- host side ---------------------------------------------------------------------------------
bool make_map16(CUtensorMap* m, const Mat16& a, long long rows, long long cols, int box_r, bool bf16) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)a.ld * 2};
  cuuint32_t box[2] = {64, (cuuint32_t)box_r};
  cuuint32_t estr[2] = {1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(a.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of features and of tokens, and CTAs to a tile: as many as still find an SM of their own (two of them share one at most), with four k-blocks each at least.
struct NarrowPlan { int tiles, columns, slices; };
NarrowPlan plan_narrow(int kind, int tokens, int features, int kb) {
  const int width = kind == FFN_GATE ? 64 : 128;
  NarrowPlan p{(features + width - 1) / width, (tokens + N_TOKENS - 1) / N_TOKENS, 1};
  while (p.slices < N_SLICES && (long long)p.tiles * p.columns * p.slices * 2 <= 2 * num_sms() && kb >= p.slices * 2 * 4) p.slices *= 2;
  return p;
}

template <int KIND, class T>
cudaError_t launch_narrow_as(int act, const FfnGemm& g, bool early, int* err, cudaStream_t st) {
  constexpr bool BF16 = !__is_same(T, __half);
  constexpr int WIDTH = KIND == FFN_GATE ? 64 : 128, EACH = KIND == FFN_GATE ? 2 : 4;
  static std::atomic<signed char> ready[64];
  auto* const kernel = ffn_narrow_kernel<KIND, T>;
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, N_RING_BYTES + 1024) == cudaSuccess; }))
    return cudaErrorInvalidDevice;
  NarrowMaps maps;
  NarrowParams p = {};
  p.tokens = g.M; p.features = g.N;
  p.n_pad = g.M < N_TOKENS ? (g.M + 15) / 16 * 16 : N_TOKENS;
  p.cols_tmem = p.n_pad <= 32 ? 32 : p.n_pad <= 64 ? 64 : 128;
  const int stage = N_A_BYTES + p.n_pad * 128;
  p.stages = N_RING_BYTES / stage < N_STAGES_MAX ? N_RING_BYTES / stage : N_STAGES_MAX;
  p.kb0 = (g.K[0] + N_BK - 1) / N_BK; p.kb = p.kb0 + (g.K[1] + N_BK - 1) / N_BK;
  p.a_mn = g.b_mn; p.act = act; p.early = early; p.err = err;
  p.vec = 1;
  for (int k = 0; k < 3; ++k) p.d[k] = g.d[k];
  p.low = g.low;
  p.gate = g.gate; p.up = g.up;
  const auto wide = [&](const void* q, int64_t ld) { return !q || (((uintptr_t)q & (2 * EACH - 1)) == 0 && ld % EACH == 0); };
  for (const Out16& o : g.d) p.vec &= wide(o.p, o.ld);
  p.vec &= wide(g.low.p, g.low.ld);
  p.vec &= wide(g.gate.p, g.gate.ld) && wide(g.up.p, g.up.ld);
  for (int s = 0; s < (KIND == FFN_GATE || g.K[1] > 0 ? 2 : 1); ++s) {
    const int a = KIND == FFN_GATE ? 0 : s, K = g.K[a];
    if (!(g.b_mn ? make_map16(&maps.m[2 * s], g.B[s], K, g.N, 64, BF16) : make_map16(&maps.m[2 * s], g.B[s], g.N, K, WIDTH, BF16)) ||
        !(KIND == FFN_GATE && s ? true : make_map16(&maps.m[2 * s + 1], g.A[a], g.M, K, p.n_pad, BF16)))
      return cudaErrorInvalidValue;
  }
  const NarrowPlan plan = plan_narrow(KIND, p.tokens, p.features, p.kb);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(plan.tiles * plan.slices), (unsigned)plan.columns);
  cfg.blockDim = dim3(N_THREADS);
  cfg.dynamicSmemBytes = N_RING_BYTES + 1024;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)plan.slices; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, maps, p);
}

}  // namespace

// 5 us for a launch, 3 for the ends of a round of CTAs (two on an SM) and 6 for another round's, and the k-blocks of an SM, or of a CTA where it has the SM for
// itself, 0.33 each: measured at 64 to 2048 tokens, 256 to 4096 columns and 256 to 8192 hidden units, within a fifth.
double ffn_narrow_us(FfnKind kind, int tokens, int features, int K) {
  const int kb = (K + N_BK - 1) / N_BK, sms = num_sms();
  const NarrowPlan p = plan_narrow(kind, tokens, features, kb);
  const double ctas = (double)p.tiles * p.columns * p.slices, share = (double)p.tiles * p.columns * kb / sms, own = (double)kb / p.slices;
  return 2.0 + 6.0 * ceil(ctas / (2 * sms)) + 0.33 * (share > own ? share : own);
}

cudaError_t launch_ffn_narrow(FfnKind kind, bool bf16, int act, const FfnGemm& g, bool early, int* err, cudaStream_t st) {
  if (kind == FFN_GATE) return bf16 ? launch_narrow_as<FFN_GATE, __nv_bfloat16>(act, g, early, err, st) : launch_narrow_as<FFN_GATE, __half>(act, g, early, err, st);
  if (kind == FFN_GRAD) return bf16 ? launch_narrow_as<FFN_GRAD, __nv_bfloat16>(act, g, early, err, st) : launch_narrow_as<FFN_GRAD, __half>(act, g, early, err, st);
  return bf16 ? launch_narrow_as<FFN_STORE, __nv_bfloat16>(act, g, early, err, st) : launch_narrow_as<FFN_STORE, __half>(act, g, early, err, st);
}

}  // namespace gn
