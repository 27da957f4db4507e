// Products of FP32 matrices over a mixture's experts on the tensor cores: the kernel of gemm_group16.cu on operands in three BF16 parts of eight bits each.
//
//   a b = sum of a_i b_j over the six pairs of parts with i + j <= 2 (0 the leading part).  Parts are rounded to nearest: |a_1| <= 2^-8 2^e, |a_2| <= 2^-16 2^e with 2^e <= |a|, so what is left out,
//   a_1 b_2 + a_2 b_1 + a_2 b_2, is below 2^-23 of |a b|, and of either sign.  (Parts cut off left out up to 3.9 times that, always towards zero.)
// Tiles of 256 x 128 of a CTA pair.  The tensor core cuts off what does not fit when it adds to a sum, always towards zero; so a sum is
// taken out of tensor memory after 256 terms, added to registers in FP32, and begun anew: four accumulators of 128 columns take turns.  The parts of h, dgate and dup are
// written by the epilogue that has them in FP32.  Taking the sums out costs a fifth of the time (dx of 16384 pairs, 1024 x 1024: 571 and 484 us before the elected lane, 353 now).
// Bound by what L2 gives to shared memory, 24 KB a CTA for 64 terms of 128 columns: 0.26 us, where the products take 0.14.  Tiles of 256 columns would read a quarter less, and
// leave half of the SMs without one in the small problems that FP32 is for: 1000 pairs of 8 experts, 784 x 300 are 24 to 56 tiles.
// Slots, tiles, roles and bounded waits are as in gemm_group16.cu.
#include "expert_kernels.h"
#include "pair_common.cuh"

namespace gn {
namespace {

constexpr int H_BM = 128, H_BK = 64, H_BN = 128, H_STAGES = 8, H_CHUNK = 4, H_BUFS = 4;
constexpr int H_A_BYTES = H_BM * H_BK * 2, H_B_BYTES = H_BN / 2 * H_BK * 2, H_STAGE_BYTES = H_A_BYTES + H_B_BYTES;
// Epilogue warps: GROUP_GRAD's time is its epilogue (an exact activation and its slope, nine matrices of parts), so it has sixteen, of 32 columns each.
template <int KIND> constexpr int tensor_warps = KIND == GROUP_GRAD ? 16 : 8;
template <int KIND> constexpr int tensor_threads = 64 + 32 * tensor_warps<KIND>;
constexpr int H_STG_ALL = 32 * 1024;
constexpr int H_SMEM = H_STAGES * H_STAGE_BYTES + H_STG_ALL + 1024 + 256;
static_assert(H_SMEM <= 232448, "more shared memory than a block can have");
constexpr int H_GRADS = 3, H_PRODUCTS = 6;
// (small products first)
__device__ __constant__ const signed char kPartA[H_PRODUCTS] = {2, 0, 1, 1, 0, 0}, kPartB[H_PRODUCTS] = {0, 2, 1, 0, 1, 0};

struct TensorGrad { int M, N, tiles_m, tiles_n, first, vec; Grads32 d; };
struct TensorParams {
  int N, tiles_n, kb, act, pairs, experts;
  int vec_gate, vec_up, vec_in;
  const ExpertTile* tiles; const int* n_tiles;
  const int *start, *count, *pair_of;
  Parts d, dgate, dup;
  FfnOut rows, gate_out, up_out;
  FfnMat gate, up;
  const float* weight; float* parts; int n_parts;
  TensorGrad grad[H_GRADS]; int n_grads, items;
  int* err;
};
template <int KIND> constexpr int tensor_maps = KIND == GROUP_GATE ? 3 : KIND == GROUP_DX ? 4 : KIND == GROUP_WEIGHT ? 2 * H_GRADS : 2;
template <int KIND> struct TensorMaps { CUtensorMap m[tensor_maps<KIND>]; };

struct TensorItem { int expert, slot, rows, padded, m0, n0, kb, grad; };
template <int KIND>
__device__ __forceinline__ TensorItem tensor_item(const TensorParams& p, int i) {
  TensorItem w;
  if constexpr (KIND == GROUP_WEIGHT) {
    w.grad = 0;
    while (w.grad + 1 < p.n_grads && i >= p.grad[w.grad + 1].first) ++w.grad;
    const TensorGrad& g = p.grad[w.grad];
    const int each = g.tiles_m * g.tiles_n, in = i - g.first;
    w.expert = in / each;
    const int t = in - w.expert * each;
    w.m0 = t / g.tiles_n * 2 * H_BM; w.n0 = t % g.tiles_n * H_BN;
    w.slot = p.start[w.expert];
    w.kb = (p.count[w.expert] + H_BK - 1) / H_BK;
    w.rows = w.padded = 0;
  } else {
    const int t = i / p.tiles_n;
    const int4 e = *reinterpret_cast<const int4*>(p.tiles + t);
    w.expert = e.x; w.slot = e.y; w.rows = e.z; w.padded = e.w;
    w.n0 = (i - t * p.tiles_n) * (KIND == GROUP_GATE ? H_BN / 2 : H_BN);
    w.m0 = 0; w.kb = p.kb; w.grad = 0;
  }
  return w;
}
__device__ __forceinline__ float4 four32(const float* row, int c, int n, bool vec) {
  if (!row || c >= n) return make_float4(0.f, 0.f, 0.f, 0.f);
  if (vec && c + 4 <= n) return *reinterpret_cast<const float4*>(row + c);
  float4 v = make_float4(row[c], 0.f, 0.f, 0.f);
  if (c + 1 < n) v.y = row[c + 1];
  if (c + 2 < n) v.z = row[c + 2];
  if (c + 3 < n) v.w = row[c + 3];
  return v;
}
// The three parts of v, and of w beside them: the first two rounded to nearest (halves away from zero), so that what is left is half as large, and of either sign; the third is all that is left.  What
// would be rounded to infinity is cut off.  An infinity is a third part alone, which meets the other number's first part and nothing else: its product is infinite (NaN with a zero, or with another
// infinity, which has no first part).  Of a NaN one part at least is one.
__device__ __forceinline__ uint32_t first_part(float v, bool infinite) {
  const uint32_t a = __float_as_uint(v);
  return infinite ? 0u : (a & 0x7fffffffu) < 0x7f7f8000u ? a + 0x8000u : a;
}
__device__ __forceinline__ uint32_t next_part(float v, bool infinite) { return infinite ? 0u : __float_as_uint(v) + 0x8000u; }
__device__ __forceinline__ float less(float v, uint32_t part) { return v - __uint_as_float(part & 0xffff0000u); }
__device__ __forceinline__ void three(float v, float w, uint32_t (&o)[3]) {
  const bool iv = fabsf(v) == __int_as_float(0x7f800000), iw = fabsf(w) == __int_as_float(0x7f800000);
  uint32_t a = first_part(v, iv), b = first_part(w, iw);
  o[0] = __byte_perm(a, b, 0x7632);
  v = less(v, a); w = less(w, b);
  a = next_part(v, iv); b = next_part(w, iw);
  o[1] = __byte_perm(a, b, 0x7632);
  o[2] = __byte_perm(__float_as_uint(less(v, a)), __float_as_uint(less(w, b)), 0x7632);
}

__device__ __forceinline__ TensorItem uniform_item(TensorItem w) {
  w.expert = uniform(w.expert); w.slot = uniform(w.slot); w.m0 = uniform(w.m0); w.n0 = uniform(w.n0); w.kb = uniform(w.kb); w.grad = uniform(w.grad);
  return w;
}

template <int KIND>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(tensor_threads<KIND>, 1)
group32_kernel(const __grid_constant__ TensorMaps<KIND> maps, const __grid_constant__ TensorParams p) {
  constexpr bool A_MN = KIND == GROUP_WEIGHT, B_MN = KIND == GROUP_GRAD || KIND == GROUP_DX || KIND == GROUP_WEIGHT;
  constexpr int WARPS = tensor_warps<KIND>, SEGMENTS = KIND == GROUP_DX ? 2 * H_PRODUCTS : H_PRODUCTS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = smem + H_STAGES * H_STAGE_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + H_STG_ALL);
  uint64_t* empty = full + H_STAGES;
  uint64_t* acc_full = empty + H_STAGES;           // [H_BUFS]
  uint64_t* acc_empty = acc_full + H_BUFS;         // [H_BUFS]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + H_BUFS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < H_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int b = 0; b < H_BUFS; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 2 * WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();
  const int items = KIND == GROUP_WEIGHT ? p.items : uniform(*dep(p.n_tiles)) * p.tiles_n;

  if (warp == 0) {
    int s = 0;
    uint32_t ph = 0;
    bool ok = true;
    const uint32_t full_leader = map_to_cta(smem_u32(&full[0]), 0);
    for (int i = pair; ok && i < items; i += p.pairs) {
      const TensorItem w = uniform_item(tensor_item<KIND>(p, i));
      const int m0 = (KIND == GROUP_WEIGHT ? w.m0 : w.slot) + (int)rank * H_BM, n0 = KIND == GROUP_GATE ? w.n0 : w.n0 + (int)rank * (H_BN / 2);
#pragma unroll 1
      for (int seg = 0; seg < SEGMENTS && ok; ++seg) {
        const int second = seg >= H_PRODUCTS ? 1 : 0, pa = kPartA[seg - second * H_PRODUCTS], pb = kPartB[seg - second * H_PRODUCTS];
#pragma unroll 1
        for (int kb = 0; kb < w.kb; ++kb) {
          if (!warp_wait_or_abort(&empty[s], ph ^ 1, abort_flag, p.err, 1)) { ok = false; break; }
          if (elect_one()) {
            if (rank == 0) mbar_expect_tx(&full[s], 2u * H_STAGE_BYTES);
            const uint32_t bar = full_leader + (uint32_t)s * 8u;
            uint8_t* const sa = smem + s * H_STAGE_BYTES;
            uint8_t* const sb = sa + H_A_BYTES;
            if constexpr (KIND == GROUP_WEIGHT) {
              const CUtensorMap* const ma = &maps.m[2 * w.grad];
              const int k0 = w.slot + kb * H_BK;
              tma2_load_3d(sa, ma, m0, k0, pa, bar);
              tma2_load_3d(sa + 8192, ma, m0 + 64, k0, pa, bar);
              tma2_load_3d(sb, ma + 1, n0, k0, pb, bar);
            } else {
              const int k0 = kb * H_BK, z = pb * p.experts + w.expert;
              tma2_load_3d(sa, &maps.m[2 * second], k0, m0, pa, bar);
              const CUtensorMap* const mb = &maps.m[KIND == GROUP_GATE ? (rank ? 2 : 1) : 2 * second + 1];
              if constexpr (!B_MN) tma2_load_3d(sb, mb, k0, n0, z, bar);
              else tma2_load_3d(sb, mb, n0, k0, z, bar);
            }
          }
          if (++s == H_STAGES) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t base = smem_u32(smem);
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(H_BN >> 3) << 17) |
                             ((uint32_t)((2 * H_BM) >> 4) << 24);
      constexpr uint64_t a_step = (A_MN ? 2048 : 32) >> 4, b_step = (B_MN ? 2048 : 32) >> 4;
      const uint64_t a0 = make_desc(base, A_MN ? 8192 : 16, 1024, 2);
      const uint64_t b0 = make_desc(base + H_A_BYTES, B_MN ? 8192 : 16, 1024, 2);
      int s = 0, ci = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int i = pair; ok && i < items; i += p.pairs) {
        const TensorItem w = uniform_item(tensor_item<KIND>(p, i));
        const int total = w.kb * SEGMENTS;
#pragma unroll 1
        for (int kb = 0; kb < total && ok; kb += H_CHUNK, ++ci) {
          const int buf = ci % H_BUFS;
          if (!warp_wait_or_abort(&acc_empty[buf], ((ci / H_BUFS) & 1) ^ 1, abort_flag, p.err, 4)) { ok = false; break; }
          tc_fence_after();
          const uint32_t tmem_d = tmem_base + (uint32_t)(buf * H_BN);
          uint32_t acc = 0u;
          const int end = min(kb + H_CHUNK, total);
#pragma unroll 1
          for (int j = kb; j < end; ++j) {
            if (!warp_wait_or_abort(&full[s], ph, abort_flag, p.err, 2)) { ok = false; break; }
            tc_fence_after();
            const uint64_t ad = a0 + (uint64_t)(s * (H_STAGE_BYTES >> 4)), bd = b0 + (uint64_t)(s * (H_STAGE_BYTES >> 4));
            if (elect_one()) {
              pair_mma<true>(tmem_d, ad, bd, idesc, acc);
              pair_mma<true>(tmem_d, ad + a_step, bd + b_step, idesc, 1u);
              pair_mma<true>(tmem_d, ad + 2 * a_step, bd + 2 * b_step, idesc, 1u);
              pair_mma<true>(tmem_d, ad + 3 * a_step, bd + 3 * b_step, idesc, 1u);
              mma2_commit_both(&empty[s]);
            }
            acc = 1u;
            if (++s == H_STAGES) { s = 0; ph ^= 1u; }
          }
          if (ok && elect_one()) mma2_commit_both(&acc_full[buf]);
        }
      }
    }
  } else {
    // Epilogue: a quadrant's two warps take half of its columns each (GROUP_GATE: of both projections; GROUP_GRAD: its four a quarter).
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const uint32_t stg = smem_u32(staging + (warp - 2) * (H_STG_ALL / WARPS));
    const uint32_t acc_leader = map_to_cta(smem_u32(&acc_empty[0]), 0);
    const int* const pair_of = dep(p.pair_of);
    const float* const weight = dep(p.weight);
    const uint32_t tq = tmem_base + ((uint32_t)(quad * 32) << 16);
    const uint32_t col0 = KIND == GROUP_GATE || KIND == GROUP_GRAD ? half * 32 : half * 64, col1 = KIND == GROUP_GATE ? 64 + half * 32 : half * 64 + 32;
    int ci = 0;
    bool ok = true;
    for (int i = pair; ok && i < items; i += p.pairs) {
      const TensorItem w = tensor_item<KIND>(p, i);
      const int r0 = (int)rank * H_BM + quad * 32;
      const int N = KIND == GROUP_WEIGHT ? p.grad[w.grad].N : p.N;
      const int rows = KIND == GROUP_WEIGHT ? p.grad[w.grad].M - w.m0 : KIND == GROUP_GRAD ? w.padded : w.rows;
      int my_pair = -1, my_slot = -1;
      if (KIND != GROUP_WEIGHT && r0 + lane < rows) {
        my_slot = w.slot + r0 + lane;
        my_pair = r0 + lane < w.rows ? pair_of[my_slot] : -1;
      }
      const auto pair_row = [&](int r) { return __shfl_sync(0xffffffffu, my_pair, r); };
      const auto slot_row = [&](int r) { return r0 + r < rows ? w.slot + r0 + r : -1; };
      float x[32], y[32];
#pragma unroll
      for (int q = 0; q < 32; ++q) x[q] = y[q] = 0.f;
      const int chunks = (w.kb * SEGMENTS + H_CHUNK - 1) / H_CHUNK;
#pragma unroll 1
      for (int c = 0; c < chunks; ++c, ++ci) {
        const int buf = ci % H_BUFS;
        int good = 1;
        if (lane == 0) good = wait_or_abort(&acc_full[buf], (ci / H_BUFS) & 1, abort_flag, p.err, 3) ? 1 : 0;
        good = __shfl_sync(0xffffffffu, good, 0);
        if (!good) { ok = false; break; }
        tc_fence_after();
        float v[32], u[32];
        if constexpr (KIND == GROUP_GRAD) tmem_ld32(tq + (uint32_t)(buf * H_BN) + col0, v);
        else tmem_ld32_pair(tq + (uint32_t)(buf * H_BN) + col0, tq + (uint32_t)(buf * H_BN) + col1, v, u);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(acc_leader + (uint32_t)buf * 8u);
#pragma unroll
        for (int q = 0; q < 32; ++q) {
          x[q] += v[q];
          if constexpr (KIND != GROUP_GRAD) y[q] += u[q];
        }
      }
      if (!ok) break;
      // 32 columns of FP32 to rows of pairs or of a gradient (as 64 of 16 bits), or in parts to slots
      const auto put32 = [&](const float (&v)[32], float* base, int64_t ld, auto row_of, int n0, bool vec) {
        uint32_t o[32];
#pragma unroll
        for (int q = 0; q < 32; ++q) o[q] = __float_as_uint(v[q]);
        put_rows<8>(o, stg, lane, base, 2 * ld, row_of, 2 * n0, 2 * N, vec);
      };
      const auto put_parts = [&](const float (&v)[32], const Parts& to, int n0) {
        uint32_t o[3][16];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          uint32_t t[3];
          three(v[2 * q], v[2 * q + 1], t);
          o[0][q] = t[0]; o[1][q] = t[1]; o[2][q] = t[2];
        }
#pragma unroll
        for (int j = 0; j < 3; ++j) put_rows<4>(o[j], stg, lane, reinterpret_cast<uint16_t*>(to.p) + j * to.rows * to.ld, to.ld, slot_row, n0, N, true);
      };
      if constexpr (KIND == GROUP_GATE) {
        const int nc = w.n0 + half * 32;
        if (r0 < rows && nc < N) {
          if (p.gate_out.p) put32(x, p.gate_out.p, p.gate_out.ld, pair_row, nc, p.vec_gate);
          if (p.up_out.p) put32(y, p.up_out.p, p.up_out.ld, pair_row, nc, p.vec_up);
          with_activation(p.act, [&](auto act) {
#pragma unroll
            for (int q = 0; q < 32; ++q) {
              float a, unused;
              activation<decltype(act)::value, false>(x[q], a, unused);
              x[q] = a * y[q];
            }
          });
          put_parts(x, p.d, nc);
        }
      } else if constexpr (KIND == GROUP_GRAD) {
        const float share = my_pair >= 0 ? weight[my_pair] : 0.f;
        float sum = 0.f;
        const float* const gate = my_pair >= 0 ? dep(p.gate.p) + my_pair * p.gate.ld : nullptr;
        const float* const up = my_pair >= 0 ? dep(p.up.p) + my_pair * p.up.ld : nullptr;
        const int nc = w.n0 + half * 32;
        if (r0 < rows && nc < N) {
          float h[32], dg[32];
          with_activation(p.act, [&](auto act) {
#pragma unroll
            for (int f = 0; f < 8; ++f) {
              const float4 g4 = four32(gate, nc + 4 * f, N, p.vec_in), u4 = four32(up, nc + 4 * f, N, p.vec_in);
              const float gs[4] = {g4.x, g4.y, g4.z, g4.w}, us[4] = {u4.x, u4.y, u4.z, u4.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float q = my_pair >= 0 ? x[4 * f + e] : 0.f;        // (an empty slot: zero, whatever the weights are)
                float a, da;
                activation<decltype(act)::value, false>(gs[e], a, da);
                const float plain = a * us[e];
                sum = fmaf(q, plain, sum);                 // (past the last column both are zero)
                h[4 * f + e] = share * plain; dg[4 * f + e] = share * q * us[e] * da; x[4 * f + e] = share * q * a;
              }
            }
          });
          put_parts(h, p.d, nc);
          put_parts(dg, p.dgate, nc);
          put_parts(x, p.dup, nc);
        }
        if (my_pair >= 0) p.parts[(int64_t)my_slot * p.n_parts + w.n0 / H_BN * 4 + half] = sum;
      } else {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int nc = w.n0 + half * 64 + b * 32;
          if (r0 >= rows || nc >= N) continue;
          if constexpr (KIND == GROUP_WEIGHT) {
            const TensorGrad& g = p.grad[w.grad];
            put32(b ? y : x, g.d.p + w.expert * g.d.stride, g.d.ld, [&](int r) { return w.m0 + r0 + r < g.M ? w.m0 + r0 + r : -1; }, nc, g.vec);
          } else {
            put32(b ? y : x, p.rows.p, p.rows.ld, pair_row, nc, true);
          }
        }
      }
    }
  }
  tc_fence_before();
  cluster_sync_all();      // neither CTA leaves (or frees tensor memory) while the other may still use it
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// ---- splitting ---------------------------------------------------------------------------------
constexpr int kSplits = 3;
struct SplitMatsList { SplitMats j[kSplits]; int vec[kSplits]; };
// A thread takes eight columns of a row: 16 bytes of each part.
__device__ __forceinline__ void split_eight(const float* row, int c, int cols, bool vec, uint4 (&o)[3]) {
  const float4 a = four32(row, c, cols, vec), b = four32(row, c + 4, cols, vec);
  uint32_t t[4][3];
  three(a.x, a.y, t[0]); three(a.z, a.w, t[1]); three(b.x, b.y, t[2]); three(b.z, b.w, t[3]);
#pragma unroll
  for (int j = 0; j < 3; ++j) o[j] = make_uint4(t[0][j], t[1][j], t[2][j], t[3][j]);
}
__global__ void __launch_bounds__(256) split_mats_kernel(const __grid_constant__ SplitMatsList list) {
  grid_dep_wait();
  grid_dep_launch();
  const SplitMats& j = list.j[blockIdx.y];
  const float* const src = dep(j.src);
  const int64_t units = j.to.ld / 8, all = j.experts * j.rows, work = all * units;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t r = work <= 0x7fffffff ? (int64_t)((uint32_t)i / (uint32_t)units) : i / units, e = work <= 0x7fffffff ? (int64_t)((uint32_t)r / (uint32_t)j.rows) : r / j.rows;
    const int c = (int)(i - r * units) * 8;
    uint4 o[3];
    split_eight(src + e * j.stride + (r - e * j.rows) * j.ld, c, j.cols, list.vec[blockIdx.y], o);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(j.to.p) + (q * all + r) * j.to.ld + c) = o[q];
  }
}
struct SplitRowsList { SplitRows j[2]; int vec[2]; int64_t tokens; int k, cols, zero; ExpertPlan plan; };
__global__ void __launch_bounds__(256) split_to_slots_kernel(const __grid_constant__ SplitRowsList p) {
  grid_dep_wait();
  grid_dep_launch();
  const SplitRows& j = p.j[blockIdx.y];
  const float* const src = dep(j.src);
  uint16_t* const to = reinterpret_cast<uint16_t*>(j.to.p);
  const int64_t units = j.to.ld / 8, part = j.to.rows * j.to.ld, work = (p.tokens + p.zero) * units;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / units;
    const int c = (int)(i - t * units) * 8;
    if (t >= p.tokens) {
      const int e = (int)(t - p.tokens), n = p.plan.count[e], end = (n + kSlots - 1) / kSlots * kSlots;
      for (int s = n; s < end; ++s)
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(to + q * part + (p.plan.start[e] + s) * j.to.ld + c) = make_uint4(0u, 0u, 0u, 0u);
      continue;
    }
    uint4 o[3];
    split_eight(src + t * j.ld, c, p.cols, p.vec[blockIdx.y], o);
    for (int q = 0; q < p.k; ++q) {
      const int slot = p.plan.slot_of[t * p.k + q];
      if (slot < 0) continue;
#pragma unroll
      for (int h = 0; h < 3; ++h) *reinterpret_cast<uint4*>(to + h * part + slot * j.to.ld + c) = o[h];
    }
  }
}

// ---- host side ---------------------------------------------------------------------------------
// 3-D map over [planes][rows][cols] without gaps between the planes; box = 64 columns x box_r rows of one.
bool make_map_planes(CUtensorMap* m, const Parts& a, long long planes, long long rows, long long cols, int box_r) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)a.ld * 2, (cuuint64_t)(rows * a.ld * 2)};
  cuuint32_t box[3] = {64, (cuuint32_t)box_r, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool vec32(const void* p, int64_t ld, int64_t stride = 0) { return !p || (((uintptr_t)p & 15) == 0 && ld % 4 == 0 && stride % 4 == 0); }

template <int KIND>
cudaError_t launch_group32_as(const TensorGroup& g, const ExpertPlan& plan, int* err, cudaStream_t st) {
  static std::atomic<signed char> ready[64];
  auto* const kernel = group32_kernel<KIND>;
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, H_SMEM) == cudaSuccess; }))
    return cudaErrorInvalidDevice;
  TensorMaps<KIND> maps;
  TensorParams p = {};
  long long most;                    // items
  bool ok = true;
  p.act = g.act; p.err = err; p.experts = plan.experts;
  p.tiles = plan.tiles; p.n_tiles = plan.n_tiles; p.start = plan.start; p.count = plan.count; p.pair_of = plan.pair_of;
  if constexpr (KIND == GROUP_WEIGHT) {
    p.n_grads = g.n_grads;
    most = 0;
    for (int i = 0; i < g.n_grads; ++i) {
      const auto& q = g.grads[i];
      TensorGrad& to = p.grad[i];
      to.M = q.M; to.N = q.N; to.tiles_m = (q.M + 2 * H_BM - 1) / (2 * H_BM); to.tiles_n = (q.N + H_BN - 1) / H_BN; to.first = (int)most; to.d = q.d;
      to.vec = vec32(q.d.p, q.d.ld, q.d.stride);
      most += (long long)plan.experts * to.tiles_m * to.tiles_n;
      if (most > 0x3fffffff) return cudaErrorInvalidValue;
      ok = ok && make_map_planes(&maps.m[2 * i], q.left, 3, q.left.rows, q.M, H_BK) && make_map_planes(&maps.m[2 * i + 1], q.right, 3, q.right.rows, q.N, H_BK);
    }
    p.items = (int)most;
  } else {
    constexpr int WIDTH = KIND == GROUP_GATE ? H_BN / 2 : H_BN;
    p.N = g.N; p.tiles_n = (g.N + WIDTH - 1) / WIDTH; p.kb = (g.K + H_BK - 1) / H_BK;
    p.d = g.d; p.dgate = g.dgate; p.dup = g.dup; p.rows = g.rows; p.gate_out = g.gate_out; p.up_out = g.up_out; p.gate = g.gate; p.up = g.up;
    p.vec_gate = vec32(p.gate_out.p, p.gate_out.ld); p.vec_up = vec32(p.up_out.p, p.up_out.ld); p.vec_in = vec32(p.gate.p, p.gate.ld) && vec32(p.up.p, p.up.ld);
    p.weight = g.weight; p.parts = g.parts; p.n_parts = tensor_parts(g.N);
    most = plan_tiles(plan.pairs, plan.experts, 2 * H_BM) * p.tiles_n;
    if (most > 0x3fffffff) return cudaErrorInvalidValue;
    for (int s = 0; s < (KIND == GROUP_DX ? 2 : 1); ++s) ok = ok && make_map_planes(&maps.m[2 * s], g.A[s], 3, g.A[s].rows, g.K, H_BM);
    const auto weights = [&](int at, int b) {
      if (KIND == GROUP_GATE || KIND == GROUP_DOWN) return make_map_planes(&maps.m[at], g.B[b], 3LL * plan.experts, g.N, g.K, H_BN / 2);
      return make_map_planes(&maps.m[at], g.B[b], 3LL * plan.experts, g.K, g.N, H_BK);
    };
    ok = ok && weights(1, 0);
    if (KIND == GROUP_GATE) ok = ok && weights(2, 1);
    if (KIND == GROUP_DX) ok = ok && weights(3, 1);
  }
  if (!ok) return cudaErrorInvalidValue;
  const int pairs = num_sms() / 2;
  p.pairs = most < pairs ? (int)most : pairs;
  return launch_pdl(kernel, 2 * p.pairs, tensor_threads<KIND>, H_SMEM, st, maps, p);
}

}  // namespace

int tensor_parts(int N) { return (N + H_BN - 1) / H_BN * 4; }

cudaError_t launch_group32(GroupKind kind, const TensorGroup& g, const ExpertPlan& plan, int* err, cudaStream_t st) {
  switch (kind) {
    case GROUP_GATE: return launch_group32_as<GROUP_GATE>(g, plan, err, st);
    case GROUP_DOWN: return launch_group32_as<GROUP_DOWN>(g, plan, err, st);
    case GROUP_GRAD: return launch_group32_as<GROUP_GRAD>(g, plan, err, st);
    case GROUP_DX: return launch_group32_as<GROUP_DX>(g, plan, err, st);
    default: return launch_group32_as<GROUP_WEIGHT>(g, plan, err, st);
  }
}

cudaError_t launch_split_mats(const SplitMats* list, int n, cudaStream_t st) {
  SplitMatsList q = {};
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    q.j[i] = list[i];
    q.vec[i] = vec32(list[i].src, list[i].ld, list[i].experts > 1 ? list[i].stride : 0);
    const int64_t work = list[i].experts * list[i].rows * (list[i].to.ld / 8);
    most = work > most ? work : most;
  }
  const int64_t want = (most + 255) / 256, cap = (int64_t)num_sms() * 16;
  return launch_pdl_grid(split_mats_kernel, dim3((unsigned)(want < cap ? want : cap), (unsigned)n), 256, 0, st, q);
}
cudaError_t launch_split_to_slots(const SplitRows* list, int n, int64_t tokens, int k, int cols, bool zero, const ExpertPlan& plan, cudaStream_t st) {
  SplitRowsList q = {};
  for (int i = 0; i < n; ++i) { q.j[i] = list[i]; q.vec[i] = vec32(list[i].src, list[i].ld); }
  q.tokens = tokens; q.k = k; q.cols = cols; q.zero = zero ? plan.experts : 0; q.plan = plan;
  const int64_t want = ((tokens + q.zero) * (list[0].to.ld / 8) + 255) / 256, cap = (int64_t)num_sms() * 16;
  return launch_pdl_grid(split_to_slots_kernel, dim3((unsigned)(want < cap ? want : cap), (unsigned)n), 256, 0, st, q);
}

}  // namespace gn
