// Products of 16-bit matrices for the gated feed-forward block: a CTA pair per tile (tcgen05.mma.cta_group::2, operands by TMA, accumulators in
// tensor memory).  ffn_pair_kernel has 256 x bn tiles, with the gate or its gradient as the epilogue; ffn_wide_kernel, below, plain products.
//
// Persistent: one pair for two SMs, tiles dealt in turn.  Warp roles in each CTA of ffn_pair_kernel:
//   warp 0      TMA producer: a ring of STAGES slots, each this CTA's 128 rows of A and its half of the B tile, 64 terms of K
//   warp 1      MMA issuer (leader CTA only), one thread
//   warps 2..   epilogue, beside the next tile's products where two accumulators fit the tensor memory (256 x 256 tiles)
//
// FFN_GATE: the B tile is bn / 2 rows of the gate's weights, staged by the leader, and the same rows of the up projection's, staged by
// the other CTA: one product gives both sums of bn / 2 hidden units, and a thread finds them in the same tensor-memory lane.
//
// A thread of the epilogue holds a row (a tensor-memory lane) of a chunk of columns.  What goes to or comes from global memory passes a
// staging tile in shared memory, so that a warp's access covers whole runs of its rows.
//
// h, and in the backward pass dgate and dup, are rounded to the type here: they are operands of the next product, which two parts of each would double (of h forward: a
// third more of the whole).  A result is then off by sqrt 2 times its own rounding (8192 x 4096 x 8192 BF16: 0.0023 of it in the 2-norm, 0.0017 with FP32 in between).
//
// Operand layouts are those of gemm_tf32.cu's FP16 copies: K-major rows of 128 bytes, or MN-major chunks of 64 columns x 64 rows, both
// with the plain 128-byte swizzle.  Every wait is bounded; a role that gives up leaves a code in *err and the CTA drains.
#include "ffn_act.cuh"
#include "ffn_kernels.h"
#include "pair_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int P_BM = 128, P_BK = 64, P_BN = 256;
constexpr int P_STAGES = 6;
constexpr int P_A_BYTES = P_BM * P_BK * 2, P_STAGE_BYTES = 2 * P_A_BYTES;
// Epilogue warps, and the 16-byte units of a staging row.  FFN_GRAD's time is latency: with eight warps a tile's epilogue takes longer than the next
// tile's products (8192 x 8192 x 4096: 757 thousand cycles, 679 with sixteen, whose staging tiles hold 32 columns); FFN_GATE's is instructions (1226 and 1259).
template <int KIND> constexpr int epi_warps = KIND == FFN_GRAD ? 16 : 8;
template <int KIND> constexpr int epi_units = KIND == FFN_GRAD ? 4 : 8;
template <int KIND> constexpr int pair_threads = 64 + 32 * epi_warps<KIND>;
constexpr int P_STG_ALL = 32 * 1024;
constexpr int P_SMEM = P_STAGES * P_STAGE_BYTES + P_STG_ALL + 1024 + 256;
static_assert(P_SMEM <= 232448, "more shared memory than a block can have");
constexpr int P_PANELS = 8;       // tiles are walked in strips of so many row panels: 74 tiles at a time read 8 panels of A and 9 of B

struct PairParams {
  int M, N, bn, tiles_m, tiles_n, tiles, pairs;
  int kb;                         // k-blocks
  int vec, act;                   // vec: bit k: 16-byte accesses for d[k]
  int b_box3;                     // an MN-major B of whole 64-column chunks: one box of several chunks instead of a box each
  Out16 d[3];
  Mat16 gate, up;
  int* err;
};
struct PairMaps { CUtensorMap m[3]; };           // A, B (FFN_GATE: gate weights, up weights)
template <int NP> struct WideMaps { CUtensorMap m[NP][4]; };   // A0, B0, A1, B1

// Place of the t-th tile.
__device__ __forceinline__ void find_tile(const PairParams& p, int t, int& m, int& n) {
  const int strip = t / (P_PANELS * p.tiles_n), rest = t - strip * P_PANELS * p.tiles_n;
  const int high = min(P_PANELS, p.tiles_m - strip * P_PANELS);
  m = strip * P_PANELS + rest % high; n = rest / high;
}

template <int KIND, class T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads<KIND>, 1)
ffn_pair_kernel(const __grid_constant__ PairMaps maps, const __grid_constant__ PairParams p) {
  static_assert(KIND == FFN_GATE || KIND == FFN_GRAD, "plain products: ffn_wide_kernel");
  constexpr bool B_MN = KIND == FFN_GRAD;          // (dy is K-major, Wd [cols][inner] is not; the forward pass' operands are)
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = smem + P_STAGES * P_STAGE_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + P_STG_ALL);
  uint64_t* empty = full + P_STAGES;
  uint64_t* acc_full = empty + P_STAGES;   // [2]
  uint64_t* acc_empty = acc_full + 2;      // [2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < P_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 2 * epi_warps<KIND>); }
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

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      const uint32_t full_leader = map_to_cta(smem_u32(&full[0]), 0);
      const int hb = p.bn >> 1;                            // B rows staged by each CTA
      const uint32_t pair_tx = 2u * (P_A_BYTES + (uint32_t)hb * 128u);
      const CUtensorMap* const ma = &maps.m[0];
      const CUtensorMap* const mb = &maps.m[KIND == FFN_GATE && rank ? 2 : 1];
      const bool b3 = p.b_box3 != 0;
      for (int t = pair; ok && t < p.tiles; t += p.pairs) {
        int tm, tn;
        find_tile(p, t, tm, tn);
        const int m0 = tm * 2 * P_BM + (int)rank * P_BM;
        const int n0 = KIND == FFN_GATE ? tn * hb : tn * p.bn + (int)rank * hb;
        // (one thread issues everything: nothing is in the loop that need not be there)
#pragma unroll 1
        for (int kb = 0; kb < p.kb; ++kb) {
          if (!wait_or_abort(&empty[s], ph ^ 1, abort_flag, p.err, 1)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(&full[s], pair_tx);
          const uint32_t bar = full_leader + (uint32_t)s * 8u;
          const int k0 = kb * P_BK;
          uint8_t* const sa = smem + s * P_STAGE_BYTES;
          uint8_t* const sb = sa + P_A_BYTES;
          tma2_load_2d(sa, ma, k0, m0, bar);
          if (!B_MN) {
            tma2_load_2d(sb, mb, k0, n0, bar);
          } else if (b3) {
            tma2_load_3d(sb, mb, 0, k0, n0 >> 6, bar);
          } else {
            tma2_load_2d(sb, mb, n0, k0, bar);
            if (hb > 64) tma2_load_2d(sb + 8192, mb, n0 + 64, k0, bar);
          }
          if (++s == P_STAGES) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && lane == 0) {
      constexpr bool BF16 = !__is_same(T, __half);
      const uint32_t base = smem_u32(smem);
      const uint32_t idesc = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(p.bn >> 3) << 17) | ((uint32_t)((2 * P_BM) >> 4) << 24);
      constexpr uint64_t a_step = 32 >> 4, b_step = (B_MN ? 2048 : 32) >> 4;
      const uint64_t a0 = make_desc(base, 16, 1024, 2);
      const uint64_t b0 = make_desc(base + P_A_BYTES, B_MN ? 8192 : 16, 1024, 2);
      int s = 0, ti = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int t = pair; ok && t < p.tiles; t += p.pairs, ++ti) {
        const int buf = ti & 1;
        if (!wait_or_abort(&acc_empty[buf], ((ti >> 1) & 1) ^ 1, abort_flag, p.err, 4)) break;
        tc_fence_after();
        const uint32_t tmem_d = tmem_base + (uint32_t)(buf * P_BN);
        uint32_t acc = 0u;
#pragma unroll 1
        for (int kb = 0; kb < p.kb; ++kb) {
          if (!wait_or_abort(&full[s], ph, abort_flag, p.err, 2)) { ok = false; break; }
          tc_fence_after();
          const uint64_t ad = a0 + (uint64_t)(s * (P_STAGE_BYTES >> 4)), bd = b0 + (uint64_t)(s * (P_STAGE_BYTES >> 4));
          pair_mma<BF16>(tmem_d, ad, bd, idesc, acc);
          acc = 1u;
          pair_mma<BF16>(tmem_d, ad + a_step, bd + b_step, idesc, 1u);
          pair_mma<BF16>(tmem_d, ad + 2 * a_step, bd + 2 * b_step, idesc, 1u);
          pair_mma<BF16>(tmem_d, ad + 3 * a_step, bd + 3 * b_step, idesc, 1u);
          mma2_commit_both(&empty[s]);
          if (++s == P_STAGES) { s = 0; ph ^= 1u; }
        }
        if (ok) mma2_commit_both(&acc_full[buf]);
      }
    }
  } else {
    // Epilogue: a quadrant's warps take its chunks of columns in turn.
    constexpr int U = epi_units<KIND>, COLS = 8 * U, STEP = epi_warps<KIND> / 4;
    const int quad = warp & 3, first = (warp - 2) >> 2;
    const uint32_t stg = smem_u32(staging + (warp - 2) * (P_STG_ALL / epi_warps<KIND>));
    const uint32_t acc_leader = map_to_cta(smem_u32(&acc_empty[0]), 0);
    int ti = 0;
    for (int t = pair; t < p.tiles; t += p.pairs, ++ti) {
      int tm, tn;
      find_tile(p, t, tm, tn);
      const int width = KIND == FFN_GATE ? p.bn >> 1 : p.bn;          // columns of the result
      const int m0 = tm * 2 * P_BM + (int)rank * P_BM + quad * 32, n0 = tn * width;
      const int chunks = m0 < p.M ? min(width / COLS, (p.N - n0 + COLS - 1) / COLS) : 0;
      const int buf = ti & 1;
      uint4 gx[4], ux[4];                        // FFN_GRAD: the stored gate and up of a chunk, the first one's requested before its sums are there
      if (KIND == FFN_GRAD && first < chunks) {
        fetch_chunk(gx, lane, dep(p.gate.p), p.gate.ld, m0, p.M, n0 + first * COLS, p.N);
        fetch_chunk(ux, lane, dep(p.up.p), p.up.ld, m0, p.M, n0 + first * COLS, p.N);
      }
      int good = 1;
      if (lane == 0) good = wait_or_abort(&acc_full[buf], (ti >> 1) & 1, abort_flag, p.err, 3) ? 1 : 0;
      good = __shfl_sync(0xffffffffu, good, 0);
      if (!good) break;
      tc_fence_after();
      const uint32_t tq = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * P_BN);
      with_activation(p.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
#pragma unroll 1
        for (int c = first; c < chunks; c += STEP) {
          const int nc = n0 + c * COLS;
          uint32_t w[4 * U], gw[4 * U], uw[4 * U];
          if constexpr (KIND == FFN_GATE) {
#pragma unroll
            for (int h = 0; h < COLS / 32; ++h) {
              float gv[32], uv[32];
              tmem_ld32_pair(tq + (uint32_t)(c * COLS + h * 32), tq + (uint32_t)(width + c * COLS + h * 32), gv, uv);
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float a0, a1, unused;
                activation<ACT, true>(gv[2 * i], a0, unused);
                activation<ACT, true>(gv[2 * i + 1], a1, unused);
                w[16 * h + i] = pack2<T>(a0 * uv[2 * i], a1 * uv[2 * i + 1]);
                gw[16 * h + i] = pack2<T>(gv[2 * i], gv[2 * i + 1]);
                uw[16 * h + i] = pack2<T>(uv[2 * i], uv[2 * i + 1]);
              }
            }
            put_chunk<U, 32>(w, stg, lane, p.d[0].p, p.d[0].ld, m0, p.M, nc, p.N, p.vec & 1);
            if (p.d[1].p) put_chunk<U, 32>(gw, stg, lane, p.d[1].p, p.d[1].ld, m0, p.M, nc, p.N, p.vec & 2);
            if (p.d[2].p) put_chunk<U, 32>(uw, stg, lane, p.d[2].p, p.d[2].ld, m0, p.M, nc, p.N, p.vec & 4);
          } else {
            turn_chunk(gx, stg, lane, gw);
            turn_chunk(ux, stg, lane, uw);
            if (c + STEP < chunks) {
              fetch_chunk(gx, lane, dep(p.gate.p), p.gate.ld, m0, p.M, nc + STEP * COLS, p.N);
              fetch_chunk(ux, lane, dep(p.up.p), p.up.ld, m0, p.M, nc + STEP * COLS, p.N);
            }
            float va[16], vb[16];
            tmem_ld16_pair(tq + (uint32_t)(c * COLS), tq + (uint32_t)(c * COLS + 16), va, vb);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float d0 = i < 8 ? va[2 * (i & 7)] : vb[2 * (i & 7)], d1 = i < 8 ? va[2 * (i & 7) + 1] : vb[2 * (i & 7) + 1];
              const float2 gt = unpack2<T>(gw[i]), up = unpack2<T>(uw[i]);
              float a0, a1, s0, s1;
              activation<ACT, true>(gt.x, a0, s0);
              activation<ACT, true>(gt.y, a1, s1);
              w[i] = pack2<T>(a0 * up.x, a1 * up.y);
              gw[i] = pack2<T>(d0 * up.x * s0, d1 * up.y * s1);
              uw[i] = pack2<T>(d0 * a0, d1 * a1);
            }
            put_chunk<U, 32>(w, stg, lane, p.d[0].p, p.d[0].ld, m0, p.M, nc, p.N, p.vec & 1);
            put_chunk<U, 32>(gw, stg, lane, p.d[1].p, p.d[1].ld, m0, p.M, nc, p.N, p.vec & 2);
            put_chunk<U, 32>(uw, stg, lane, p.d[2].p, p.d[2].ld, m0, p.M, nc, p.N, p.vec & 4);
          }
        }
      });
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_relaxed(acc_leader + (uint32_t)buf * 8u);
    }
  }
  tc_fence_before();
  cluster_sync_all();      // neither CTA leaves (or frees tensor memory) while the other may still use it
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
}

// ---- plain products: 256 x 512 tiles ------------------------------------------------------------
// With 256 x 256 tiles an SM's shared memory takes in 32 KB of operands and gives out 32 KB of them for every 512 cycles of its tensor core: all that
// it can move, and the tensor core is busy 81 % of the time (8192 x 8192 x 4096).  A tile of 512 columns, two products of 256 on the same rows of
// A, takes in 48 KB for 1024 cycles.  It fills the tensor memory, so the next tile waits until the epilogue warps have the sums: they take
// all of theirs to registers first, rounded to the type (128 words each), let the next tile start, and store after that.
// Tiles left over after the whole rounds of the pairs go as halves of 256 columns where those fit a single round.
// Fewer tiles than pairs and a long K (a weight gradient of narrow layers, the gradient of a few hundred rows): K is cut into slices whose sums go
// to the workspace in FP32 and are added, in order of the slices, by ffn_sum_kernel.
constexpr int W_STAGES = 4, W_STAGE_BYTES = 3 * P_A_BYTES, W_BN = 512;
constexpr int W_EPI_WARPS = 16, W_THREADS = 64 + 32 * W_EPI_WARPS, W_STG_BYTES = 32 * 64;
constexpr int W_SMEM = W_STAGES * W_STAGE_BYTES + W_EPI_WARPS * W_STG_BYTES + 1024 + 256;
static_assert(W_SMEM <= 232448, "more shared memory than a block can have");

struct WideProblem {
  int M, N, tiles_m, tiles_n, tiles;     // tiles of 256 x 512
  int kb0, kb, a_mn, b_mn, a_box3, b_box3, vec;
  int slices;                            // of K; of more than one, the sums are those of a slice and go to the workspace
  Out16 d;
};
// Work list: items 0 .. whole - 1 are tiles, then halves of the tiles from `whole` on; or (CUT) slices of tiles, those of a tile side by side.
template <int NP> struct WideParams { WideProblem p[NP]; int n, pairs, whole, items; float* ws; int* err; };
constexpr int W_SLOT = 256 * W_BN;       // floats of an item's sums: 32 x 32 pieces, 16 to a row of them, four columns of a piece's 32 rows side by side

struct WideItem { int k, m0, n0, halves, kb0, kb1; };
template <int NP, bool CUT>
__device__ __forceinline__ WideItem wide_item(const WideParams<NP>& g, int i) {
  WideItem w;
  const int rest = CUT ? -1 : i - g.whole;
  int t = rest < 0 ? i : g.whole + (rest >> 1);
  w.halves = rest < 0 ? 2 : 1;
  int k = 0;
  if (NP > 1)
    while (k + 1 < g.n && t >= g.p[k].tiles * (CUT ? g.p[k].slices : 1)) { t -= g.p[k].tiles * (CUT ? g.p[k].slices : 1); ++k; }
  const WideProblem& p = g.p[k];
  int slice = 0;
  if (CUT) { slice = t % p.slices; t /= p.slices; }
  const int strip = t / (P_PANELS * p.tiles_n), in = t - strip * P_PANELS * p.tiles_n;
  const int high = min(P_PANELS, p.tiles_m - strip * P_PANELS);
  w.k = k;
  w.m0 = (strip * P_PANELS + in % high) * 2 * P_BM;
  w.n0 = in / high * W_BN + (rest < 0 ? 0 : (rest & 1) * P_BN);
  if (w.n0 + P_BN >= p.N) w.halves = w.n0 < p.N ? 1 : 0;       // (a second half, or a left-over half, without columns)
  w.kb0 = CUT ? (int)((long long)p.kb * slice / p.slices) : 0;
  w.kb1 = CUT ? (int)((long long)p.kb * (slice + 1) / p.slices) : p.kb;
  return w;
}

template <class T, int NP, bool CUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(W_THREADS, 1)
ffn_wide_kernel(const __grid_constant__ WideMaps<NP> maps, const __grid_constant__ WideParams<NP> g) {
  constexpr bool BF16 = !__is_same(T, __half);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = smem + W_STAGES * W_STAGE_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + W_EPI_WARPS * W_STG_BYTES);
  uint64_t* empty = full + W_STAGES;
  uint64_t* acc_full = empty + W_STAGES;
  uint64_t* acc_empty = acc_full + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < W_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 2 * W_EPI_WARPS);
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

  if (warp == 0) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      const uint32_t full_leader = map_to_cta(smem_u32(&full[0]), 0);
      for (int i = pair; ok && i < g.items; i += g.pairs) {
        const WideItem w = wide_item<NP, CUT>(g, i);
        if (w.halves == 0) continue;
        const WideProblem& p = g.p[w.k];
        const bool a_mn = p.a_mn != 0, b_mn = p.b_mn != 0, a3 = p.a_box3 != 0, b3 = p.b_box3 != 0, two = w.halves == 2;
        const int m0 = w.m0 + (int)rank * P_BM, n0 = w.n0 + (int)rank * P_BM;
        const uint32_t pair_tx = 2u * P_A_BYTES * (1u + (uint32_t)w.halves);
#pragma unroll 1
        for (int part = 0; part < 2 && ok; ++part) {
          const int from = part ? p.kb0 : 0, end = min(w.kb1, part ? p.kb : p.kb0) - from;
          const CUtensorMap* const ma = &maps.m[w.k][2 * part];
          const CUtensorMap* const mb = ma + 1;
#pragma unroll 1
          for (int kb = max(w.kb0 - from, 0); kb < end; ++kb) {
            if (!wait_or_abort(&empty[s], ph ^ 1, abort_flag, g.err, 1)) { ok = false; break; }
            if (rank == 0) mbar_expect_tx(&full[s], pair_tx);
            const uint32_t bar = full_leader + (uint32_t)s * 8u;
            const int k0 = kb * P_BK;
            uint8_t* const sa = smem + s * W_STAGE_BYTES;
            uint8_t* const sb = sa + P_A_BYTES;
            if (!a_mn) {
              tma2_load_2d(sa, ma, k0, m0, bar);
            } else if (a3) {
              tma2_load_3d(sa, ma, 0, k0, m0 >> 6, bar);
            } else {
              tma2_load_2d(sa, ma, m0, k0, bar);
              tma2_load_2d(sa + 8192, ma, m0 + 64, k0, bar);
            }
            if (!b_mn) {
              tma2_load_2d(sb, mb, k0, n0, bar);
              if (two) tma2_load_2d(sb + P_A_BYTES, mb, k0, n0 + P_BN, bar);
            } else if (b3) {
              tma2_load_3d(sb, mb, 0, k0, n0 >> 6, bar);
              if (two) tma2_load_3d(sb + P_A_BYTES, mb, 0, k0, (n0 + P_BN) >> 6, bar);
            } else {
              tma2_load_2d(sb, mb, n0, k0, bar);
              tma2_load_2d(sb + 8192, mb, n0 + 64, k0, bar);
              if (two) {
                tma2_load_2d(sb + P_A_BYTES, mb, n0 + P_BN, k0, bar);
                tma2_load_2d(sb + P_A_BYTES + 8192, mb, n0 + P_BN + 64, k0, bar);
              }
            }
            if (++s == W_STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && lane == 0) {
      const uint32_t base = smem_u32(smem);
      int s = 0, ti = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int i = pair; ok && i < g.items; i += g.pairs) {
        const WideItem w = wide_item<NP, CUT>(g, i);
        if (w.halves == 0) continue;
        const WideProblem& p = g.p[w.k];
        const uint32_t idesc = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) |
                               ((uint32_t)(P_BN >> 3) << 17) | ((uint32_t)((2 * P_BM) >> 4) << 24);
        const uint64_t a_step = (p.a_mn ? 2048 : 32) >> 4, b_step = (p.b_mn ? 2048 : 32) >> 4;
        const uint64_t a0 = make_desc(base, p.a_mn ? 8192 : 16, 1024, 2);
        const uint64_t b0 = make_desc(base + P_A_BYTES, p.b_mn ? 8192 : 16, 1024, 2);
        if (!wait_or_abort(acc_empty, (ti & 1) ^ 1, abort_flag, g.err, 4)) break;
        tc_fence_after();
        uint32_t acc = 0u;
        const int kbs = w.kb1 - w.kb0;
        const bool two = w.halves == 2;
#pragma unroll 1
        for (int kb = 0; kb < kbs; ++kb) {
          if (!wait_or_abort(&full[s], ph, abort_flag, g.err, 2)) { ok = false; break; }
          tc_fence_after();
          const uint64_t ad = a0 + (uint64_t)(s * (W_STAGE_BYTES >> 4)), bd = b0 + (uint64_t)(s * (W_STAGE_BYTES >> 4));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t on = k ? 1u : acc;
            pair_mma<BF16>(tmem_base, ad + k * a_step, bd + k * b_step, idesc, on);
            if (two) pair_mma<BF16>(tmem_base + P_BN, ad + k * a_step, bd + (P_A_BYTES >> 4) + k * b_step, idesc, on);
          }
          acc = 1u;
          mma2_commit_both(&empty[s]);
          if (++s == W_STAGES) { s = 0; ph ^= 1u; }
        }
        if (ok) mma2_commit_both(acc_full);
        ++ti;
      }
    }
  } else {
    const int quad = warp & 3, first = (warp - 2) >> 2;
    const uint32_t stg = smem_u32(staging + (warp - 2) * W_STG_BYTES);
    const uint32_t acc_leader = map_to_cta(smem_u32(acc_empty), 0);
    const uint32_t tq = tmem_base + ((uint32_t)(quad * 32) << 16);
    int ti = 0;
    for (int i = pair; i < g.items; i += g.pairs) {
      const WideItem w = wide_item<NP, CUT>(g, i);
      if (w.halves == 0) continue;
      const WideProblem& p = g.p[w.k];
      const int m0 = w.m0 + (int)rank * P_BM + quad * 32;
      const int chunks = m0 < p.M ? min(4 * w.halves, (p.N - w.n0 + 63) / 64) : 0;      // of 64 columns; this warp's are first and first + 4
      int good = 1;
      if (lane == 0) good = wait_or_abort(acc_full, ti & 1, abort_flag, g.err, 3) ? 1 : 0;
      good = __shfl_sync(0xffffffffu, good, 0);
      if (!good) break;
      ++ti;
      tc_fence_after();
      if (CUT && p.slices > 1) {
        float* const slot = g.ws + (int64_t)i * W_SLOT + ((int)rank * 4 + quad) * 16 * 1024 + lane * 4;
#pragma unroll 1
        for (int c = 2 * first; c < 2 * chunks; c += c & 1 ? 7 : 1) {
          float v[32];
          tmem_ld32(tq + (uint32_t)(c * 32), v);
#pragma unroll
          for (int q = 0; q < 8; ++q) __stcg(reinterpret_cast<float4*>(slot + c * 1024 + q * 128), make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(acc_leader);
        continue;
      }
      uint32_t x[2][32];
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (4 * c + first < chunks) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float a[16], b[16];
            const uint32_t at = tq + (uint32_t)((4 * c + first) * 64 + 32 * h);
            tmem_ld16_pair(at, at + 16u, a, b);
#pragma unroll
            for (int q = 0; q < 8; ++q) { x[c][16 * h + q] = pack2<T>(a[2 * q], a[2 * q + 1]); x[c][16 * h + 8 + q] = pack2<T>(b[2 * q], b[2 * q + 1]); }
          }
        }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_relaxed(acc_leader);
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (4 * c + first < chunks) {
          const int n = w.n0 + (4 * c + first) * 64;
          if (p.vec && n + 64 <= p.N) {                  // (rows of 64 bytes are as good as rows of 128 where they are whole, and take fewer steps)
            put_whole(x[c], stg, lane, p.d.p, p.d.ld, m0, p.M, n);
            put_whole(x[c] + 16, stg, lane, p.d.p, p.d.ld, m0, p.M, n + 32);
          } else {
            put_chunk<8, 16>(x[c], stg, lane, p.d.p, p.d.ld, m0, p.M, n, p.N, p.vec);
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

// The sums of the slices of a tile, added in their order, to the result: blockIdx.x = 32 columns of a tile, warp = 32 rows.
template <class T, int NP>
__global__ void __launch_bounds__(256) ffn_sum_kernel(const __grid_constant__ WideParams<NP> g) {
  __shared__ __align__(16) uint8_t staging[8][32 * 64];
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int t = blockIdx.x / 16, item = 0, k = 0;
  const int c = blockIdx.x % 16;
  while (k + 1 < g.n && (g.p[k].slices == 1 || t >= g.p[k].tiles)) {
    if (g.p[k].slices > 1) t -= g.p[k].tiles;
    item += g.p[k].tiles * g.p[k].slices;
    ++k;
  }
  const WideProblem& p = g.p[k];
  item += t * p.slices;
  const WideItem w = wide_item<NP, true>(g, item);
  const int m0 = w.m0 + warp * 32, n0 = w.n0 + c * 32;
  if (m0 >= p.M || n0 >= p.N) return;
  const float* const from = dep(g.ws) + (int64_t)item * W_SLOT + (warp * 16 + c) * 1024 + lane * 4;
  float v[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) v[e] = 0.f;
#pragma unroll 2
  for (int s = 0; s < p.slices; ++s) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(from + (int64_t)s * W_SLOT + q * 128));
      v[4 * q] += x.x; v[4 * q + 1] += x.y; v[4 * q + 2] += x.z; v[4 * q + 3] += x.w;
    }
  }
  uint32_t o[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) o[e] = pack2<T>(v[2 * e], v[2 * e + 1]);
  put_chunk<4, 32>(o, smem_u32(staging[warp]), lane, p.d.p, p.d.ld, m0, p.M, n0, p.N, p.vec);
}

// ---- host side ---------------------------------------------------------------------------------
// Maps of a plain product's operands, those that it has.
bool encode_problem(CUtensorMap* maps, const FfnGemm& g, bool a_box3, bool b_box3, bool bf16) {
  for (int s = 0; s < (g.K[1] > 0 ? 2 : 1); ++s) {
    const int K = g.K[s];
    const auto encode = [&](CUtensorMap* to, const Mat16& mat, bool mn, bool box3, int MN) {
      return !mn ? make_map16(to, mat, MN, K, P_BM, bf16) : box3 ? make_map16_chunks(to, mat, K, MN, P_BM / 64, bf16) : make_map16(to, mat, K, MN, 64, bf16);
    };
    if (!encode(&maps[2 * s], g.A[s], g.a_mn, a_box3, g.M) || !encode(&maps[2 * s + 1], g.B[s], g.b_mn, b_box3, g.N)) return false;
  }
  return true;
}

// Width of the tiles: that of the fewer rounds, a round of narrow ones taking a little over half the time of one of wide ones.
long long pair_rounds(int kind, int M, int N, int bn) {
  const int width = kind == FFN_GATE ? bn / 2 : bn, pairs = num_sms() / 2;
  return ((long long)((M + 255) / 256) * ((N + width - 1) / width) + pairs - 1) / pairs;
}
int pair_width(int kind, int M, int N) { return pair_rounds(kind, M, N, 128) * 5 < pair_rounds(kind, M, N, 256) * 8 ? 128 : 256; }

template <int KIND, class T>
cudaError_t launch_pair_as(int act, const FfnGemm& g, int* err, cudaStream_t st) {
  constexpr bool BF16 = !__is_same(T, __half);
  static std::atomic<signed char> ready[64];
  auto* const kernel = ffn_pair_kernel<KIND, T>;
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, P_SMEM) == cudaSuccess; }))
    return cudaErrorInvalidDevice;
  PairMaps maps;
  PairParams p = {};
  const int pairs = num_sms() / 2, bn = pair_width(KIND, g.M, g.N), width = KIND == FFN_GATE ? bn / 2 : bn;
  p.M = g.M; p.N = g.N; p.bn = bn;
  p.tiles_m = (p.M + 255) / 256; p.tiles_n = (p.N + width - 1) / width;
  const long long tiles = (long long)p.tiles_m * p.tiles_n;
  if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
  p.tiles = (int)tiles;
  p.pairs = p.tiles < pairs ? p.tiles : pairs;
  p.kb = (g.K[0] + P_BK - 1) / P_BK;
  p.b_box3 = KIND == FFN_GRAD && p.N % 64 == 0;
  for (int k = 0; k < 3; ++k) p.d[k] = g.d[k];
  p.gate = g.gate; p.up = g.up;
  p.vec = vec16(p.d[0]) | vec16(p.d[1]) << 1 | vec16(p.d[2]) << 2;
  p.act = act; p.err = err;
  const auto rows_of_b = [&](CUtensorMap* m, const Mat16& b) { return make_map16(m, b, g.N, g.K[0], bn / 2, BF16); };
  bool ok = make_map16(&maps.m[0], g.A[0], g.M, g.K[0], P_BM, BF16);
  if constexpr (KIND == FFN_GATE) ok = ok && rows_of_b(&maps.m[1], g.B[0]) && rows_of_b(&maps.m[2], g.B[1]);
  else ok = ok && (p.b_box3 ? make_map16_chunks(&maps.m[1], g.B[0], g.K[0], g.N, bn / 128, BF16) : make_map16(&maps.m[1], g.B[0], g.K[0], g.N, 64, BF16));
  if (!ok) return cudaErrorInvalidValue;
  return launch_pdl(kernel, 2 * p.pairs, pair_threads<KIND>, P_SMEM, st, maps, p);
}

// How a group of products is cut: slices of K for each (all 1: none), and the items that makes.  Estimated times, in us: a k-block of a 256 x 512 tile 0.36
// (a pair by itself as well: it waits for its loads), an item 4 more; a list takes as long as its longest item, its share of all, or its
// bytes at 5 TB/s; slices cost a second kernel, 6, and their sums' way out and back at 4 TB/s.
struct WidePlan { int slices[kFfnGroup]; int items; bool cut; double us; };
WidePlan plan_wide(const FfnGemm* g, int n) {
  const int pairs = num_sms() / 2;
  long long tiles = 0, work = 0;
  double bytes_us = 0.0;
  int kb[kFfnGroup], tl[kFfnGroup], longest = 0;
  WidePlan best{};
  for (int i = 0; i < n; ++i) {
    const long long t = (long long)((g[i].M + 255) / 256) * ((g[i].N + W_BN - 1) / W_BN);
    kb[i] = (g[i].K[0] + P_BK - 1) / P_BK + (g[i].K[1] + P_BK - 1) / P_BK;
    tl[i] = (int)(t < 0x1fffffff ? t : 0x1fffffff);
    tiles += t; work += t * kb[i];
    longest = kb[i] > longest ? kb[i] : longest;
    bytes_us += (((double)g[i].M + g[i].N) * ((double)g[i].K[0] + g[i].K[1]) + (double)g[i].M * g[i].N) * 2.0 / 5e6;
    best.slices[i] = 1;
  }
  const auto list_us = [&](int most, long long items) {
    const double one = most * 0.36 + 4.0, share = (work * 0.36 + items * 4.0) / pairs * (items > pairs ? 1.15 : 1.0);
    const double list = one > share ? one : share;
    return list > bytes_us ? list : bytes_us;
  };
  double best_us = list_us(longest, tiles);
  best.us = best_us;
  if (tiles >= 4 * pairs) return best;
  for (int len = longest; len >= 4; len = len > 32 ? len * 7 / 8 : len - 1) {
    WidePlan p{};
    long long items = 0, cut = 0;
    int most = 0;
    for (int i = 0; i < n; ++i) {
      p.slices[i] = (kb[i] + len - 1) / len;
      items += (long long)tl[i] * p.slices[i];
      if (p.slices[i] > 1) cut += (long long)tl[i] * p.slices[i];
      const int each = (kb[i] + p.slices[i] - 1) / p.slices[i];
      most = each > most ? each : most;
    }
    if (items > 8 * pairs) break;
    const double us = list_us(most, items) + 6.0 + cut * (W_SLOT * 4.0 * 2.0 / 4e6);
    if (cut > 0 && us < 0.9 * best_us) { best_us = us; p.items = (int)items; p.cut = true; p.us = us; best = p; }
  }
  return best;
}

template <class T, int NP, bool CUT>
cudaError_t launch_wide_as(const FfnGemm* g, int n, const WidePlan& plan, void* ws, int* err, cudaStream_t st) {
  constexpr bool BF16 = !__is_same(T, __half);
  static std::atomic<signed char> ready[64];
  auto* const kernel = ffn_wide_kernel<T, NP, CUT>;
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W_SMEM) == cudaSuccess; }))
    return cudaErrorInvalidDevice;
  WideMaps<NP> maps;
  WideParams<NP> q = {};
  q.n = n; q.err = err; q.ws = (float*)ws;
  long long tiles = 0, summed = 0;
  for (int i = 0; i < n; ++i) {
    WideProblem& p = q.p[i];
    p.M = g[i].M; p.N = g[i].N;
    p.tiles_m = (p.M + 255) / 256; p.tiles_n = (p.N + W_BN - 1) / W_BN;
    tiles += (long long)p.tiles_m * p.tiles_n;
    if (tiles > 0x1fffffff) return cudaErrorInvalidValue;
    p.tiles = p.tiles_m * p.tiles_n;
    p.slices = plan.slices[i];
    if (p.slices > 1) summed += p.tiles;
    p.kb0 = (g[i].K[0] + P_BK - 1) / P_BK; p.kb = p.kb0 + (g[i].K[1] + P_BK - 1) / P_BK;
    p.a_mn = g[i].a_mn; p.b_mn = g[i].b_mn;
    p.a_box3 = p.a_mn && p.M % 64 == 0; p.b_box3 = p.b_mn && p.N % 64 == 0;
    p.d = g[i].d[0];
    p.vec = vec16(p.d);
    if (!encode_problem(maps.m[i], g[i], p.a_box3, p.b_box3, BF16)) return cudaErrorInvalidValue;
  }
  const int pairs = num_sms() / 2, rem = (int)(tiles % pairs);
  q.whole = (int)(2 * rem <= pairs ? tiles - rem : tiles);
  q.items = CUT ? plan.items : (int)(q.whole + 2 * (tiles - q.whole));
  q.pairs = q.items < pairs ? q.items : pairs;
  cudaError_t e = launch_pdl(kernel, 2 * q.pairs, W_THREADS, W_SMEM, st, maps, q);
  if constexpr (CUT)
    if (e == cudaSuccess) e = launch_pdl(ffn_sum_kernel<T, NP>, (int)summed * 16, 256, 0, st, q);
  return e;
}

}  // namespace

// 8 us for a launch and the last round's epilogue; a k-block 0.40 of a wide tile and 0.28 of a narrow one; an epilogue 7, beside the next round's products.
double ffn_pair_us(FfnKind kind, int M, int N, int K) {
  const int bn = pair_width(kind, M, N), kb = (K + P_BK - 1) / P_BK;
  const double round = kb * (bn == 256 ? 0.40 : 0.28);
  return 8.0 + round + (pair_rounds(kind, M, N, bn) - 1) * (round > 7.0 ? round : 7.0);
}
double ffn_pair_list_us(const FfnGemm* g, int n) { return n > 0 ? plan_wide(g, n).us : 0.0; }

int64_t ffn_pair_workspace(const FfnGemm* g, int n) {
  const WidePlan p = plan_wide(g, n);
  return p.cut ? (int64_t)p.items * W_SLOT * 4 : 0;
}

cudaError_t launch_ffn_pair(FfnKind kind, bool bf16, int act, const FfnGemm* g, int n, void* ws, int* err, cudaStream_t st) {
  if (kind == FFN_GATE) return bf16 ? launch_pair_as<FFN_GATE, __nv_bfloat16>(act, *g, err, st) : launch_pair_as<FFN_GATE, __half>(act, *g, err, st);
  if (kind == FFN_GRAD) return bf16 ? launch_pair_as<FFN_GRAD, __nv_bfloat16>(act, *g, err, st) : launch_pair_as<FFN_GRAD, __half>(act, *g, err, st);
  const WidePlan plan = plan_wide(g, n);
  const auto launch = [&](auto t) {
    using T = decltype(t);
    if (n == 1) return plan.cut ? launch_wide_as<T, 1, true>(g, n, plan, ws, err, st) : launch_wide_as<T, 1, false>(g, n, plan, ws, err, st);
    return plan.cut ? launch_wide_as<T, kFfnGroup, true>(g, n, plan, ws, err, st) : launch_wide_as<T, kFfnGroup, false>(g, n, plan, ws, err, st);
  };
  return bf16 ? launch(__nv_bfloat16()) : launch(__half());
}

}  // namespace gn
