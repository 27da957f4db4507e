// Products of 16-bit matrices over a mixture's experts: CTA pairs (tcgen05.mma.cta_group::2, operands by TMA, accumulators in tensor memory) on tiles of 256 x 256 (GROUP_GRAD: 128)
// elements, the tiles of all experts dealt to the pairs in turn.
//
// The rows of the left operand are slots: an expert's tokens side by side from a multiple of 64 on (expert_kernels.h).  A tile has up to 256 slots of one expert;
// what it reads of the next expert's is never stored.  How many tiles there are only the device knows: a persistent pair
// walks the plan's list, all columns of a tile of slots before the next, so that the pairs at work together share an expert's weights.
// In GROUP_WEIGHT the slots are the terms: whole blocks of 64, the empty ones among them zero on both sides, and an expert without tokens has a gradient of zero.
//
// Weights are three-dimensional to TMA (expert, row, column), so that a box past the edge of an expert's matrix reads zeros, not its neighbour.
// Warp roles as in gemm_pair16.cu: warp 0 TMA producer, warp 1 of the leader CTA issues the products, warps 2.. are the epilogue, beside the next tile's
// products (two accumulators of 256 columns; GROUP_GRAD: four of 128).  What belongs to the pairs of token and choice (gate, up, the products' results) is read and written
// in the pairs' order, a row's place found by a shuffle from the lane that has the row.  Results of GROUP_DOWN and GROUP_DX stay FP32 until a token's k rows are added.
//
// GROUP_GATE: the B tile is 128 rows of the gate's weights and the same 128 of the up projection's.  h, dgate and dup are rounded to the type: they are operands of the
// next product.  (Rows of GROUP_DOWN and GROUP_DX in the type would save 270 MB at 8192 tokens, 4 choices and 2048 columns, and make the error of y and dx 1.7 times
// that of their own rounding instead of 1.4.)
// GROUP_GRAD: dweight, the sum of q act(gate) up, is an FP32 result.  The tensor core cuts off what does not fit when it adds to a sum, always towards zero: 1e-6 of q for each thousand terms.  So its tiles have
// 128 columns and four accumulators take turns: a sum is taken out after 256 to 512 terms and added to registers, a thread's 64 columns, in FP32.  A quarter of the terms at a time lets a whole tile of products run
// beside the epilogue of the one before.  8192 tokens, 4 of 32 experts, 2048 x 1024: 211 us, where tiles of 256 columns and sums of all terms took 172 (and sums of 256 terms a quarter
// more than 211); dweight is 0.5e-6 off in BF16 and 0.66e-6 in FP16, where it was 2.1e-6 and 2.5e-6.  Its sums over a thread's columns are added in order elsewhere.
// Bound, with all pairs at work, by what L2 gives to shared memory: 32 KB a CTA for 64 terms, 0.37 us (13 TB/s), where the products take 0.27; and by the power cap.
// 8192 tokens, 4 of 64 experts, 2048 x 1408: gate 361 us (1047 TFLOP/s, a fifth of the rows padding), with Wd 185; 4 of 32, 2048 x 1024: gate's gradient 211 (11 TB/s from L2), dx 216, three
// weight gradients 334.  16 tokens, 4 of 32 experts: 48 and 28, the weights at 4.7 TB/s (224 tiles are 3.03 rounds of the pairs).
// Every wait is bounded; a role that gives up leaves a code in *err and the CTA drains.
#include "expert_kernels.h"
#include "pair_common.cuh"

namespace gn {
namespace {

constexpr int G_BM = 128, G_BK = 64, G_STG_ALL = 32 * 1024;
// A pair's tile has BN columns; each CTA has 128 rows of A and half of B's columns in a stage.  BUFS accumulators share tensor memory's 512 columns.
template <int KIND> struct GroupTile {
  static constexpr int BN = KIND == GROUP_GRAD ? 128 : 256, STAGES = KIND == GROUP_GRAD ? 8 : 6, BUFS = 512 / BN;
  static constexpr int A_BYTES = G_BM * G_BK * 2, STAGE_BYTES = A_BYTES + BN / 2 * G_BK * 2;
};
constexpr int G_RING = 192 * 1024, G_SMEM = G_RING + G_STG_ALL + 1024 + 256;
static_assert(GroupTile<GROUP_GRAD>::STAGES * GroupTile<GROUP_GRAD>::STAGE_BYTES == G_RING && GroupTile<GROUP_GATE>::STAGES * GroupTile<GROUP_GATE>::STAGE_BYTES == G_RING, "the stages fill the ring");
static_assert(G_SMEM <= 232448, "more shared memory than a block can have");
static_assert(kGroupHeight == 2 * G_BM, "a tile of slots is a pair's rows");
// Epilogue warps: with 16 in GROUP_GRAD a thread has 96 registers and keeps 1.3 KB of its values in local memory, more than the L1 has beside the stages (203 us where eight took 172, tiles of 256 columns).
constexpr int G_WARPS = 8, G_THREADS = 64 + 32 * G_WARPS;
constexpr int G_GRADS = 3;

struct GroupGrad { int M, N, tiles_m, tiles_n, first, vec; Grads16 d; };
struct GroupParams {
  int N, tiles_n, kb0, kb, chunk, act, pairs;    // chunk: blocks of terms after which a sum of GROUP_GRAD leaves tensor memory
  int vec_gate, vec_up;
  const ExpertTile* tiles; const int* n_tiles;
  const int *start, *count, *pair_of;
  Out16 d, dgate, dup, gate_out, up_out;
  FfnOut rows;
  Mat16 gate, up;
  const float* weight; float* parts; int n_parts;
  GroupGrad grad[G_GRADS]; int n_grads, items;
  int* err;
};
template <int KIND> constexpr int group_maps = KIND == GROUP_GATE ? 3 : KIND == GROUP_DX ? 4 : KIND == GROUP_WEIGHT ? 2 * G_GRADS : 2;
template <int KIND> struct GroupMaps { CUtensorMap m[group_maps<KIND>]; };        // A, B (GROUP_GATE: Wg, Wu); A0, B0, A1, B1; left, right of each gradient

// What a warp of GROUP_GRAD's epilogue has of an item: its first slot, rows (empty slots among them), first column and how many times 32 of them; the pair of this lane's row (-1: none) and
// that one's weight.
struct GradRows { int slot, rows, n0, pieces, pair; float share; };
// What a pair works on: rows from `slot` on (GROUP_WEIGHT: rows m0 and columns n0 of a gradient, terms from `slot` on).
struct GroupItem { int expert, slot, rows, padded, m0, n0, kb, grad; };
template <int KIND>
__device__ __forceinline__ GroupItem group_item(const GroupParams& p, int i) {
  GroupItem w;
  if constexpr (KIND == GROUP_WEIGHT) {
    w.grad = 0;
    while (w.grad + 1 < p.n_grads && i >= p.grad[w.grad + 1].first) ++w.grad;
    const GroupGrad& g = p.grad[w.grad];
    const int each = g.tiles_m * g.tiles_n, in = i - g.first;
    w.expert = in / each;
    const int t = in - w.expert * each;
    w.m0 = t / g.tiles_n * 2 * G_BM; w.n0 = t % g.tiles_n * GroupTile<KIND>::BN;
    w.slot = p.start[w.expert];
    w.kb = (p.count[w.expert] + G_BK - 1) / G_BK;
    w.rows = w.padded = 0;
  } else {
    const int t = i / p.tiles_n;
    const int4 e = *reinterpret_cast<const int4*>(p.tiles + t);
    w.expert = e.x; w.slot = e.y; w.rows = e.z; w.padded = e.w;
    w.n0 = (i - t * p.tiles_n) * (KIND == GROUP_GATE ? GroupTile<KIND>::BN / 2 : GroupTile<KIND>::BN);
    w.m0 = 0; w.kb = p.kb; w.grad = 0;
  }
  return w;
}

__device__ __forceinline__ GroupItem uniform_item(GroupItem w) {
  w.expert = uniform(w.expert); w.slot = uniform(w.slot); w.m0 = uniform(w.m0); w.n0 = uniform(w.n0); w.kb = uniform(w.kb); w.grad = uniform(w.grad);
  return w;
}

template <int KIND, class T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(G_THREADS, 1)
group_kernel(const __grid_constant__ GroupMaps<KIND> maps, const __grid_constant__ GroupParams p) {
  constexpr bool A_MN = KIND == GROUP_WEIGHT, B_MN = KIND == GROUP_GRAD || KIND == GROUP_DX || KIND == GROUP_WEIGHT;
  using Tile = GroupTile<KIND>;
  constexpr int EPI = G_WARPS, BN = Tile::BN, STAGES = Tile::STAGES, STAGE_BYTES = Tile::STAGE_BYTES, BUFS = Tile::BUFS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* staging = smem + G_RING;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + G_STG_ALL);
  uint64_t* empty = full + STAGES;
  uint64_t* acc_full = empty + STAGES;     // [BUFS]
  uint64_t* acc_empty = acc_full + BUFS;   // [BUFS]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + BUFS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int b = 0; b < BUFS; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 2 * EPI); }
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
      const GroupItem w = uniform_item(group_item<KIND>(p, i));
      const int m0 = (KIND == GROUP_WEIGHT ? w.m0 : w.slot) + (int)rank * G_BM, n0 = KIND == GROUP_GATE ? w.n0 : w.n0 + (int)rank * (BN / 2);
#pragma unroll 1
      for (int kb = 0; kb < w.kb; ++kb) {
        if (!warp_wait_or_abort(&empty[s], ph ^ 1, abort_flag, p.err, 1)) { ok = false; break; }
        if (elect_one()) {
          if (rank == 0) mbar_expect_tx(&full[s], 2u * STAGE_BYTES);
          const uint32_t bar = full_leader + (uint32_t)s * 8u;
          uint8_t* const sa = smem + s * STAGE_BYTES;
          uint8_t* const sb = sa + Tile::A_BYTES;
          if constexpr (KIND == GROUP_WEIGHT) {
            const CUtensorMap* const ma = &maps.m[2 * w.grad];
            const int k0 = w.slot + kb * G_BK;
            tma2_load_2d(sa, ma, m0, k0, bar);
            tma2_load_2d(sa + 8192, ma, m0 + 64, k0, bar);
            tma2_load_2d(sb, ma + 1, n0, k0, bar);
            tma2_load_2d(sb + 8192, ma + 1, n0 + 64, k0, bar);
          } else {
            const int part = KIND == GROUP_DX && kb >= p.kb0 ? 1 : 0, k0 = (part ? kb - p.kb0 : kb) * G_BK;
            tma2_load_2d(sa, &maps.m[2 * part], k0, m0, bar);
            const CUtensorMap* const mb = &maps.m[KIND == GROUP_GATE ? (rank ? 2 : 1) : 2 * part + 1];
            if constexpr (!B_MN) {
              tma2_load_3d(sb, mb, k0, n0, w.expert, bar);
            } else {
              tma2_load_3d(sb, mb, n0, k0, w.expert, bar);
              if constexpr (BN == 256) tma2_load_3d(sb + 8192, mb, n0 + 64, k0, w.expert, bar);
            }
          }
        }
        if (++s == STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      constexpr bool BF16 = !__is_same(T, __half);
      const uint32_t base = smem_u32(smem);
      const uint32_t idesc = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) |
                             ((uint32_t)((2 * G_BM) >> 4) << 24);
      constexpr uint64_t a_step = (A_MN ? 2048 : 32) >> 4, b_step = (B_MN ? 2048 : 32) >> 4;
      const uint64_t a0 = make_desc(base, A_MN ? 8192 : 16, 1024, 2);
      const uint64_t b0 = make_desc(base + Tile::A_BYTES, B_MN ? 8192 : 16, 1024, 2);
      int s = 0, ci = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int i = pair; ok && i < items; i += p.pairs) {
        const GroupItem w = uniform_item(group_item<KIND>(p, i));
        const int chunk = KIND == GROUP_GRAD ? p.chunk : w.kb;
#pragma unroll 1
        for (int k0 = 0; k0 < w.kb && ok; k0 += chunk, ++ci) {
          const int buf = ci % BUFS;
          if (!warp_wait_or_abort(&acc_empty[buf], ((ci / BUFS) & 1) ^ 1, abort_flag, p.err, 4)) { ok = false; break; }
          tc_fence_after();
          const uint32_t tmem_d = tmem_base + (uint32_t)(buf * BN);
          uint32_t acc = 0u;
          const int end = KIND == GROUP_GRAD ? min(k0 + chunk, w.kb) : w.kb;
#pragma unroll 1
          for (int kb = k0; kb < end; ++kb) {
            if (!warp_wait_or_abort(&full[s], ph, abort_flag, p.err, 2)) { ok = false; break; }
            tc_fence_after();
            const uint64_t ad = a0 + (uint64_t)(s * (STAGE_BYTES >> 4)), bd = b0 + (uint64_t)(s * (STAGE_BYTES >> 4));
            if (elect_one()) {
              pair_mma<BF16>(tmem_d, ad, bd, idesc, acc);
              pair_mma<BF16>(tmem_d, ad + a_step, bd + b_step, idesc, 1u);
              pair_mma<BF16>(tmem_d, ad + 2 * a_step, bd + 2 * b_step, idesc, 1u);
              pair_mma<BF16>(tmem_d, ad + 3 * a_step, bd + 3 * b_step, idesc, 1u);
              mma2_commit_both(&empty[s]);
            }
            acc = 1u;
            if (++s == STAGES) { s = 0; ph ^= 1u; }
          }
          if (ok && elect_one()) mma2_commit_both(&acc_full[buf]);
        }
      }
    }
  } else {
    // Epilogue: a quadrant's warps take its chunks of columns in turn, or (GROUP_GRAD) half of its columns each.
    constexpr bool ROWS = KIND == GROUP_DOWN || KIND == GROUP_DX;
    constexpr int U = KIND == GROUP_GRAD ? 4 : 8, COLS = ROWS ? 32 : 8 * U, STEP = EPI / 4;
    const int quad = warp & 3, first = (warp - 2) >> 2;
    const uint32_t stg = smem_u32(staging + (warp - 2) * (G_STG_ALL / EPI));
    const uint32_t acc_leader = map_to_cta(smem_u32(&acc_empty[0]), 0);
    const int* const pair_of = dep(p.pair_of);
    const float* const weight = dep(p.weight);
    const uint32_t tq0 = tmem_base + ((uint32_t)(quad * 32) << 16);
    int ci = 0;
    // Sums of accumulator ci are there; they have been read.
    const auto begin = [&](int buf) {
      int good = 1;
      if (lane == 0) good = wait_or_abort(&acc_full[buf], (ci / BUFS) & 1, abort_flag, p.err, 3) ? 1 : 0;
      good = __shfl_sync(0xffffffffu, good, 0);
      tc_fence_after();
      return good != 0;
    };
    const auto end = [&](int buf) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_relaxed(acc_leader + (uint32_t)buf * 8u);
      ++ci;
    };
    const int r0 = (int)rank * G_BM + quad * 32;                      // this warp's rows of a tile
    [[maybe_unused]] uint4 gx[4], ux[4];                              // GROUP_GRAD: 32 columns of the stored gate and up
    [[maybe_unused]] const auto rows_of = [&](const GroupItem& w) {
      GradRows g{w.slot, w.padded, w.n0 + first * 64, 0, -1, 0.f};
      g.pieces = r0 < w.padded ? max(0, min(2, (p.N - g.n0 + 31) / 32)) : 0;
      if (r0 + lane < w.rows) { g.pair = pair_of[w.slot + r0 + lane]; g.share = weight[g.pair]; }
      return g;
    };
    [[maybe_unused]] const auto request = [&](const GradRows& g, int c) {
      if (g.pieces == 0) return;
      const auto row_of = [&](int r) { return __shfl_sync(0xffffffffu, g.pair, r); };
      fetch_rows(gx, lane, dep(p.gate.p), p.gate.ld, row_of, g.n0 + c * 32, p.N);
      fetch_rows(ux, lane, dep(p.up.p), p.up.ld, row_of, g.n0 + c * 32, p.N);
    };
    [[maybe_unused]] GradRows next{};
    if constexpr (KIND == GROUP_GRAD) {
      if (pair < items) next = rows_of(group_item<KIND>(p, pair));
      request(next, 0);
    }
    bool ok = true;
    for (int i = pair; ok && i < items; i += p.pairs) {
      if constexpr (KIND == GROUP_GRAD) {
        // (this item's rows have been looked up, and the stored gate and up of its first 32 columns requested, beside the item before)
        const GradRows now = next;
        const int j = i + p.pairs;
        next = GradRows{};
        if (j < items) next = rows_of(group_item<KIND>(p, j));
        float x[32], y[32];          // q
#pragma unroll
        for (int q = 0; q < 32; ++q) x[q] = y[q] = 0.f;
#pragma unroll 1
        for (int k0 = 0; k0 < p.kb; k0 += p.chunk) {
          const int buf = ci % BUFS;
          if (!begin(buf)) { ok = false; break; }
          float a[32], b[32];
          tmem_ld32_pair(tq0 + (uint32_t)(buf * BN + first * 64), tq0 + (uint32_t)(buf * BN + first * 64 + 32), a, b);
          end(buf);
#pragma unroll
          for (int q = 0; q < 32; ++q) { x[q] += a[q]; y[q] += b[q]; }
        }
        if (!ok) break;
        const auto slot_row = [&](int r) { return r0 + r < now.rows ? now.slot + r0 + r : -1; };
        float sum = 0.f;
        if (now.pieces == 0) request(next, 0);
        with_activation(p.act, [&](auto act) {
          constexpr int ACT = decltype(act)::value;
#pragma unroll 1
          for (int c = 0; c < now.pieces; ++c) {
            const int n = now.n0 + c * 32;
            uint32_t o[16], gw[16], uw[16];
            turn_chunk(gx, stg, lane, gw);
            turn_chunk(ux, stg, lane, uw);
            if (c + 1 < now.pieces) request(now, c + 1);
            else request(next, 0);
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              float d0 = x[2 * q], d1 = x[2 * q + 1];
              if (now.pair < 0) d0 = d1 = 0.f;                        // (an empty slot: zero, whatever the weights are)
              const float2 gt = unpack2<T>(gw[q]), up = unpack2<T>(uw[q]);
              float a0, a1, s0, s1;
              activation<ACT, true>(gt.x, a0, s0);
              activation<ACT, true>(gt.y, a1, s1);
              const float h0 = a0 * up.x, h1 = a1 * up.y;
              // (past the last column q, gate and up are zero)
              sum = fmaf(d0, h0, sum); sum = fmaf(d1, h1, sum);
              d0 *= now.share; d1 *= now.share;
              o[q] = pack2<T>(now.share * h0, now.share * h1);
              gw[q] = pack2<T>(d0 * up.x * s0, d1 * up.y * s1);
              uw[q] = pack2<T>(d0 * a0, d1 * a1);
              x[2 * q] = y[2 * q]; x[2 * q + 1] = y[2 * q + 1];
            }
            put_rows<U>(o, stg, lane, p.d.p, p.d.ld, slot_row, n, p.N, true);
            put_rows<U>(gw, stg, lane, p.dgate.p, p.dgate.ld, slot_row, n, p.N, true);
            put_rows<U>(uw, stg, lane, p.dup.p, p.dup.ld, slot_row, n, p.N, true);
          }
        });
        if (now.pair >= 0) p.parts[(int64_t)(now.slot + r0 + lane) * p.n_parts + now.n0 / 64] = sum;
      } else {
        const GroupItem w = group_item<KIND>(p, i);
        constexpr int WIDTH = KIND == GROUP_GATE ? BN / 2 : BN;         // columns of the result
        const int N = KIND == GROUP_WEIGHT ? p.grad[w.grad].N : p.N;
        const int rows = KIND == GROUP_WEIGHT ? p.grad[w.grad].M - w.m0 : w.rows;     // of the tile
        // This lane's row: its pair.
        const int my_pair = KIND != GROUP_WEIGHT && r0 + lane < rows ? pair_of[w.slot + r0 + lane] : -1;
        [[maybe_unused]] const auto pair_row = [&](int r) { return __shfl_sync(0xffffffffu, my_pair, r); };
        [[maybe_unused]] const auto slot_row = [&](int r) { return r0 + r < rows ? w.slot + r0 + r : -1; };
        const int chunks = r0 < rows ? min(WIDTH / COLS, (N - w.n0 + COLS - 1) / COLS) : 0;
        const bool none = KIND == GROUP_WEIGHT && w.kb == 0;
        const int buf = ci % BUFS;
        if (!none && !begin(buf)) break;
        const uint32_t tq = tq0 + (uint32_t)(buf * BN);
        const auto whole = [&](auto act) {
          [[maybe_unused]] constexpr int ACT = decltype(act)::value;
#pragma unroll 1
          for (int c = first; c < chunks; c += STEP) {
            const int nc = w.n0 + c * COLS;
            uint32_t o[4 * U];
            if constexpr (KIND == GROUP_GATE) {
              uint32_t gw[4 * U], uw[4 * U];
#pragma unroll
              for (int h = 0; h < COLS / 32; ++h) {
                float gv[32], uv[32];
                tmem_ld32_pair(tq + (uint32_t)(c * COLS + h * 32), tq + (uint32_t)(WIDTH + c * COLS + h * 32), gv, uv);
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                  float a0, a1, unused;
                  activation<ACT, true>(gv[2 * q], a0, unused);
                  activation<ACT, true>(gv[2 * q + 1], a1, unused);
                  o[16 * h + q] = pack2<T>(a0 * uv[2 * q], a1 * uv[2 * q + 1]);
                  gw[16 * h + q] = pack2<T>(gv[2 * q], gv[2 * q + 1]);
                  uw[16 * h + q] = pack2<T>(uv[2 * q], uv[2 * q + 1]);
                }
              }
              put_rows<U>(o, stg, lane, p.d.p, p.d.ld, slot_row, nc, N, true);
              if (p.gate_out.p) put_rows<U>(gw, stg, lane, p.gate_out.p, p.gate_out.ld, pair_row, nc, N, p.vec_gate);
              if (p.up_out.p) put_rows<U>(uw, stg, lane, p.up_out.p, p.up_out.ld, pair_row, nc, N, p.vec_up);
            } else if constexpr (ROWS) {
              // (32 columns of FP32 are 64 of 16 bits)
              float v[32];
              tmem_ld32(tq + (uint32_t)(c * COLS), v);
#pragma unroll
              for (int q = 0; q < 32; ++q) o[q] = __float_as_uint(v[q]);
              put_rows<8>(o, stg, lane, p.rows.p, 2 * p.rows.ld, pair_row, 2 * nc, 2 * N, true);
            } else {
#pragma unroll
              for (int h = 0; h < COLS / 32; ++h) {
                float a[16], b[16];
                if (none) {
#pragma unroll
                  for (int q = 0; q < 16; ++q) a[q] = b[q] = 0.f;
                } else {
                  tmem_ld16_pair(tq + (uint32_t)(c * COLS + h * 32), tq + (uint32_t)(c * COLS + h * 32 + 16), a, b);
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) { o[16 * h + q] = pack2<T>(a[2 * q], a[2 * q + 1]); o[16 * h + 8 + q] = pack2<T>(b[2 * q], b[2 * q + 1]); }
              }
              const GroupGrad& g = p.grad[w.grad];
              put_chunk<U, 32>(o, stg, lane, reinterpret_cast<uint16_t*>(g.d.p) + w.expert * g.d.stride, g.d.ld, w.m0 + r0, g.M, nc, N, g.vec);
            }
          }
        };
        if constexpr (KIND == GROUP_GATE) with_activation(p.act, whole);
        else whole(ActIs<GN_ACT_RELU>{});
        if (!none) end(buf);
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

// ---- host side ---------------------------------------------------------------------------------
// 3-D map over [experts][rows][cols]; box = 64 columns x box_r rows of one expert.
bool make_map_weights(CUtensorMap* m, const Weights16& a, int experts, long long rows, long long cols, int box_r, bool bf16) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)experts};
  cuuint64_t strides[2] = {(cuuint64_t)a.ld * 2, (cuuint64_t)a.stride * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_r, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(a.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND, class T>
cudaError_t launch_group_as(const GroupGemm& g, const ExpertPlan& plan, int* err, cudaStream_t st) {
  constexpr bool BF16 = !__is_same(T, __half);
  static std::atomic<signed char> ready[64];
  auto* const kernel = group_kernel<KIND, T>;
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G_SMEM) == cudaSuccess; }))
    return cudaErrorInvalidDevice;
  GroupMaps<KIND> maps;
  GroupParams p = {};
  long long most;                    // items
  bool ok = true;
  p.act = g.act; p.err = err;
  p.tiles = plan.tiles; p.n_tiles = plan.n_tiles; p.start = plan.start; p.count = plan.count; p.pair_of = plan.pair_of;
  if constexpr (KIND == GROUP_WEIGHT) {
    p.n_grads = g.n_grads;
    most = 0;
    for (int i = 0; i < g.n_grads; ++i) {
      const auto& q = g.grads[i];
      GroupGrad& to = p.grad[i];
      to.M = q.M; to.N = q.N; to.tiles_m = (q.M + 2 * G_BM - 1) / (2 * G_BM); to.tiles_n = (q.N + GroupTile<KIND>::BN - 1) / GroupTile<KIND>::BN; to.first = (int)most; to.d = q.d;
      to.vec = vec16(q.d) && q.d.stride % 8 == 0;
      most += (long long)plan.experts * to.tiles_m * to.tiles_n;
      if (most > 0x3fffffff) return cudaErrorInvalidValue;
      ok = ok && make_map16(&maps.m[2 * i], q.left, g.slots, q.M, G_BK, BF16) && make_map16(&maps.m[2 * i + 1], q.right, g.slots, q.N, G_BK, BF16);
    }
    p.items = (int)most;
  } else {
    constexpr int WIDTH = KIND == GROUP_GATE ? GroupTile<KIND>::BN / 2 : GroupTile<KIND>::BN;
    p.N = g.N; p.tiles_n = (g.N + WIDTH - 1) / WIDTH;
    p.kb0 = (g.K + G_BK - 1) / G_BK; p.kb = KIND == GROUP_DX ? 2 * p.kb0 : p.kb0;
    p.chunk = p.kb0 <= 16 ? 4 : p.kb0 >= 32 ? 8 : (p.kb0 + 3) / 4;
    p.d = g.d; p.dgate = g.dgate; p.dup = g.dup; p.gate_out = g.gate_out; p.up_out = g.up_out; p.gate = g.gate; p.up = g.up;
    p.rows = g.rows; p.vec_gate = vec16(p.gate_out); p.vec_up = vec16(p.up_out);
    p.weight = g.weight; p.parts = g.parts; p.n_parts = group_parts(g.N);
    most = plan_tiles(plan.pairs, plan.experts, kGroupHeight) * p.tiles_n;
    if (most > 0x3fffffff) return cudaErrorInvalidValue;
    for (int s = 0; s < (KIND == GROUP_DX ? 2 : 1); ++s) ok = ok && make_map16(&maps.m[2 * s], g.A[s], g.slots, g.K, G_BM, BF16);
    const auto weights = [&](int at, int b) {
      if (KIND == GROUP_GATE || KIND == GROUP_DOWN) return make_map_weights(&maps.m[at], g.B[b], plan.experts, g.N, g.K, G_BM, BF16);
      return make_map_weights(&maps.m[at], g.B[b], plan.experts, g.K, g.N, G_BK, BF16);
    };
    ok = ok && weights(1, 0);
    if (KIND == GROUP_GATE) ok = ok && weights(2, 1);
    if (KIND == GROUP_DX) ok = ok && weights(3, 1);
  }
  if (!ok) return cudaErrorInvalidValue;
  const int pairs = num_sms() / 2;
  p.pairs = most < pairs ? (int)most : pairs;
  return launch_pdl(kernel, 2 * p.pairs, G_THREADS, G_SMEM, st, maps, p);
}
template <class T>
cudaError_t launch_group_of(GroupKind kind, const GroupGemm& g, const ExpertPlan& plan, int* err, cudaStream_t st) {
  switch (kind) {
    case GROUP_GATE: return launch_group_as<GROUP_GATE, T>(g, plan, err, st);
    case GROUP_DOWN: return launch_group_as<GROUP_DOWN, T>(g, plan, err, st);
    case GROUP_GRAD: return launch_group_as<GROUP_GRAD, T>(g, plan, err, st);
    case GROUP_DX: return launch_group_as<GROUP_DX, T>(g, plan, err, st);
    default: return launch_group_as<GROUP_WEIGHT, T>(g, plan, err, st);
  }
}

}  // namespace

int group_parts(int N) { return (N + 127) / 128 * 2; }         // of 64 columns each

cudaError_t launch_group(GroupKind kind, bool bf16, const GroupGemm& g, const ExpertPlan& plan, int* err, cudaStream_t st) {
  return bf16 ? launch_group_of<__nv_bfloat16>(kind, g, plan, err, st) : launch_group_of<__half>(kind, g, plan, err, st);
}

}  // namespace gn
