// Products of a few tokens with 4-bit weights: bound by the weights' bytes, half a byte each, and close behind by what it takes to make operands of them.
//
// The weights are laid out for the kernel: a record of 1 KB has 16 rows by 128 columns, 16 bytes for each lane of a warp from rows 0..7 and 16 from rows 8..15, so
// that a warp's load is 512 bytes in a row and a tile's records follow one another.  A lane's word has eight neighbouring columns, the even ones in its low
// halves' nibbles: a mask and an or make two of them a pair of 16-bit numbers, 128 + q say, from which 136 is taken: q - 8 exactly.  The tensor core's m16n8k16 takes
// them against eight tokens; its 32-bit sums of a group of columns get the group's scale.  (A tile of tcgen05 would need the operands in shared memory, as many bytes
// again as 16-bit weights.  A second product, of the tokens with 136, in the place of the operands' subtractions took longer: 31 against 25 us for a token
// through 4096 x 8192.)
//
// Measured in a graph: one BF16 token by 8192 x 4096 7.5 us (17 MB; the same stream without the products 3.8), by 16384 x 8192 25 (16), through a layer of 4096 x 8192 22 (13), 8
// tokens through that layer 24, 16 tokens 33, 32 tokens 64; 8 FP16 tokens through 8 of 64 experts of 2048 x 1024 49 (140 MB).
// FP32 tokens are columns of three BF16 parts of eight bits each, exact; the hidden units of a gated layer of two (17 bits) where the result is rounded to 16
// bits, as the first kernel has written them.
// Four or eight warps share a block: W of them a tile of 16 rows (of both matrices, gate), each with every W-th record; their sums are added in order in shared memory.  W is
// what it takes to give every SM its warps: a warp with many records streams them, through a ring of its own in shared memory that asynchronous copies fill
// several records ahead (a lane reads back what it has asked for itself, and the scales what its warp has).
#pragma once
#include "ffn_act.cuh"
#include "tc_common.cuh"
#include "weight4_kernels.h"

namespace gn {
namespace {

constexpr int Q_WARPS = 8, Q_THREADS = 32 * Q_WARPS;           // of a block at most
struct Product4Params {
  int rows, cols, act, kblocks, tiles, split, log_split, log_block, early, k, token_rows, tokens;
  const void* x; int64_t ldx, part_stride;
  const uint8_t* q[2]; const void* scale[2];
  int64_t q_stride, scale_stride;    // from expert to expert
  void* d; int64_t ldd, part_stride_d; int d32;
  const ExpertTile* list; const int* n_list; const int* pair_of;
};

// Columns 2 i and 2 i + 1 of a word, less 8: q + 128 in BF16's seven bits of fraction; in FP16's ten q + 1024, or q + 64 four bits up, which is a shift for two pairs.
template <class O>
__device__ __forceinline__ uint32_t quarter_pair(uint32_t w, int i) {
  if constexpr (__is_same(O, __half)) {
    const uint32_t x = i < 2 ? w : w >> 8, v = i & 1 ? (x & 0x00f000f0u) | 0x54005400u : (x & 0x000f000fu) | 0x64006400u, by = i & 1 ? 0xd480d480u : 0xe408e408u;
    const __half2 h = __hadd2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&by));
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const uint32_t v = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u, by = 0xc308c308u;
    const __nv_bfloat162 h = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&by));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
// d = a b, or with `more` d += a b.
template <class O>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, bool more) {
  const float c0 = more ? d[0] : 0.f, c1 = more ? d[1] : 0.f, c2 = more ? d[2] : 0.f, c3 = more ? d[3] : 0.f;
  if constexpr (__is_same(O, __half))
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

// Eight neighbouring columns of a row of operands, which starts on 16 bytes and has whole eights (zero past its end).
template <class O>
__device__ __forceinline__ uint4 load_eight(const O* row, int c, int cols) {
  return row && c < cols ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0u, 0u, 0u, 0u);
}
// An FP32 number as PARTS BF16 numbers that add up to it: the leading 8 bits of what is left, cut off, three times (exact), or once and the rest rounded.
// Infinities leave nothing.
template <int PARTS>
__device__ __forceinline__ void split_parts(float v, __nv_bfloat16 (&o)[PARTS]) {
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    if (i == 1 && PARTS == 2) { o[i] = __float2bfloat16_rn(v); break; }
    const uint32_t high = __float_as_uint(v) & 0xffff0000u;
    o[i] = __nv_bfloat16(__nv_bfloat16_raw{(unsigned short)(high >> 16)});
    v = fabsf(v) == __int_as_float(0x7f800000) ? 0.f : v - __uint_as_float(high);
  }
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// A warp's ring: of each record, for each of M matrices, the 1 KB of weights and 16 rows' scales.
template <class T, int G, int M> constexpr int q_piece = 1024 + 16 * G * (int)sizeof(T);
template <int M> constexpr int q_stages = M == 2 ? 4 : 6;
template <class T, int G, int M> constexpr int q_ring = q_stages<M> * M * q_piece<T, G, M>;
constexpr int Q_PITCH = 17;          // of a column's 16 sums
template <class T, int G, int NT, int M> constexpr int q_smem = q_ring<T, G, M> > M * 8 * NT * Q_PITCH * 4 ? q_ring<T, G, M> : M * 8 * NT * Q_PITCH * 4;     // of a warp

// T: type of the scales and of the result; O: of the operands; PARTS columns to a token; G groups of a record; NT tiles of eight columns; M matrices (2: gate).
template <class T, class O, int PARTS, int G, int NT, int M>
__global__ void __launch_bounds__(Q_THREADS, NT * M == 1 ? 3 : 2) product4_kernel(const __grid_constant__ Product4Params p) {
  constexpr int COLUMNS = 8 * NT, TOKENS = COLUMNS / PARTS, STAGES = q_stages<M>, PIECE = q_piece<T, G, M>, SCALE_UNITS = G * (int)sizeof(T);
  static_assert(M * SCALE_UNITS <= 32, "a lane copies one unit of the scales");
  extern __shared__ __align__(16) uint8_t smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int slice = warp & (p.split - 1), tile = (blockIdx.x << p.log_block) + (warp >> p.log_split);
  const bool on = tile < p.tiles;
  uint8_t* const ring = smem + warp * q_ring<T, G, M>;
  const uint32_t to = smem_u32(ring);
  int expert = 0, tokens = 0, slot = 0;
  // What a list says, and weights, need not wait for the kernel before this one where that has waited for what has written them.
  const auto place = [&] {
    if (p.list) {
      if ((int)blockIdx.y >= *p.n_list) return false;
      const int4 e = *reinterpret_cast<const int4*>(p.list + blockIdx.y);
      expert = e.x; slot = e.y; tokens = e.z;
    } else {
      tokens = min(p.tokens - (int)blockIdx.y * TOKENS, TOKENS);
    }
    return true;
  };
  // This lane's 16 bytes of the next record to ask for, of each matrix, and of the scales.
  const uint8_t *from[M], *from_scale = nullptr;
  const uint32_t to_lane = to + lane * 16, to_scale = to + (M == 2 && lane >= SCALE_UNITS ? PIECE : 0) + 1024 + lane % SCALE_UNITS * 16;
  const int step = p.split * 1024, step_scale = p.split * 16 * SCALE_UNITS;
  int left = 0;                      // records to ask for
  const auto request = [&](int stage) {
    if (left > 0) {
#pragma unroll
      for (int m = 0; m < M; ++m) {
        cp_async16(to_lane + stage * (M * PIECE) + m * PIECE, from[m]);
        cp_async16(to_lane + stage * (M * PIECE) + m * PIECE + 512, from[m] + 512);
        from[m] += step;
      }
      if (lane < M * SCALE_UNITS) cp_async16(to_scale + stage * (M * PIECE), from_scale);
      from_scale += step_scale;
      --left;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const auto begin = [&] {
    const int64_t record = (int64_t)tile * p.kblocks + slice;
    left = on && slice < p.kblocks ? (p.kblocks - slice + p.split - 1) / p.split : 0;
#pragma unroll
    for (int m = 0; m < M; ++m) from[m] = p.q[m] + expert * p.q_stride + record * 1024 + lane * 16;
    from_scale = (const uint8_t*)p.scale[M == 2 && lane >= SCALE_UNITS && lane < 2 * SCALE_UNITS ? 1 : 0] +
                 (expert * p.scale_stride + record * (16 * G)) * (int64_t)sizeof(T) + lane % SCALE_UNITS * 16;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) request(i);
  };
  bool some = true;
  if (p.early) {
    some = place();
    if (some) begin();
  }
  grid_dep_wait();
  grid_dep_launch();
  if (!p.early) {
    some = place();
    if (some) begin();
  }
  if (!some) return;
  const auto row_of = [&](int c) { return p.list ? p.pair_of[slot + c] : (int)blockIdx.y * TOKENS + c; };
  const int columns = tokens * PARTS;            // column PARTS i + j: part j of token i
  const O* row[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    row[n] = nullptr;
    const int c = 8 * n + g;
    if (c < columns) {
      int r = row_of(c / PARTS);
      if (p.token_rows && p.k > 1) r = (int)((unsigned)r / (unsigned)p.k);
      row[n] = (const O*)p.x + r * p.ldx + c % PARTS * p.part_stride;
    }
  }
  float acc[M][NT][4] = {};
  if (on) {
    int stage = 0;
    // Eight tokens' columns of the next record (of two matrices: with one the loads ahead took longer, 35 us instead of 25 for 16384 x 8192).
    uint4 ahead[NT == 1 ? 4 : 1];
    const auto look_ahead = [&](int kb) {
      if constexpr (NT == 1 && M == 2) {
#pragma unroll
        for (int b = 0; b < 4; ++b) ahead[b] = load_eight(row[0], kb * 128 + b * 32 + t * 8, p.cols);
      }
    };
    look_ahead(slice);
#pragma unroll 1
    for (int kb = slice; kb < p.kblocks; kb += p.split) {
      // The tokens' columns: of the whole record, or (many tokens) of a quarter of it and the next.
      constexpr int QUARTERS = NT <= 2 ? 4 : 2;
      uint4 x[QUARTERS][NT];
      const int c0 = kb * 128 + t * 8;
#pragma unroll
      for (int b = 0; b < (NT <= 2 ? 4 : 1); ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n) x[b][n] = NT == 1 && M == 2 ? ahead[b] : load_eight(row[n], c0 + b * 32, p.cols);
      look_ahead(kb + p.split);
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncwarp();
      request(stage == 0 ? STAGES - 1 : stage - 1);
      const uint8_t* const at = ring + stage * (M * PIECE);
      uint4 w[M][2];
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) w[m][h] = *reinterpret_cast<const uint4*>(at + m * PIECE + h * 512 + lane * 16);
      // (two chains of products side by side where a group is long enough and there is room)
      constexpr int CHAINS = NT == 1 && G == 1 ? 2 : 1;
      float part[CHAINS][M][NT][4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (NT > 2 && b < 3) {
#pragma unroll
          for (int n = 0; n < NT; ++n) x[(b + 1) % QUARTERS][n] = load_eight(row[n], c0 + (b + 1) * 32, p.cols);
        }
        const bool more = b % (4 / G) >= CHAINS;
        uint32_t a[M][2][4];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t word = b == 0 ? w[m][h].x : b == 1 ? w[m][h].y : b == 2 ? w[m][h].z : w[m][h].w;
#pragma unroll
            for (int i = 0; i < 4; ++i) a[m][h][i] = quarter_pair<O>(word, i);
          }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (NT > 1 && 8 * n >= columns) break;
          const uint4 y = x[b % QUARTERS][n];
#pragma unroll
          for (int m = 0; m < M; ++m) {
            float (&sum)[4] = part[b % CHAINS][m][n];
            mma16816<O>(sum, a[m][0][0], a[m][1][0], a[m][0][1], a[m][1][1], y.x, y.y, more);
            mma16816<O>(sum, a[m][0][2], a[m][1][2], a[m][0][3], a[m][1][3], y.z, y.w, true);
          }
        }
        if (b % (4 / G) == 4 / G - 1) {
#pragma unroll
          for (int m = 0; m < M; ++m) {
            const T* const scale = reinterpret_cast<const T*>(at + m * PIECE + 1024) + g * G + b * G / 4;
            const float low = to_f(scale[0]), high = to_f(scale[8 * G]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (NT > 1 && 8 * n >= columns) break;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float v = CHAINS == 2 ? part[0][m][n][i] + part[CHAINS - 1][m][n][i] : part[0][m][n][i];
                acc[m][n][i] = fmaf(i < 2 ? low : high, v, acc[m][n][i]);
              }
            }
          }
        }
      }
      if (++stage == STAGES) stage = 0;
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();                   // (the rings are free)
  float* const sums = reinterpret_cast<float*>(smem);            // [warp][M][COLUMNS][Q_PITCH]
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[((warp * M + m) * COLUMNS + 8 * n + 2 * t + (i & 1)) * Q_PITCH + g + 8 * (i >> 1)] = acc[m][n][i];
  __syncthreads();
  // 16 rows of a tile to neighbouring threads
  for (int i = threadIdx.x; i < tokens << (4 + p.log_block); i += blockDim.x) {
    const int r = i & 15, in = (i >> 4) & ((1 << p.log_block) - 1), c = i >> (4 + p.log_block);
    const int at = ((blockIdx.x << p.log_block) + in) * 16 + r;
    if (at >= (M == 2 ? (p.rows + 7) / 8 * 8 : p.rows)) continue;     // (rows of operands are whole eights: what is past the end is 0, an infinite token's too)
    float s[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      s[m] = 0.f;
      for (int w = 0; w < p.split; ++w)
#pragma unroll
        for (int j = PARTS - 1; j >= 0; --j) s[m] += sums[((((in << p.log_split) + w) * M + m) * COLUMNS + c * PARTS + j) * Q_PITCH + r];
    }
    const int64_t d = row_of(c) * p.ldd + at;
    if constexpr (M == 2) {
      // the parts that the second product takes
      constexpr int OUT = sizeof(T) == 4 ? 3 : 2;
      with_activation(p.act, [&](auto act) {
        float h, unused;
        activation<decltype(act)::value, sizeof(T) == 2>(s[0], h, unused);
        if (at >= p.rows) h = s[1] = 0.f;
        __nv_bfloat16 o[OUT];
        split_parts<OUT>(h * s[1], o);
#pragma unroll
        for (int j = 0; j < OUT; ++j) ((__nv_bfloat16*)p.d)[d + j * p.part_stride_d] = o[j];
      });
    } else {
      if (p.d32) ((float*)p.d)[d] = s[0];
      else ((T*)p.d)[d] = from_f<T>(s[0]);
    }
  }
}

template <class T, class O, int PARTS, int G, int NT, int M>
cudaError_t launch_product4_as(const Product4& a, cudaStream_t st) {
  Product4Params p = {};
  p.rows = a.rows; p.cols = a.cols; p.act = a.act; p.kblocks = (int)w4_blocks(a.cols); p.tiles = (int)w4_tiles(a.rows);
  p.early = a.early; p.k = a.k; p.token_rows = a.token_rows; p.tokens = (int)a.tokens; p.x = a.x; p.ldx = a.ldx; p.part_stride = a.part_stride;
  p.d = a.d; p.ldd = a.ldd; p.d32 = a.d32; p.part_stride_d = a.part_stride_d;
  if (((uintptr_t)a.x & 15) || a.ldx % 8 || a.part_stride % 8) return cudaErrorInvalidValue;
  for (int m = 0; m < M; ++m) { p.q[m] = a.w[m].q; p.scale[m] = a.w[m].scale; }
  p.q_stride = w4_bytes(a.rows, a.cols); p.scale_stride = w4_scales(a.rows, a.cols, a.group);
  int64_t columns, busy;             // tiles of columns, and how many of them there are about
  if (a.plan) {
    p.list = a.plan->tiles; p.n_list = a.plan->n_tiles; p.pair_of = a.plan->pair_of;
    columns = plan_tiles(a.plan->pairs, a.plan->experts, a.tile_tokens);
    busy = a.plan->pairs < a.plan->experts ? a.plan->pairs : (int64_t)a.plan->experts;
  } else {
    busy = columns = (a.tokens + 8 * NT / PARTS - 1) / (8 * NT / PARTS);
  }
  // Warps to a tile: as many as the SMs have room for at once, 24 or 16 each (a few blocks too many would take as long again), of two records each at least.
  int log_split = 0;
  while ((2 << log_split) <= Q_WARPS && (4 << log_split) <= p.kblocks && p.tiles * busy * (2 << log_split) <= (NT * M == 1 ? 24LL : 16LL) * num_sms()) ++log_split;
  p.split = 1 << log_split;
  const int warps = p.split > 4 ? p.split : 4, per_block = warps / p.split;
  p.log_split = log_split; p.log_block = log_split >= 2 ? 0 : 2 - log_split;
  if (columns > 65535) return cudaErrorInvalidValue;
  auto* const kernel = product4_kernel<T, O, PARTS, G, NT, M>;
  constexpr int SMEM = q_smem<T, G, NT, M>;
  static std::atomic<signed char> ready[64];
  if (!once_per_device(ready, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Q_WARPS * SMEM) == cudaSuccess; })) return cudaErrorInvalidDevice;
  return launch_pdl_grid(kernel, dim3((unsigned)((p.tiles + per_block - 1) / per_block), (unsigned)columns), 32 * warps, warps * SMEM, st, p);
}
template <class T, class O, int PARTS, int G, int M>
cudaError_t launch_product4_nt(const Product4& a, cudaStream_t st) {
  // columns of a tile: those of the plan's tiles, or of all tokens up to 32
  const int64_t columns = (a.plan ? (int64_t)a.tile_tokens : a.tokens) * PARTS;
  if (columns <= 8 / PARTS * PARTS) return launch_product4_as<T, O, PARTS, G, 1, M>(a, st);
  return columns <= 16 / PARTS * PARTS ? launch_product4_as<T, O, PARTS, G, 2, M>(a, st) : launch_product4_as<T, O, PARTS, G, 4, M>(a, st);
}
template <class T, class O, int PARTS, int M>
cudaError_t launch_product4_of(const Product4& a, cudaStream_t st) {
  return a.group == 32 ? launch_product4_nt<T, O, PARTS, 4, M>(a, st) : a.group == 64 ? launch_product4_nt<T, O, PARTS, 2, M>(a, st) : launch_product4_nt<T, O, PARTS, 1, M>(a, st);
}

}  // namespace
}  // namespace gn
