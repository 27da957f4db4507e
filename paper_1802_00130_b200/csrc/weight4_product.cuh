// Products of a few tokens with 4-bit weights: bound by the weights' bytes, half a byte each, and close behind by what it takes to make operands of them.
//
// The weights are laid out for the kernel: a record of 1 KB has 16 rows by 128 columns, 16 bytes for each lane of a warp from rows 0..7 and 16 from rows 8..15, so
// that a warp's load is 512 bytes in a row and a tile's records follow one another.  A lane's word has eight neighbouring columns, the even ones in its low
// halves' nibbles: a mask and an exclusive or make two of them a pair of 16-bit numbers, 128 + q or 1024 + q, from which 136 or 1032 is
// taken: q - 8 exactly.  The tensor core's m16n8k16 takes them against eight tokens; its 32-bit sums of a group of columns get the group's scale.  (A tile of
// tcgen05 would need the operands in shared memory, as many bytes again as sixteen-bit weights.)
//
// FP32 tokens go in three 16-bit parts of eight bits each, exact; the hidden units of a gated layer, FP32 as the first kernel leaves them, in two (17 bits) where the result is
// rounded to 16 bits.
// Eight warps share a block: W of them a tile of 16 rows (of both matrices, gate), each with every W-th record; their sums are added in order in shared memory.  A
// warp has the loads of the next records under way while it computes.
#pragma once
#include "ffn_act.cuh"
#include "tc_common.cuh"
#include "weight4_kernels.h"

namespace gn {
namespace {

constexpr int Q_WARPS = 8, Q_THREADS = 32 * Q_WARPS;
struct Product4Params {
  int rows, cols, act, kblocks, tiles, split, early, vec, k, token_rows;
  int64_t tokens;
  const void* x; int64_t ldx;
  const uint8_t* q[2]; const void* scale[2];
  int64_t q_stride, scale_stride;    // from expert to expert
  void* d; int64_t ldd; int d32;
  const ExpertTile* list; const int* n_list; const int* pair_of;
};

template <class T> struct Half2Of { using type = __nv_bfloat162; };
template <> struct Half2Of<__half> { using type = __half2; };
// Columns 2 i and 2 i + 1 of a word, less 8.
template <class T>
__device__ __forceinline__ uint32_t quarter_pair(uint32_t w, int i) {
  if constexpr (__is_same(T, __half)) {
    const uint32_t v = ((w >> (4 * i)) & 0x000f000fu) | 0x64006400u;
    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&v), __half2(__half_raw{0x6408}, __half_raw{0x6408}));
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const uint32_t v = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;
    const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), __nv_bfloat162(__nv_bfloat16_raw{0x4308}, __nv_bfloat16_raw{0x4308}));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
template <class T>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (__is_same(T, __half))
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight neighbouring columns of a token as PARTS parts of four pairs.
template <int PARTS> struct Eight { uint32_t w[PARTS][4]; };
// The leading 8 bits of v as a BF16 (cut off), and what is left of it; infinities leave nothing.
__device__ __forceinline__ uint32_t leading(float v, float& rest) {
  const uint32_t high = __float_as_uint(v) & 0xffff0000u;
  rest = fabsf(v) == __int_as_float(0x7f800000) ? 0.f : v - __uint_as_float(high);
  return high >> 16;
}
template <class X, int PARTS>
__device__ __forceinline__ Eight<PARTS> load_eight(const X* row, int c, int cols, bool vec) {
  Eight<PARTS> r;
  const int left = row ? cols - c : 0;
  if constexpr (sizeof(X) == 2) {
    static_assert(PARTS == 1, "16-bit tokens are operands as they are");
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (vec && left >= 8) {
      v = *reinterpret_cast<const uint4*>(row + c);
    } else if (left > 0) {
      uint32_t o[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) o[e >> 1] |= (uint32_t) * reinterpret_cast<const uint16_t*>(row + c + e) << (16 * (e & 1));
      v = make_uint4(o[0], o[1], o[2], o[3]);
    }
    r.w[0][0] = v.x; r.w[0][1] = v.y; r.w[0][2] = v.z; r.w[0][3] = v.w;
  } else {
    float f[8];
    if (vec && left >= 8) {
      const float4 a = *reinterpret_cast<const float4*>(row + c), b = *reinterpret_cast<const float4*>(row + c + 4);
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e < left ? row[c + e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = f[2 * i], b = f[2 * i + 1];
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        if (part == PARTS - 1 && PARTS == 2) {
          r.w[part][i] = pack2<__nv_bfloat16>(a, b);           // (the last of two is rounded)
        } else {
          float ra, rb;
          const uint32_t lo = leading(a, ra), hi = leading(b, rb);
          r.w[part][i] = lo | hi << 16;
          a = ra; b = rb;
        }
      }
    }
  }
  return r;
}

// G scales of a row for a record's groups.
template <class T, int G> struct Scales { T s[G]; };
template <class T, int G>
__device__ __forceinline__ Scales<T, G> load_scales(const T* p) {
  Scales<T, G> r;
  constexpr int BYTES = G * (int)sizeof(T);
  if constexpr (BYTES == 16) *reinterpret_cast<uint4*>(r.s) = *reinterpret_cast<const uint4*>(p);
  else if constexpr (BYTES == 8) *reinterpret_cast<uint2*>(r.s) = *reinterpret_cast<const uint2*>(p);
  else if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(r.s) = *reinterpret_cast<const uint32_t*>(p);
  else r.s[0] = *p;
  return r;
}

// T: type of the scales and of the result; X: of the tokens; G groups of a record; NT tiles of eight tokens; M matrices (2: gate).
template <class T, class X, int PARTS, int G, int NT, int M>
__global__ void __launch_bounds__(Q_THREADS, NT == 1 && M == 1 ? 3 : 2) product4_kernel(const __grid_constant__ Product4Params p) {
  using O = typename std::conditional<__is_same(X, __half), __half, __nv_bfloat16>::type;    // operands
  constexpr int COLUMNS = 8 * NT, PITCH = 17;
  __shared__ float sums[Q_WARPS][M][COLUMNS][PITCH];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int per_block = Q_WARPS / p.split, slice = warp % p.split;
  const int tile = blockIdx.x * per_block + warp / p.split;
  const bool on = tile < p.tiles;
  struct Record { uint4 w[M][2]; Scales<T, G> s[M][2]; };
  Record next;
  int expert = 0;
  const uint8_t* q[M];
  const T* scale[M];
  const auto base = [&] {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      q[m] = p.q[m] + expert * p.q_stride + (int64_t)tile * p.kblocks * 1024 + lane * 16;
      scale[m] = (const T*)p.scale[m] + expert * p.scale_stride + (int64_t)tile * p.kblocks * (16 * G) + g * G;
    }
  };
  const auto fetch = [&](int kb) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        next.w[m][h] = *reinterpret_cast<const uint4*>(q[m] + (int64_t)kb * 1024 + h * 512);
        next.s[m][h] = load_scales<T, G>(scale[m] + kb * (16 * G) + h * 8 * G);
      }
  };
  // (weights of one matrix that nothing before this kernel can still be writing need not wait)
  const bool ahead = p.early && !p.list && on && slice < p.kblocks;
  if (ahead) { base(); fetch(slice); }
  grid_dep_wait();
  grid_dep_launch();
  int columns, slot = 0;
  if (p.list) {
    if ((int)blockIdx.y >= *p.n_list) return;
    const int4 e = *reinterpret_cast<const int4*>(p.list + blockIdx.y);
    expert = e.x; slot = e.y; columns = e.z;
  } else {
    const int64_t left = p.tokens - (int64_t)blockIdx.y * COLUMNS;
    columns = (int)(left < COLUMNS ? left : COLUMNS);
  }
  const auto row_of = [&](int c) -> int64_t { return p.list ? p.pair_of[slot + c] : (int64_t)blockIdx.y * COLUMNS + c; };
  const X* row[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    row[n] = nullptr;
    if (8 * n + g < columns) {
      const int64_t r = row_of(8 * n + g);
      row[n] = (const X*)p.x + (p.token_rows ? r / p.k : r) * p.ldx;
    }
  }
  float acc[M][NT][4] = {};
  if (on && slice < p.kblocks) {
    if (!ahead) { base(); fetch(slice); }
#pragma unroll 1
    for (int kb = slice; kb < p.kblocks; kb += p.split) {
      const Record r = next;
      if (kb + p.split < p.kblocks) fetch(kb + p.split);
      float part[M][NT][4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b % (4 / G) == 0) {
#pragma unroll
          for (int m = 0; m < M; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) part[m][n][i] = 0.f;
        }
        uint32_t a[M][2][4];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t w = b == 0 ? r.w[m][h].x : b == 1 ? r.w[m][h].y : b == 2 ? r.w[m][h].z : r.w[m][h].w;
#pragma unroll
            for (int i = 0; i < 4; ++i) a[m][h][i] = quarter_pair<O>(w, i);
          }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const Eight<PARTS> x = load_eight<X, PARTS>(row[n], kb * 128 + b * 32 + t * 8, p.cols, p.vec);
#pragma unroll
          for (int m = 0; m < M; ++m)
#pragma unroll
            for (int part_x = PARTS - 1; part_x >= 0; --part_x) {
              mma16816<O>(part[m][n], a[m][0][0], a[m][1][0], a[m][0][1], a[m][1][1], x.w[part_x][0], x.w[part_x][1]);
              mma16816<O>(part[m][n], a[m][0][2], a[m][1][2], a[m][0][3], a[m][1][3], x.w[part_x][2], x.w[part_x][3]);
            }
        }
        if (b % (4 / G) == 4 / G - 1) {
#pragma unroll
          for (int m = 0; m < M; ++m) {
            const float low = to_f(r.s[m][0].s[b * G / 4]), high = to_f(r.s[m][1].s[b * G / 4]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              acc[m][n][0] = fmaf(low, part[m][n][0], acc[m][n][0]); acc[m][n][1] = fmaf(low, part[m][n][1], acc[m][n][1]);
              acc[m][n][2] = fmaf(high, part[m][n][2], acc[m][n][2]); acc[m][n][3] = fmaf(high, part[m][n][3], acc[m][n][3]);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums[warp][m][8 * n + 2 * t + (i & 1)][g + 8 * (i >> 1)] = acc[m][n][i];
  __syncthreads();
  // 16 rows of a tile to neighbouring threads
  for (int i = threadIdx.x; i < per_block * 16 * columns; i += Q_THREADS) {
    const int r = i & 15, in = (i >> 4) % per_block, c = (i >> 4) / per_block;
    const int at = (blockIdx.x * per_block + in) * 16 + r;
    if (at >= p.rows) continue;
    float s[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      s[m] = sums[in * p.split][m][c][r];
      for (int w = 1; w < p.split; ++w) s[m] += sums[in * p.split + w][m][c][r];
    }
    const int64_t to = row_of(c) * p.ldd + at;
    if constexpr (M == 2) {
      with_activation(p.act, [&](auto act) {
        float h, unused;
        activation<decltype(act)::value, sizeof(T) == 2>(s[0], h, unused);
        ((float*)p.d)[to] = h * s[1];
      });
    } else {
      if (p.d32) ((float*)p.d)[to] = s[0];
      else ((T*)p.d)[to] = from_f<T>(s[0]);
    }
  }
}

template <class T, class X, int PARTS, int G, int NT, int M>
cudaError_t launch_product4_as(const Product4& a, cudaStream_t st) {
  Product4Params p = {};
  p.rows = a.rows; p.cols = a.cols; p.act = a.act; p.kblocks = (int)w4_blocks(a.cols); p.tiles = (int)w4_tiles(a.rows);
  p.early = a.early; p.k = a.k; p.token_rows = a.token_rows; p.tokens = a.tokens; p.x = a.x; p.ldx = a.ldx; p.d = a.d; p.ldd = a.ldd; p.d32 = a.d32;
  p.vec = ((uintptr_t)a.x & 15) == 0 && a.ldx * (int64_t)sizeof(X) % 16 == 0;
  for (int m = 0; m < M; ++m) { p.q[m] = a.w[m].q; p.scale[m] = a.w[m].scale; }
  p.q_stride = w4_bytes(a.rows, a.cols); p.scale_stride = w4_scales(a.rows, a.cols, a.group);
  int64_t columns;
  if (a.plan) {
    p.list = a.plan->tiles; p.n_list = a.plan->n_tiles; p.pair_of = a.plan->pair_of;
    columns = plan_tiles(a.plan->pairs, a.plan->experts, 8 * NT);
  } else {
    columns = (a.tokens + 8 * NT - 1) / (8 * NT);
  }
  // Warps to a tile: two records each at least, eight warps at most.
  p.split = 1;
  while (p.split < Q_WARPS && p.split * 4 <= p.kblocks) p.split *= 2;
  const int per_block = Q_WARPS / p.split;
  if (columns > 65535) return cudaErrorInvalidValue;
  return launch_pdl_grid(product4_kernel<T, X, PARTS, G, NT, M>, dim3((unsigned)((p.tiles + per_block - 1) / per_block), (unsigned)columns), Q_THREADS, 0, st, p);
}
template <class T, class X, int PARTS, int G>
cudaError_t launch_product4_g(const Product4& a, cudaStream_t st) {
  if constexpr (sizeof(X) == sizeof(T)) {
    if (a.gate) return a.columns == 8 ? launch_product4_as<T, X, PARTS, G, 1, 2>(a, st) : launch_product4_as<T, X, PARTS, G, 4, 2>(a, st);
  }
  return a.columns == 8 ? launch_product4_as<T, X, PARTS, G, 1, 1>(a, st) : launch_product4_as<T, X, PARTS, G, 4, 1>(a, st);
}
template <class T, class X, int PARTS>
cudaError_t launch_product4_x(const Product4& a, cudaStream_t st) {
  return a.group == 32 ? launch_product4_g<T, X, PARTS, 4>(a, st) : a.group == 64 ? launch_product4_g<T, X, PARTS, 2>(a, st) : launch_product4_g<T, X, PARTS, 1>(a, st);
}

}  // namespace
}  // namespace gn
