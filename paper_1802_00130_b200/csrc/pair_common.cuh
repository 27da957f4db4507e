// What the kernels of CTA pairs on 16-bit operands share (gemm_pair16.cu, gemm_group16.cu): the product instruction, sums from tensor memory,
// and the way of a tile's chunks between a thread's row in registers and whole runs of rows in global memory.
#pragma once
#include "ffn_act.cuh"
#include "ffn_kernels.h"
#include "tc_common.cuh"

namespace gn {
namespace {

template <bool BF16>
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accum) : "memory");
}

// Two times 32 columns of this warp's quadrant (lane = row), waited for in the same statement: nothing may move a value before it is there.
__device__ __forceinline__ void tmem_ld32_pair(uint32_t a, uint32_t b, float (&x)[32], float (&y)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%65];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]),
        "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]),
        "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]),
        "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31]), "=f"(y[0]), "=f"(y[1]), "=f"(y[2]), "=f"(y[3]), "=f"(y[4]), "=f"(y[5]),
        "=f"(y[6]), "=f"(y[7]), "=f"(y[8]), "=f"(y[9]), "=f"(y[10]), "=f"(y[11]), "=f"(y[12]), "=f"(y[13]), "=f"(y[14]), "=f"(y[15]),
        "=f"(y[16]), "=f"(y[17]), "=f"(y[18]), "=f"(y[19]), "=f"(y[20]), "=f"(y[21]), "=f"(y[22]), "=f"(y[23]), "=f"(y[24]),
        "=f"(y[25]), "=f"(y[26]), "=f"(y[27]), "=f"(y[28]), "=f"(y[29]), "=f"(y[30]), "=f"(y[31])
      : "r"(a), "r"(b) : "memory");
}

__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
// A warp's staging tile: 32 rows of U units of 16 bytes (8 or 4: 64 or 32 columns), a row's units permuted by the row's low bits so that neither
// whole rows nor one unit of many rows meet in a bank.
template <int U>
__device__ __forceinline__ uint32_t stg_at(uint32_t stg, int row, int unit) {
  return stg + (uint32_t)(row * 16 * U + ((unit ^ (U == 8 ? row & 7 : row >> 1 & 3)) << 4));
}

__device__ __forceinline__ uint16_t lds2(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
  return v;
}
// A unit's part of a row of `cols` columns to where it does not start on 16 bytes: a store's 16 bytes are put together from two units of the staging tile, and the up to seven elements
// before the row's first such place, and those after its last, go one by one.
// 8000 tokens, 1001 columns, 3001 hidden units forward: 172 us where no matrix is aligned (228 in words of four bytes, a row at a time), 143 where all are.
template <int U>
__device__ __forceinline__ void put_loose(uint16_t* p, uint32_t stg, int row, int unit, int cols) {
  const int head = min(cols, (int)(-(reinterpret_cast<uintptr_t>(p) >> 1) & 7)), wholes = (cols - head) >> 3;
  if (unit < wholes) {
    const uint4 x = lds16(stg_at<U>(stg, row, unit)), y = lds16(stg_at<U>(stg, row, unit + (head > 0)));
    const bool two = head & 4, one = head & 2;
    const uint32_t a0 = two ? x.z : x.x, a1 = two ? x.w : x.y, a2 = two ? y.x : x.z, a3 = two ? y.y : x.w, a4 = two ? y.z : y.x, a5 = two ? y.w : y.y;
    const uint32_t b0 = one ? a1 : a0, b1 = one ? a2 : a1, b2 = one ? a3 : a2, b3 = one ? a4 : a3, b4 = one ? a5 : a4;
    const uint32_t by = (head & 1) * 16;
    *reinterpret_cast<uint4*>(p + head + unit * 8) =
        make_uint4(__funnelshift_r(b0, b1, by), __funnelshift_r(b1, b2, by), __funnelshift_r(b2, b3, by), __funnelshift_r(b3, b4, by));
  }
  for (int i = unit; i < cols - 8 * wholes; i += U) {
    const int e = i < head ? i : 8 * wholes + i;
    p[e] = lds2(stg_at<U>(stg, row, e >> 3) + (e & 7) * 2u);
  }
}
// This thread's row of a chunk, 8 U elements in 4 U words, to columns n0.. (of N) of row_of(its number of 0..31) of a matrix (negative: no such row), by way of the
// staging tile, in stores of 16 bytes.  vec: the rows' chunks start where such a store may.
template <int U, class RowOf>
__device__ __forceinline__ void put_rows(const uint32_t (&w)[4 * U], uint32_t stg, int lane, void* base, int64_t ld, RowOf row_of, int n0, int N, bool vec) {
  const int cols = min(8 * U, N - n0), unit = lane % U;
#pragma unroll
  for (int q = 0; q < U; ++q) sts16(stg_at<U>(stg, lane, q), make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]));
  __syncwarp();
  uint16_t* const at = reinterpret_cast<uint16_t*>(base) + n0;
  if (vec) {
#pragma unroll
    for (int it = 0; it < U; ++it) {
      const int row = it * (32 / U) + lane / U, m = row_of(row);
      if (m >= 0 && unit * 8 + 8 <= cols) *reinterpret_cast<uint4*>(at + m * ld + unit * 8) = lds16(stg_at<U>(stg, row, unit));
    }
    if (cols & 7) {
      const int m = row_of(lane);
      if (m >= 0)
        for (int e = cols & ~7; e < cols; ++e) at[m * ld + e] = lds2(stg_at<U>(stg, lane, e >> 3) + (e & 7) * 2u);
    }
  } else {
#pragma unroll 2
    for (int it = 0; it < U; ++it) {
      const int row = it * (32 / U) + lane / U, m = row_of(row);
      if (m >= 0) put_loose<U>(at + m * ld, stg, row, unit, cols);
    }
  }
  __syncwarp();
}
// The same to rows m0.. (of M), which follow one another, ROWS rows at a time.  (Taken for rows of a list they cost the backward passes of few tokens a microsecond, 28.9 instead of 28.0 us
// for one token of 1024 columns and 4096 hidden units.)
template <int U, int ROWS>
__device__ __forceinline__ void put_chunk(const uint32_t (&w)[4 * U], uint32_t stg, int lane, void* base, int64_t ld, int m0, int M, int n0, int N, bool vec) {
  const int cols = min(8 * U, N - n0), unit = lane % U;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += ROWS) {
    if (ROWS == 32 || lane / ROWS == r0 / ROWS) {
#pragma unroll
      for (int q = 0; q < U; ++q) sts16(stg_at<U>(stg, lane % ROWS, q), make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]));
    }
    __syncwarp();
    uint16_t* const at = reinterpret_cast<uint16_t*>(base) + (int64_t)(m0 + r0) * ld + n0;
    if (vec) {
      if (unit * 8 + 8 <= cols) {
#pragma unroll
        for (int it = 0; it < ROWS * U / 32; ++it) {
          const int row = it * (32 / U) + lane / U;
          const uint4 v = lds16(stg_at<U>(stg, row, unit));
          if (m0 + r0 + row < M) *reinterpret_cast<uint4*>(at + (int64_t)row * ld + unit * 8) = v;
        }
      }
      if (lane < ROWS && m0 + r0 + lane < M)
        for (int e = cols & ~7; e < cols; ++e) at[(int64_t)lane * ld + e] = lds2(stg_at<U>(stg, lane, e >> 3) + (e & 7) * 2u);
    } else {
#pragma unroll 2
      for (int it = 0; it < ROWS * U / 32; ++it) {
        const int row = it * (32 / U) + lane / U;
        if (m0 + r0 + row >= M) break;
        put_loose<U>(at + (int64_t)row * ld, stg, row, unit, cols);
      }
    }
    __syncwarp();
  }
}
// A chunk of 32 columns, all of them there and addressable in units of 16 bytes.
__device__ __forceinline__ void put_whole(const uint32_t* w, uint32_t stg, int lane, void* base, int64_t ld, int m0, int M, int n0) {
#pragma unroll
  for (int q = 0; q < 4; ++q) sts16(stg_at<4>(stg, lane, q), make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]));
  __syncwarp();
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int row = it * 8 + lane / 4;
    const uint4 v = lds16(stg_at<4>(stg, row, lane & 3));
    if (m0 + row < M) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + (int64_t)(m0 + row) * ld + n0 + (lane & 3) * 8) = v;
  }
  __syncwarp();
}
// The other way, of a matrix whose rows start where an access of 16 bytes may: four units of a chunk of 32 columns, eight rows apart, as a
// warp's accesses cover them; then by rows.
template <class RowOf>
__device__ __forceinline__ void fetch_rows(uint4 (&v)[4], int lane, const void* base, int64_t ld, RowOf row_of, int n0, int N) {
  const int n = n0 + (lane & 3) * 8;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int m = row_of(it * 8 + (lane >> 2));
    v[it] = make_uint4(0u, 0u, 0u, 0u);
    if (m < 0 || n >= N) continue;
    const uint16_t* const p = reinterpret_cast<const uint16_t*>(base) + m * ld + n;
    if (n + 8 <= N) {
      v[it] = __ldg(reinterpret_cast<const uint4*>(p));
    } else {
      unsigned long long half[2] = {0, 0};
#pragma unroll 1
      for (int e = N - n - 1; e >= 0; --e) {               // (the last one read is the lowest)
        half[1] = half[1] << 16 | half[0] >> 48;
        half[0] = half[0] << 16 | __ldg(p + e);
      }
      v[it] = make_uint4((uint32_t)half[0], (uint32_t)(half[0] >> 32), (uint32_t)half[1], (uint32_t)(half[1] >> 32));
    }
  }
}
__device__ __forceinline__ void fetch_chunk(uint4 (&v)[4], int lane, const void* base, int64_t ld, int m0, int M, int n0, int N) {
  fetch_rows(v, lane, base, ld, [&](int r) { return m0 + r < M ? m0 + r : -1; }, n0, N);
}
__device__ __forceinline__ void turn_chunk(const uint4 (&v)[4], uint32_t stg, int lane, uint32_t (&w)[16]) {
#pragma unroll
  for (int it = 0; it < 4; ++it) sts16(stg_at<4>(stg, it * 8 + (lane >> 2), lane & 3), v[it]);
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint4 x = lds16(stg_at<4>(stg, lane, q));
    w[4 * q] = x.x; w[4 * q + 1] = x.y; w[4 * q + 2] = x.z; w[4 * q + 3] = x.w;
  }
  __syncwarp();
}
// Two times 16 columns of this warp's quadrant (lane = row), waited for in the same statement: nothing may move a value before it is there.
__device__ __forceinline__ void tmem_ld16_pair(uint32_t a, uint32_t b, float (&x)[16], float (&y)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]),
        "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(y[0]), "=f"(y[1]), "=f"(y[2]), "=f"(y[3]),
        "=f"(y[4]), "=f"(y[5]), "=f"(y[6]), "=f"(y[7]), "=f"(y[8]), "=f"(y[9]), "=f"(y[10]), "=f"(y[11]), "=f"(y[12]), "=f"(y[13]),
        "=f"(y[14]), "=f"(y[15])
      : "r"(a), "r"(b) : "memory");
}

// ---- host side ---------------------------------------------------------------------------------
// 2-D map over a row-major [rows][cols] matrix of 16-bit elements; box = 64 columns x box_r rows.
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
// The same of a [K][MN] matrix of whole 64-column chunks: one box holds 64 rows of `chunks` chunks, chunk after chunk.
bool make_map16_chunks(CUtensorMap* m, const Mat16& a, long long rows, long long cols, int chunks, bool bf16) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(cols / 64)};
  cuuint64_t strides[2] = {(cuuint64_t)a.ld * 2, 128};
  cuuint32_t box[3] = {64, 64, (cuuint32_t)chunks};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(a.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <class P> bool vec16(const P& m) { return !m.p || (((uintptr_t)m.p & 15) == 0 && m.ld % 8 == 0); }

}  // namespace
}  // namespace gn
