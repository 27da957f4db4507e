// Launch interface between the calls on 4-bit weights (weight4.cu) and their products' kernel (weight4_product.cuh, once for each type).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "expert_kernels.h"

namespace gn {

// Tokens of a call stay below this: ten to a tile (FP32), and two tiles for an expert's last, are fewer tiles than a grid has in its second dimension.
constexpr int kMostTokens4 = 1 << 19;
static_assert(kMostTokens4 / 10 + 1 + kMostExperts <= 65535, "tiles of tokens fit a grid");
// 4-bit weights of one matrix [rows][cols], or of every expert's, as they are laid out: see gn.h.
struct Weight4 { const uint8_t* q = nullptr; const void* scale = nullptr; };
inline int64_t w4_tiles(int64_t rows) { return (rows + 15) / 16; }
inline int64_t w4_blocks(int64_t cols) { return (cols + 127) / 128; }
inline int64_t w4_bytes(int64_t rows, int64_t cols) { return w4_tiles(rows) * w4_blocks(cols) * 1024; }                                   // of an expert's q
inline int64_t w4_scales(int64_t rows, int64_t cols, int group) { return w4_tiles(rows) * w4_blocks(cols) * 16 * (128 / group); }          // of an expert

// d [tokens][rows] = x w^T.  gate: w[0] and w[1], d = act(.) * (.).
//   x        16-bit operands in rows that start on 16 bytes and are whole eights, zero past `cols`: tokens of the type; or BF16 rows that add up to each token, part_stride apart
//   d        of the type, or (d32) FP32; gate: BF16 parts that add up to it, two or (FP32) three, part_stride_d apart
struct Product4 {
  int rows = 0, cols = 0, group = 128, act = 0;
  int64_t tokens = 0;
  bool gate = false, in_parts = false, d32 = false, early = false;       // early: weights and plan may be read before the kernel before this one is done
  const void* x = nullptr; int64_t ldx = 0, part_stride = 0;
  Weight4 w[2];
  void* d = nullptr; int64_t ldd = 0, part_stride_d = 0;
  const ExpertPlan* plan = nullptr; int tile_tokens = 0;         // the tokens are pairs of a plan with tiles of so many, of at most 32 operand rows
  int k = 1; bool token_rows = false;            // of a plan: rows of x are the tokens', else the pairs'
};
inline int w4_parts(bool f32, bool in_parts) { return f32 ? 3 : in_parts ? 2 : 1; }
cudaError_t launch_product4_f32(const Product4& p, cudaStream_t st);
cudaError_t launch_product4_bf16(const Product4& p, cudaStream_t st);
cudaError_t launch_product4_f16(const Product4& p, cudaStream_t st);
// Rows of tokens as operands: 16-bit ones as they are, FP32 ones in three BF16 parts: to [1 or 3][rows][ld_out], ld_out = cols rounded up to 8.  operands_ok: they are that already.
inline bool operands_ok(const void* x, int64_t ldx, int64_t cols, int bytes) { return bytes == 2 && ((uintptr_t)x & 15) == 0 && ldx % 8 == 0 && cols % 8 == 0; }
cudaError_t launch_operands(const void* x, int64_t ldx, int64_t rows, int cols, int bytes, void* to, cudaStream_t st);

}  // namespace gn
