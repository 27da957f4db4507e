// Launch interface between the calls on 4-bit weights (weight4.cu) and their products' kernel (weight4_product.cuh, once for each type).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "expert_kernels.h"

namespace gn {

// 4-bit weights of one matrix [rows][cols], or of every expert's, as they are laid out: see gn.h.
struct Weight4 { const uint8_t* q = nullptr; const void* scale = nullptr; };
inline int64_t w4_tiles(int64_t rows) { return (rows + 15) / 16; }
inline int64_t w4_blocks(int64_t cols) { return (cols + 127) / 128; }
inline int64_t w4_bytes(int64_t rows, int64_t cols) { return w4_tiles(rows) * w4_blocks(cols) * 1024; }                                   // of an expert's q
inline int64_t w4_scales(int64_t rows, int64_t cols, int group) { return w4_tiles(rows) * w4_blocks(cols) * 16 * (128 / group); }          // of an expert

// d [columns][rows] = x w^T, columns being tokens (or pairs of a plan: a tile of up to 8 or 32 of an expert's).  gate: w[0] and w[1], d = act(.) * (.) in FP32.
//   x        of the type, or (x32) FP32: what the gate has written
//   d        of the type, or (d32) FP32
struct Product4 {
  int rows = 0, cols = 0, group = 128, act = 0;
  int64_t tokens = 0;
  bool gate = false, x32 = false, d32 = false, early = false;        // early: the weights may be loaded before the kernel before this one is done
  const void* x = nullptr; int64_t ldx = 0;
  Weight4 w[2];
  void* d = nullptr; int64_t ldd = 0;
  const ExpertPlan* plan = nullptr;  // its tiles have 8 or 32 columns
  int k = 1; bool token_rows = false;            // of a plan: rows of x are the tokens', else the pairs'
  int columns = 8;                   // of a tile
};
cudaError_t launch_product4_f32(const Product4& p, cudaStream_t st);
cudaError_t launch_product4_bf16(const Product4& p, cudaStream_t st);
cudaError_t launch_product4_f16(const Product4& p, cudaStream_t st);

}  // namespace gn
