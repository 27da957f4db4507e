// Launch interface between the gated feed-forward block's calls (gated_ffn.cu) and its tensor-core kernels.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace gn {

// A stored matrix of 16-bit elements, 16-byte aligned with a leading dimension that is a multiple of 8 where TMA is to read it.
struct Mat16 { const void* p = nullptr; int64_t ld = 0; };
struct Out16 { void* p = nullptr; int64_t ld = 0; };

// What becomes of the sums acc(m, n) = sum_k A(m, k) B(k, n) (+ the same of a second operand pair):
//   FFN_STORE  d[0] = acc
//   FFN_GATE   two right operands, B[0] and B[1], one sum each: gate and up.  d[0] = h = act(gate) * up; d[1], d[2] = gate, up (optional);
//              low = what the rounding of h has left (optional, the kernel for few tokens only)
//   FFN_GRAD   acc = dh: d[0] = act(gate) * up, d[1] = dh up act'(gate), d[2] = dh act(gate), from the stored gate and up
enum FfnKind { FFN_STORE = 0, FFN_GATE = 1, FFN_GRAD = 2 };
struct FfnGemm {
  int M = 0, N = 0;
  int K[2] = {0, 0};             // K[1] > 0: a second operand pair (FFN_STORE)
  bool a_mn = false, b_mn = false;   // stored [K][M], [K][N] instead of [M][K], [N][K]
  Mat16 A[2], B[2];
  Out16 d[3], low;
  Mat16 gate, up;
};
constexpr int kFfnGroup = 4;     // problems of one launch (FFN_STORE)

// The current device's word for the code of a bounded wait that ran out (nullptr: there is none); gn_gated_ffn_status looks at it, and clears it.
int* ffn_error_word();

// CTA-pair kernels (gemm_pair16.cu).  Returns cudaSuccess, or what the launch or the maps failed with.  ws: ffn_pair_workspace bytes for the same
// products (FFN_STORE; sizes alone count).  Of FFN_GATE (operands K-major) and FFN_GRAD (B [K][N]) one product with one pair of operands.
int64_t ffn_pair_workspace(const FfnGemm* g, int n);
cudaError_t launch_ffn_pair(FfnKind kind, bool bf16, int act, const FfnGemm* g, int n, void* ws, int* err, cudaStream_t st);

// One product with few tokens (gemm_narrow16.cu): A K-major.  early: the kernel before it on the stream is one of these
// kernels, of the same call, that writes none of the right operands.
cudaError_t launch_ffn_narrow(FfnKind kind, bool bf16, int act, const FfnGemm& g, bool early, int* err, cudaStream_t st);
// Estimated times, to choose between the two: of a product of M = tokens and N = features (K terms, of both operand pairs), and of a list of FFN_STORE products.
constexpr int kFfnNarrow = 128;          // tokens up to which the choice is the narrow form without a look
double ffn_narrow_us(FfnKind kind, int tokens, int features, int K);
double ffn_pair_us(FfnKind kind, int M, int N, int K);
double ffn_pair_list_us(const FfnGemm* g, int n);

// One FP32 product of the forward pass on FMAs, for few tokens (always up to kFfnDot of them; ffn_dot.cu): d[0] = x w[0]^T, or with w[1] act(x w[0]^T) * (x w[1]^T) and
// the two projections to d[1], d[2] (optional).  Any alignment.
constexpr int kFfnDot = 8;
struct FfnMat { const float* p = nullptr; int64_t ld = 0; };
struct FfnOut { float* p = nullptr; int64_t ld = 0; };
struct FfnDot { int tokens, features, K, act; FfnMat x, w[2]; FfnOut d[3]; };
cudaError_t launch_ffn_dot(const FfnDot& g, cudaStream_t st);

// FP32 products of a small backward pass on FMAs, n of them as one launch (ffn_small.cu): d [M][N] = sum over s of A_s B_s, B stored [K][N], A [M][K] or
// (a_mn) [K][M].  With `grad` the one product is dh, and what is written is h, dgate and dup.  Any alignment.  ffn_small_us: an estimate.
struct FfnSmall { int M = 0, N = 0, K[2] = {0, 0}; bool a_mn = false; FfnMat A[2], B[2]; FfnOut d; };
struct FfnSmallGrad { int act; FfnMat gate, up; FfnOut out[3]; };
double ffn_small_us(const FfnSmall* g, int n);
cudaError_t launch_ffn_small(const FfnSmall* g, int n, const FfnSmallGrad* grad, cudaStream_t st);

}  // namespace gn
