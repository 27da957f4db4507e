// Launch interface between the mixture of experts' calls (experts.cu) and their kernels.
//
// A pair is a token and one of its k choices, number token * k + choice.  A slot is a pair's place in the order of the experts: each
// expert's pairs side by side, in their own order, from a slot that is a multiple of kSlots on; the slots up to the next such multiple are empty.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "ffn_kernels.h"

namespace gn {

constexpr int kSlots = 64;
constexpr int kMostExperts = 1024;

// Some of an expert's slots: rows of them hold pairs, `padded` with the empty ones behind the expert's last.
struct alignas(16) ExpertTile { int expert, slot, rows, padded; };
struct ExpertPlan {
  int experts = 0;
  int64_t pairs = 0;
  int *start = nullptr, *count = nullptr;        // of each expert: first slot, pairs
  int *slot_of = nullptr, *pair_of = nullptr;    // of a pair (-1: of no expert), of a slot (-1: empty)
  ExpertTile* tiles = nullptr; int* n_tiles = nullptr;
  int* hist = nullptr;
};
// Slots and tiles that there can be.
inline int64_t plan_slots(int64_t pairs, int experts) { return (pairs + (kSlots - 1) * (pairs < experts ? pairs : (int64_t)experts) + kSlots - 1) / kSlots * kSlots; }
inline int64_t plan_tiles(int64_t pairs, int experts, int height) { return pairs / height + (pairs < experts ? pairs : (int64_t)experts); }
int64_t plan_ints(int64_t pairs, int experts, int height);                          // words of a plan's memory
ExpertPlan plan_at(int* mem, int64_t pairs, int experts, int height);               // the plan's parts in it (16-byte aligned)
// The plan of an index table, with tiles of `height` slots (where `padded` is looked at, a multiple of kSlots).
cudaError_t launch_plan(const int* index, const ExpertPlan& plan, int height, cudaStream_t st);

// Rows of tokens, of 16-bit elements, to their pairs' slots: dst[slot of (t, j)] = src[t]; zero: empty slots are written too, zero.  Rows of dst are 16-byte aligned.
struct RowCopy { const void* src; int64_t ld; void* dst; int64_t ld_dst; };
cudaError_t launch_to_slots(const RowCopy* list, int n, int64_t tokens, int k, int cols, bool zero, const ExpertPlan& plan, cudaStream_t st);

// d[t] = sum over the choices j that are experts of weight[t k + j] (1 without weights) src[t k + j], d of type `type` (NULL: not wanted).  parts: with them,
// dweight[t k + j] = the sum of n_parts partial sums at parts[(slot of the pair) n_parts], in order; 0 for a choice that is no expert.
struct Combine {
  int64_t tokens; int k, cols, experts; const int* index; const float* weight;
  const float* src; int64_t ld; void* d; int64_t ld_d;
  const float* parts; int n_parts; const int* slot_of; float* dweight;
};
cudaError_t launch_combine(int type, const Combine& c, cudaStream_t st);

// Copies of 16-bit matrices of every expert (or of one) with rows that TMA can address: [experts][rows][cols], rows `ld` and experts `stride` apart, to rows
// ld_out apart without gaps between experts.
constexpr int kPackMats = 5;
struct PackMats { const void* src; void* dst; int64_t ld, stride, ld_out, rows; int experts, cols; };
cudaError_t launch_pack_mats(const PackMats* list, int n, cudaStream_t st);

// ---- products of 16-bit matrices over the experts' slots (gemm_group16.cu) ---------------------------------------------------
// A weight of every expert: [experts][rows][cols], experts `stride` elements apart.
struct Weights16 { const void* p = nullptr; int64_t ld = 0, stride = 0; };
struct Grads16 { void* p = nullptr; int64_t ld = 0, stride = 0; };
//   GROUP_GATE   slots: d = act(gate) * up with gate = x Wg^T, up = x Wu^T; pairs: gate, up (optional)
//   GROUP_DOWN   pairs: rows = h Wd^T, FP32
//   GROUP_GRAD   q = dy Wd; slots: d = weight act(gate) up, dgate = weight q up act'(gate), dup = weight q act(gate), from the pairs' gate and up;
//                parts[slot][n_parts]: sums over columns of q act(gate) up
//   GROUP_DX     pairs: rows = dgate Wg + dup Wu, FP32
//   GROUP_WEIGHT experts: grads[i] = sum over the expert's slots of (left row)^T (right row)
enum GroupKind { GROUP_GATE = 0, GROUP_DOWN = 1, GROUP_GRAD = 2, GROUP_DX = 3, GROUP_WEIGHT = 4 };
struct GroupGemm {
  int act = 0, N = 0, K = 0;         // columns of the result, terms (of each operand pair)
  int64_t slots = 0;
  Mat16 A[2];                        // rows of slots
  Weights16 B[2];
  Out16 d, dgate, dup;
  FfnOut rows;
  Mat16 gate, up; Out16 gate_out, up_out;
  const float* weight = nullptr; float* parts = nullptr;
  struct { int M = 0, N = 0; Mat16 left, right; Grads16 d; } grads[3];
  int n_grads = 0;
};
constexpr int kGroupHeight = 256;    // slots of a plan's tile for these kernels
int group_parts(int N);              // partial sums of a slot's gradient of its weight
cudaError_t launch_group(GroupKind kind, bool bf16, const GroupGemm& g, const ExpertPlan& plan, int* err, cudaStream_t st);

// ---- the same in FP32 on FMAs (gemm_group_fma.cu): any alignment; rows of tokens and pairs where they lie, no slots ----------
struct Weights32 { const float* p = nullptr; int64_t ld = 0, stride = 0; };
struct Grads32 { float* p = nullptr; int64_t ld = 0, stride = 0; };
struct FmaGroup {
  int act = 0, N = 0, K = 0, k = 1;  // k: choices of a token
  FfnMat A[2]; bool token_rows = false;          // rows of A are tokens', else pairs'
  Weights32 B[2];
  FfnOut d, dgate, dup;                          // (all of them pairs')
  FfnMat gate, up; FfnOut gate_out, up_out;
  const float* weight = nullptr; float* parts = nullptr;
  struct { int M = 0, N = 0; FfnMat left, right; bool left_tokens = false, right_tokens = false; Grads32 d; } grads[3];
  int n_grads = 0;
};
constexpr int kFmaHeight = 64, kFmaSmall = 32;       // slots of a plan's tile for these kernels, in large and small tiles
bool fma_small(int64_t pairs, int experts, int cols, int inner);                     // which a call takes
int fma_parts(int N, bool small);
cudaError_t launch_group_fma(GroupKind kind, const FmaGroup& g, bool small, const ExpertPlan& plan, cudaStream_t st);

// ---- the same in FP32 on the tensor cores (gemm_group32.cu) -------------------------------------------------------------------
// An FP32 matrix as three BF16 parts that add up to it, each with rows that TMA can address: [3][rows][ld], of every expert [3][experts][rows][ld].
struct Parts { void* p = nullptr; int64_t ld = 0, rows = 0; };
struct SplitMats { const float* src; int64_t ld, stride; Parts to; int64_t rows; int experts, cols; };
cudaError_t launch_split_mats(const SplitMats* list, int n, cudaStream_t st);           // up to three
// Rows of tokens to their pairs' slots, in parts; zero: the empty slots too.
struct SplitRows { const float* src; int64_t ld; Parts to; };
cudaError_t launch_split_to_slots(const SplitRows* list, int n, int64_t tokens, int k, int cols, bool zero, const ExpertPlan& plan, cudaStream_t st);
struct TensorGroup {
  int act = 0, N = 0, K = 0;
  Parts A[2], B[2];                  // rows of slots; weights
  Parts d, dgate, dup;               // in slots
  FfnOut rows;                       // of pairs
  FfnMat gate, up; FfnOut gate_out, up_out;
  const float* weight = nullptr; float* parts = nullptr;
  struct { int M = 0, N = 0; Parts left, right; Grads32 d; } grads[3];
  int n_grads = 0;
};
int tensor_parts(int N);
cudaError_t launch_group32(GroupKind kind, const TensorGroup& g, const ExpertPlan& plan, int* err, cudaStream_t st);

}  // namespace gn
