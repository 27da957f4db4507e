// 4-bit weights: their layout, from and to what they stand for, and the calls on them.  The products' kernel is in weight4_product.cuh.
#include <math.h>

#include "op_common.cuh"
#include "tc_common.cuh"
#include "weight4_kernels.h"

namespace gn {
namespace {

// The word of eight columns from c0 on of a row: its place in an expert's q.
__device__ __forceinline__ int64_t word_at(int64_t r, int64_t c0, int64_t kblocks) {
  const int in = (int)(r & 15), lane = (in & 7) * 4 + (int)(c0 >> 3 & 3);
  return (((r >> 4) * kblocks + (c0 >> 7)) * 2 + (in >> 3)) * 128 + lane * 4 + (c0 >> 5 & 3);
}
__device__ __forceinline__ int64_t scale_at(int64_t r, int64_t c0, int64_t kblocks, int group) {
  return (((r >> 4) * kblocks + (c0 >> 7)) * 16 + (r & 15)) * (128 / group) + (c0 & 127) / group;
}
__device__ __forceinline__ uint32_t nibble(uint32_t q, int e) { return q << (4 * ((e & 1) * 4 + (e >> 1))); }

// A thread has a group of a row, those that fill up the last record and the last rows of a tile included (q = 8, which stands for 0, and a scale of 0).  Done once for a model, element by
// element: 64 experts of 2048 x 1024 in BF16, groups of 32 and of 128: quantised in 0.58 and 1.16 ms, packed in 0.15 and 0.57, unpacked in 0.34 (a prompt's way).
struct Layout4 {
  int64_t rows, cols, tiles, kblocks; int experts, group;
  const void* from; int64_t ld, stride;          // weights, or their q in bytes
  const void* scales;                            // [experts][rows][groups]
  uint32_t* q; void* scale;
  void* to;                                      // unpacked
};
template <class T, bool QUANTIZE>
__global__ void __launch_bounds__(256) pack4_kernel(const __grid_constant__ Layout4 p) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t groups = p.kblocks * (128 / p.group), rows = p.tiles * 16, work = p.experts * rows * groups;
  const int64_t real = (p.cols + p.group - 1) / p.group;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t e = i / (rows * groups), r = i / groups % rows, g = i % groups, c0 = g * p.group;
    const int n = r < p.rows && c0 < p.cols ? (int)min((int64_t)p.group, p.cols - c0) : 0;
    uint32_t* const q = p.q + e * p.tiles * p.kblocks * 256;
    T* const scale = (T*)p.scale + e * rows * groups;
    T s = from_f<T>(0.f);
    if constexpr (QUANTIZE) {
      const T* const w = (const T*)dep(p.from) + e * p.stride + r * p.ld + c0;
      float most = 0.f;
      for (int k = 0; k < n; ++k) most = max_nan(most, fabsf(to_f(w[k])));
      s = from_f<T>(most / 7.f);
      const float by = to_f(s);
      for (int k = 0; k < p.group; k += 8) {
        uint32_t word = 0;
        for (int j = 0; j < 8; ++j) {
          int v = 0;
          if (k + j < n && by != 0.f) v = max(-8, min(7, __float2int_rn(__fdiv_rn(to_f(w[k + j]), by))));      // (NaN: 0)
          word |= nibble((uint32_t)(v + 8), j);
        }
        q[word_at(r, c0 + k, p.kblocks)] = word;
      }
    } else {
      const uint8_t* const w = (const uint8_t*)dep(p.from) + e * p.stride + r * p.ld + c0;
      if (n > 0) s = ((const T*)dep(p.scales))[(e * p.rows + r) * real + g];
      for (int k = 0; k < p.group; k += 8) {
        uint32_t word = 0;
        for (int j = 0; j < 8; ++j) word |= nibble(k + j < n ? w[k + j] & 15u : 8u, j);
        q[word_at(r, c0 + k, p.kblocks)] = word;
      }
    }
    scale[scale_at(r, c0, p.kblocks, p.group)] = s;
  }
}
template <class T>
__global__ void __launch_bounds__(256) unpack4_kernel(const __grid_constant__ Layout4 p) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t eights = (p.cols + 7) / 8, work = p.experts * p.rows * eights;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t e = i / (p.rows * eights), r = i / eights % p.rows, c0 = i % eights * 8;
    const uint32_t word = p.q[e * p.tiles * p.kblocks * 256 + word_at(r, c0, p.kblocks)];
    const float s = to_f(((const T*)p.scale)[e * p.tiles * 16 * p.kblocks * (128 / p.group) + scale_at(r, c0, p.kblocks, p.group)]);
    T* const to = (T*)p.to + e * p.stride + r * p.ld + c0;
    for (int j = 0; j < 8; ++j)
      if (c0 + j < p.cols) to[j] = from_f<T>((float)((int)(word >> (4 * ((j & 1) * 4 + (j >> 1))) & 15) - 8) * s);
  }
}
template <class T>
cudaError_t run_layout(const Layout4& p, int what, cudaStream_t st) {
  const int64_t work = what == 2 ? p.experts * p.rows * ((p.cols + 7) / 8) : p.experts * p.tiles * 16 * p.kblocks * (128 / p.group);
  const int64_t want = (work + 255) / 256, most = (int64_t)num_sms() * 8;
  const int grid = (int)(want < most ? want : most);
  if (what == 2) return launch_pdl(unpack4_kernel<T>, grid, 256, 0, st, p);
  return launch_pdl(what ? pack4_kernel<T, true> : pack4_kernel<T, false>, grid, 256, 0, st, p);
}

const char* sizes4(int type, int64_t experts, int64_t rows, int64_t cols, int group) {
  if (!type_ok(type)) return "type is not a gn_dtype";
  if (experts < 1 || experts > kMostExperts) return "experts must be in [1, 1024]";
  if (rows < 1 || cols < 1 || rows > (1 << 20) || cols > (1 << 20) || rows * cols >= (int64_t(1) << 31)) return "rows and cols must be in [1, 2^20] with a product below 2^31";
  if (group != 32 && group != 64 && group != 128) return "group must be 32, 64 or 128";
  return nullptr;
}
bool packed_ok(const void* q, const void* scale) { return q && scale && ((uintptr_t)q & 15) == 0 && ((uintptr_t)scale & 15) == 0; }
const char* const kPackedWhy = "q or scale of packed weights: null or not 16-byte aligned";

gn_status layout4(int what, gn_dtype type, int32_t experts, int64_t rows, int64_t cols, int32_t group, const void* from, int64_t ld, int64_t stride, const void* scales,
                  void* d_q, void* d_scale, void* to, void* stream, char* errbuf, int64_t errbuf_len) {
  const char* why = sizes4(type, experts, rows, cols, group);
  const void* const flat = what == 2 ? to : from;
  if (!why) {
    if (!packed_ok(d_q, d_scale)) why = kPackedWhy;
    else if (!flat || (what && (uintptr_t)flat % (uintptr_t)type_bytes(type)) || ld < cols || ld >= (int64_t(1) << 40) ||
             (experts > 1 && (stride < (rows - 1) * ld + cols || stride >= (int64_t(1) << 40))))
      why = "weights: null, misaligned, or a leading dimension or stride too small";
    else if (what == 0 && (!scales || (uintptr_t)scales % (uintptr_t)type_bytes(type))) why = "scales: null or misaligned";
  }
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  const Layout4 p{rows, cols, w4_tiles(rows), w4_blocks(cols), experts, group, from, ld, experts == 1 ? 0 : stride, scales, (uint32_t*)d_q, d_scale, to};
  cudaStream_t st = (cudaStream_t)stream;
  return op_done(type == GN_F32 ? run_layout<float>(p, what, st) : type == GN_BF16 ? run_layout<__nv_bfloat16>(p, what, st) : run_layout<__half>(p, what, st), errbuf, errbuf_len);
}

cudaError_t launch_product4(int type, const Product4& p, cudaStream_t st) {
  return type == GN_F32 ? launch_product4_f32(p, st) : type == GN_BF16 ? launch_product4_bf16(p, st) : launch_product4_f16(p, st);
}

// ---- the gated layer ----------------------------------------------------------------------------
struct Workspace {               // hands out 256-byte aligned pieces (of no memory at all where a call is only measured)
  char* p; int64_t used = 0;
  void* take(int64_t bytes) { void* r = p + used; used += (bytes + 255) / 256 * 256; return r; }
};
char* const kNowhere = reinterpret_cast<char*>(256);
inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

const char* ffn4_args(const gn_ffn4* f) {
  if (!f) return "no arguments";
  if (f->act < GN_ACT_SIGMOID || f->act > GN_ACT_RELU) return "act is not a gn_act";
  const char* why = sizes4(f->type, f->experts, f->inner, f->cols, f->group);
  if (why) return why;
  if (f->k < 1 || f->k > 32) return "k must be in [1, 32]";
  if (f->tokens < 0 || f->tokens >= kMostTokens4 || f->tokens * f->k >= kMostTokens4) return "tokens times k must be in [0, 2^19)";
  if (f->tokens > 0 && !f->index && (f->experts != 1 || f->k != 1)) return "without an index there is one expert, and one choice";
  if (!packed_ok(f->q_gate, f->s_gate) || !packed_ok(f->q_up, f->s_up) || !packed_ok(f->q_down, f->s_down)) return kPackedWhy;
  if (f->tokens == 0) return nullptr;
  if (!mat_ok(f->x.p, f->x.ld, f->cols, f->type)) return "x: null, misaligned, or a leading dimension below cols";
  if (!mat_ok(f->y.p, f->y.ld, f->cols, f->type)) return "y: null, misaligned, or a leading dimension below cols";
  if ((uintptr_t)f->index & 3) return "index: misaligned";
  if (f->index && (!f->weight || ((uintptr_t)f->weight & 3))) return "weight: null or misaligned";
  return nullptr;
}
struct Few4 { ExpertPlan plan; void *x, *h; float* out; int64_t ld_x, ld_h, ld_out; int tile; };
// Tokens of a plan's tile, whose operand rows (two a token in the second product, three in FP32) are eight columns of the tensor core, 16 or 32: for twice what the experts
// that can have one have on average.
int tile_tokens(int64_t pairs, int experts, bool f32) {
  const int64_t some = pairs < experts ? pairs : (int64_t)experts;
  if (f32) return pairs <= some ? 2 : 2 * pairs <= 5 * some ? 5 : 10;
  return pairs <= 2 * some ? 4 : pairs <= 4 * some ? 8 : 16;
}
int64_t lay_out(const gn_ffn4& f, char* base, Few4& w) {
  Workspace ws{base};
  const int64_t pairs = f.tokens * f.k;
  const bool f32 = f.type == GN_F32;
  w = Few4{};
  w.tile = tile_tokens(pairs, f.experts, f32);
  w.ld_x = up8(f.cols); w.ld_h = up8(f.inner); w.ld_out = up8(f.cols);
  if (!operands_ok(f.x.p, f.x.ld, f.cols, type_bytes(f.type))) w.x = ws.take((f32 ? 3 : 1) * f.tokens * w.ld_x * 2);
  w.h = ws.take((f32 ? 3 : 2) * pairs * w.ld_h * 2);
  if (f.index) {
    w.plan = plan_at((int*)ws.take(plan_ints(pairs, f.experts, w.tile) * 4), pairs, f.experts, w.tile);
    w.out = (float*)ws.take(pairs * w.ld_out * 4);
  }
  return ws.used + 256;
}
cudaError_t run_ffn4(const gn_ffn4& f, const Few4& w, cudaStream_t st) {
  const int64_t pairs = f.tokens * f.k;
  cudaError_t e = f.index ? launch_plan(f.index, w.plan, w.tile, st) : cudaSuccess;
  Product4 a, b;
  a.rows = f.inner; a.cols = f.cols; a.group = b.group = f.group; a.act = f.act; a.tokens = b.tokens = f.tokens; a.k = b.k = f.k; a.tile_tokens = b.tile_tokens = w.tile;
  a.gate = true; a.x = f.x.p; a.ldx = f.x.ld; a.token_rows = true;
  if (w.x) {
    if (e == cudaSuccess) e = launch_operands(f.x.p, f.x.ld, f.tokens, f.cols, type_bytes(f.type), w.x, st);
    a.x = w.x; a.ldx = w.ld_x; a.part_stride = f.tokens * w.ld_x;
  }
  a.w[0] = {(const uint8_t*)f.q_gate, f.s_gate}; a.w[1] = {(const uint8_t*)f.q_up, f.s_up};
  a.d = w.h; a.ldd = w.ld_h; a.part_stride_d = pairs * w.ld_h;
  b.rows = f.cols; b.cols = f.inner; b.x = w.h; b.ldx = w.ld_h; b.part_stride = a.part_stride_d; b.in_parts = true; b.early = true;
  b.w[0] = {(const uint8_t*)f.q_down, f.s_down};
  if (f.index) { a.plan = b.plan = &w.plan; b.d = w.out; b.ldd = w.ld_out; b.d32 = true; }
  else { b.d = f.y.p; b.ldd = f.y.ld; }
  if (e == cudaSuccess) e = launch_product4(f.type, a, st);
  if (e == cudaSuccess) e = launch_product4(f.type, b, st);
  if (!f.index || e != cudaSuccess) return e;
  Combine c = {};
  c.tokens = f.tokens; c.k = f.k; c.cols = f.cols; c.experts = f.experts; c.index = f.index; c.weight = f.weight; c.src = w.out; c.ld = w.ld_out; c.d = f.y.p; c.ld_d = f.y.ld;
  return launch_combine(f.type, c, st);
}

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" int64_t gn_weight4_bytes(int32_t experts, int64_t rows, int64_t cols) {
  return sizes4(GN_F32, experts, rows, cols, 128) ? -1 : experts * w4_bytes(rows, cols);
}
extern "C" int64_t gn_weight4_scales(int32_t experts, int64_t rows, int64_t cols, int32_t group) {
  return sizes4(GN_F32, experts, rows, cols, group) ? -1 : experts * w4_scales(rows, cols, group);
}
extern "C" gn_status gn_pack4(gn_dtype type, int32_t experts, int64_t rows, int64_t cols, int32_t group, const uint8_t* d_from, int64_t ld, int64_t stride, const void* d_scales,
                              void* d_q, void* d_scale, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return layout4(0, type, experts, rows, cols, group, d_from, ld, stride, d_scales, d_q, d_scale, nullptr, cuda_stream, errbuf, errbuf_len);
}
extern "C" gn_status gn_quantize4(gn_dtype type, int32_t experts, int64_t rows, int64_t cols, int32_t group, const void* d_w, int64_t ld, int64_t stride, void* d_q, void* d_scale,
                                  void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return layout4(1, type, experts, rows, cols, group, d_w, ld, stride, nullptr, d_q, d_scale, nullptr, cuda_stream, errbuf, errbuf_len);
}
extern "C" gn_status gn_unpack4(gn_dtype type, int32_t experts, int64_t rows, int64_t cols, int32_t group, const void* d_q, const void* d_scale, void* d_w, int64_t ld, int64_t stride,
                                void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  return layout4(2, type, experts, rows, cols, group, nullptr, ld, stride, nullptr, const_cast<void*>(d_q), const_cast<void*>(d_scale), d_w, cuda_stream, errbuf, errbuf_len);
}
extern "C" int64_t gn_matvec4_workspace(gn_dtype type, int64_t tokens, int64_t cols, const void* d_x, int64_t ldx) {
  if (!type_ok(type) || tokens < 0 || tokens >= kMostTokens4 || cols < 1 || cols > (1 << 20)) return -1;
  return operands_ok(d_x, ldx, cols, type_bytes(type)) ? 0 : (type == GN_F32 ? 3 : 1) * tokens * up8(cols) * 2;
}
extern "C" gn_status gn_matvec4(gn_dtype type, int64_t tokens, int64_t rows, int64_t cols, int32_t group, const void* d_x, int64_t ldx, const void* d_q, const void* d_scale,
                                void* d_y, int64_t ldy, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = sizes4(type, 1, rows, cols, group);
  if (!why) {
    const int64_t need = gn_matvec4_workspace(type, tokens, cols, d_x, ldx);
    if (need < 0) why = "tokens must be in [0, 2^19)";
    else if (!packed_ok(d_q, d_scale)) why = kPackedWhy;
    else if (tokens > 0 && !mat_ok(d_x, ldx, cols, type)) why = "x: null, misaligned, or a leading dimension below cols";
    else if (tokens > 0 && !mat_ok(d_y, ldy, rows, type)) why = "y: null, misaligned, or a leading dimension below rows";
    else if (need > 0 && (!d_ws || ((uintptr_t)d_ws & 15) || ws_bytes < need)) why = "workspace: null, not 16-byte aligned or too small";
  }
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  if (tokens == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  Product4 p;
  p.rows = (int)rows; p.cols = (int)cols; p.group = group; p.tokens = tokens; p.x = d_x; p.ldx = ldx; p.w[0] = {(const uint8_t*)d_q, d_scale}; p.d = d_y; p.ldd = ldy;
  cudaError_t e = cudaSuccess;
  if (!operands_ok(d_x, ldx, cols, type_bytes(type))) {
    e = launch_operands(d_x, ldx, tokens, (int)cols, type_bytes(type), d_ws, st);
    p.x = d_ws; p.ldx = up8(cols); p.part_stride = tokens * up8(cols);
  }
  return op_done(e == cudaSuccess ? launch_product4(type, p, st) : e, errbuf, errbuf_len);
}
extern "C" int64_t gn_gated_ffn4_workspace(const gn_ffn4* args) {
  Few4 w;
  return ffn4_args(args) ? -1 : lay_out(*args, kNowhere, w);
}
extern "C" gn_status gn_gated_ffn4(const gn_ffn4* args, void* d_ws, int64_t ws_bytes, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = ffn4_args(args);
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  Few4 w;
  char* const base = (char*)(((uintptr_t)d_ws + 255) & ~(uintptr_t)255);
  if (!d_ws || ((uintptr_t)d_ws & 15) || ws_bytes < lay_out(*args, base, w))
    return op_fail(GN_EINVAL, "workspace: null, not 16-byte aligned or too small", errbuf, errbuf_len);
  if (args->tokens == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  return op_done(run_ffn4(*args, w, (cudaStream_t)cuda_stream), errbuf, errbuf_len);
}
