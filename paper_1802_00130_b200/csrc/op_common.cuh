// What the feed-forward block's operators (layer_norm.cu, dropout.cu, gated_ffn.cu and its kernels) share: the element types,
// and the checks and errors of calls without a context.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/gn.h"

namespace gn {
namespace {

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

// (NaN where one of them is)
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }

// 16 bytes of a matrix' row, as they are stored.
template <class T>
struct Pack {
  static constexpr int V = 16 / sizeof(T);
  uint4 w;
  __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(word(e));
    else if constexpr (__is_same(T, __half)) { const __half_raw h{(unsigned short)(word(e >> 1) >> (16 * (e & 1)))}; return __half2float(__half(h)); }
    else return __uint_as_float(e & 1 ? word(e >> 1) & 0xffff0000u : word(e >> 1) << 16);   // (BF16 is FP32's upper half)
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) o[i] = __float_as_uint(x[i]);
      else if constexpr (__is_same(T, __half)) { const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]); o[i] = *reinterpret_cast<const uint32_t*>(&h); }
      else { const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]); o[i] = *reinterpret_cast<const uint32_t*>(&h); }
    }
    w = make_uint4(o[0], o[1], o[2], o[3]);
  }
};
// Column of element e of a thread's unit u of a row that `threads` threads share: neighbours where 16-byte accesses can be made to the rows (VEC), else
// `threads` apart, so that a warp's accesses to single elements are to consecutive ones.  Elements from cols on read as zero and are not written.
template <bool VEC, class T>
__device__ __forceinline__ int pack_col(int u, int e, int thread, int threads) {
  return VEC ? (u * threads + thread) * Pack<T>::V + e : (u * Pack<T>::V + e) * threads + thread;
}
template <bool VEC, class T>
__device__ __forceinline__ Pack<T> load_pack(const T* row, int u, int thread, int threads, int cols) {
  Pack<T> p{make_uint4(0u, 0u, 0u, 0u)};
  if constexpr (VEC) {
    const int c = pack_col<true, T>(u, 0, thread, threads);
    if (c + Pack<T>::V <= cols) { p.w = *reinterpret_cast<const uint4*>(row + c); return p; }
    if (c >= cols) return p;
  }
  uint32_t o[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < Pack<T>::V; ++e) {
    const int c = pack_col<VEC, T>(u, e, thread, threads);
    if (c < cols) {
      if constexpr (sizeof(T) == 4) o[e] = *reinterpret_cast<const uint32_t*>(row + c);
      else o[e >> 1] |= (uint32_t) * reinterpret_cast<const uint16_t*>(row + c) << (16 * (e & 1));
    }
  }
  p.w = make_uint4(o[0], o[1], o[2], o[3]);
  return p;
}
template <bool VEC, class T>
__device__ __forceinline__ void store_pack(T* row, const Pack<T>& p, int u, int thread, int threads, int cols) {
  if constexpr (VEC) {
    const int c = pack_col<true, T>(u, 0, thread, threads);
    if (c + Pack<T>::V <= cols) { *reinterpret_cast<uint4*>(row + c) = p.w; return; }
    if (c >= cols) return;
  }
#pragma unroll
  for (int e = 0; e < Pack<T>::V; ++e) {
    const int c = pack_col<VEC, T>(u, e, thread, threads);
    if (c < cols) {
      if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(row + c) = p.word(e);
      else *reinterpret_cast<uint16_t*>(row + c) = (uint16_t)(p.word(e >> 1) >> (16 * (e & 1)));
    }
  }
}

inline gn_status op_fail(gn_status st, const char* why, char* errbuf, int64_t errbuf_len) {
  if (errbuf && errbuf_len > 0) snprintf(errbuf, (size_t)errbuf_len, "%s", why);
  return st;
}
// The end of a call that has launched: what the launches said of themselves.
inline gn_status op_done(cudaError_t e, char* errbuf, int64_t errbuf_len) {
  if (e == cudaSuccess) { if (errbuf && errbuf_len > 0) errbuf[0] = 0; return GN_OK; }
  cudaGetLastError();
  return op_fail(e == cudaErrorMemoryAllocation ? GN_ENOMEM : GN_ECUDA, cudaGetErrorString(e), errbuf, errbuf_len);
}
inline int type_bytes(int type) { return type == GN_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == GN_F32 || type == GN_BF16 || type == GN_F16; }
// Whether 16-byte accesses can be made to a matrix or (ld == 0) to a vector.
inline bool wide_ok(const void* p, int64_t ld, int type) { return ((uintptr_t)p & 15) == 0 && ld * type_bytes(type) % 16 == 0; }
// A matrix argument: its base aligned to its elements, its rows not overlapping.
inline bool mat_ok(const void* p, int64_t ld, int64_t cols, int type) {
  return p && ((uintptr_t)p % (uintptr_t)type_bytes(type)) == 0 && ld >= cols && ld < (int64_t(1) << 40);
}

}  // namespace
}  // namespace gn
