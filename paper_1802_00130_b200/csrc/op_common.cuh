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

inline gn_status op_fail(gn_status st, const char* why, char* errbuf, int64_t errbuf_len) {
  if (errbuf && errbuf_len > 0) snprintf(errbuf, (size_t)errbuf_len, "%s", why);
  return st;
}
// The end of a call that has launched: what the runtime says of it.
inline gn_status op_done(cudaError_t e, char* errbuf, int64_t errbuf_len) {
  if (e == cudaSuccess) e = cudaGetLastError(); else cudaGetLastError();
  if (e == cudaSuccess) { if (errbuf && errbuf_len > 0) errbuf[0] = 0; return GN_OK; }
  return op_fail(e == cudaErrorMemoryAllocation ? GN_ENOMEM : GN_ECUDA, cudaGetErrorString(e), errbuf, errbuf_len);
}
inline int type_bytes(int type) { return type == GN_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == GN_F32 || type == GN_BF16 || type == GN_F16; }
// A matrix argument: its base aligned to its elements, its rows not overlapping.
inline bool mat_ok(const void* p, int64_t ld, int64_t cols, int type) {
  return p && ((uintptr_t)p % (uintptr_t)type_bytes(type)) == 0 && ld >= cols && ld < (int64_t(1) << 40);
}

}  // namespace
}  // namespace gn
