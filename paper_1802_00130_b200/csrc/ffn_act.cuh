// The gated block's activations and their derivatives, and two 16-bit elements to a word.
#pragma once
#include "op_common.cuh"

namespace gn {
namespace {

// 1 / (1 + exp(-v)) and 1 / (1 + exp(v)), each to full relative accuracy: one minus the other would lose it where it is small.
// FAST: the hardware's exponential and reciprocal, off by at most (4 + |v|) 2^-23: for results that are rounded to 16 bits, 2^-12 at best.
template <bool FAST>
__device__ __forceinline__ void sigmoids(float v, float& z, float& nz) {
  const float e = FAST ? __expf(-fabsf(v)) : expf(-fabsf(v)), r = FAST ? __fdividef(1.f, 1.f + e) : 1.f / (1.f + e);
  z = v < 0.f ? e * r : r; nz = v < 0.f ? r : e * r;
}
// act(v) and its derivative.  A NaN stays one: comparisons with it fall to the branch that computes with it.
template <int ACT, bool FAST>
__device__ __forceinline__ void activation(float v, float& a, float& da) {
  float z, nz;
  if (ACT == GN_ACT_RELU) {
    a = v < 0.f ? 0.f : v; da = v > 0.f ? 1.f : 0.f;
  } else if (ACT == GN_ACT_GELU) {
    const float cdf = 0.5f * erfcf(-0.70710678118654752f * v);
    a = v * cdf; da = cdf + v * 0.39894228040143268f * (FAST ? __expf(-0.5f * v * v) : expf(-0.5f * v * v));
  } else if (ACT == GN_ACT_GELU_TANH) {        // (1 + tanh q) / 2 = 1 / (1 + exp(-2 q))
    const float k = 1.5957691216057308f;       // 2 sqrt(2 / pi)
    sigmoids<FAST>(k * (v + 0.044715f * v * v * v), z, nz);
    a = v * z; da = z + v * z * nz * k * (1.f + 0.134145f * v * v);
  } else if (ACT == GN_ACT_SIGMOID) {
    sigmoids<FAST>(v, z, nz); a = z; da = z * nz;
  } else {
    sigmoids<FAST>(v, z, nz); a = v * z; da = z + v * z * nz;
  }
}
// f(integral constant) of the activation that a call names.
template <int V> struct ActIs { static constexpr int value = V; };
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
  switch (act) {
    case GN_ACT_RELU: f(ActIs<GN_ACT_RELU>{}); break;
    case GN_ACT_GELU: f(ActIs<GN_ACT_GELU>{}); break;
    case GN_ACT_GELU_TANH: f(ActIs<GN_ACT_GELU_TANH>{}); break;
    case GN_ACT_SIGMOID: f(ActIs<GN_ACT_SIGMOID>{}); break;
    default: f(ActIs<GN_ACT_SILU>{});
  }
}

template <class T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <class T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w)); }
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

}  // namespace
}  // namespace gn
