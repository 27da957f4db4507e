// The gated block's activations and their derivatives, and two 16-bit elements to a word.
#pragma once
#include "op_common.cuh"

namespace gn {
namespace {

__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rcp_fast(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// 1 / (1 + exp(-v)) and 1 / (1 + exp(v)), each to full relative accuracy: one minus the other would lose it where it is small.
// FAST: the hardware's exponential and reciprocal, off by at most (4 + |v|) 2^-23, for results that are rounded to 16 bits (2^-12 at best), and without
// a branch on the sign.  It takes v from kSigmoidLow on: exp(-v) is below 2^126 there, where its reciprocal is still a normal number and their product one.
constexpr float kSigmoidLow = -87.3f;
template <bool FAST>
__device__ __forceinline__ void sigmoids(float v, float& z, float& nz) {
  if (FAST) {
    const float e = exp2_fast(v * -1.4426950408889634f);
    z = rcp_fast(1.f + e); nz = e * z;
  } else {
    const float e = expf(-fabsf(v)), r = 1.f / (1.f + e);
    z = v < 0.f ? e * r : r; nz = v < 0.f ? r : e * r;
  }
}
// Phi(v), the normal distribution function, and exp(-v^2 / 2), each to full relative accuracy.  FAST: Phi(-|v|) exp(v^2 / 2) = t P(t) with
// t = 1 / (1 + 0.35 |v| / sqrt 2); P, of degree 7, was fitted to the smallest largest relative error over t in (0, 1], 8.2e-7 (iterated weighted least
// squares in 64 bits).  With the exponential's share that is 3e-6 up to |v| = 6 and 7e-6 up to 13.
template <bool FAST>
__device__ __forceinline__ void normal(float v, float& cdf, float& e) {
  if (FAST) {
    const float t = rcp_fast(fmaf(fabsf(v), 0.24748737341529162f, 1.f));
    e = exp2_fast(v * v * -0.72134752044448170f);
    float p = -0.04255257174372673f;
    p = fmaf(p, t, 0.1006045714020729f);
    p = fmaf(p, t, -0.007274771109223366f);
    p = fmaf(p, t, 0.08147183060646057f);
    p = fmaf(p, t, 0.07733616977930069f);
    p = fmaf(p, t, 0.09295466542243958f);
    p = fmaf(p, t, 0.0987265482544899f);
    p = fmaf(p, t, 0.09873314201831818f);
    const float q = p * t * e;
    cdf = v < 0.f ? q : 1.f - q;
  } else {
    // (the roundings of v / sqrt 2 and of v^2 come with a factor of v^2 in the tails, 45 steps at |v| = 6: taken back to first order, where e is not zero)
    const float c = -0.70710678118654752f, q = copysignf(fminf(fabsf(v), 30.f), v), s = q * q, x = c * q;
    e = expf(-0.5f * s);
    e = fmaf(-0.5f * fmaf(q, q, -s), e, e);
    cdf = fmaf(-0.56418958354775629f * e, fmaf(c, q, -x) + q * -1.2101617e-8f, 0.5f * erfcf(c * v));       // 1 / sqrt pi; what c's rounding has left
  }
}
// act(v) and its derivative.  A NaN stays one: comparisons with it fall to the branch that computes with it.
// FAST: what is so far below that sigmoids takes it no more is as the last value that it takes, v itself in v z too (they are less than 2e-36 there).
template <int ACT, bool FAST>
__device__ __forceinline__ void activation(float v, float& a, float& da) {
  float z, nz;
  if (FAST && (ACT == GN_ACT_SIGMOID || ACT == GN_ACT_SILU)) v = max_nan(v, kSigmoidLow);
  if (FAST && ACT == GN_ACT_GELU_TANH) v = max_nan(v, -9.99f);       // (2 q = -87.1)
  if (ACT == GN_ACT_RELU) {
    a = v < 0.f ? 0.f : v; da = v > 0.f ? 1.f : 0.f;
  } else if (ACT == GN_ACT_GELU) {
    normal<FAST>(v, z, nz);
    a = v * z; da = fmaf(v * nz, 0.39894228040143268f, z);
  } else if (ACT == GN_ACT_GELU_TANH) {        // (1 + tanh q) / 2 = 1 / (1 + exp(-2 q)), q = sqrt(2 / pi) (v + 0.044715 v^3)
    const float s = v * v;
    sigmoids<FAST>(v * fmaf(s, 0.071354816272810f, 1.5957691216057308f), z, nz);
    // (beyond |v| = 100, where z nz is zero, v^2 is bounded: it would overflow, and zero times infinity is not zero)
    a = v * z; da = fmaf(a * nz, fmaf(fminf(s, 1e4f), 0.214064448818430f, 1.5957691216057308f), z);
  } else if (ACT == GN_ACT_SIGMOID) {
    sigmoids<FAST>(v, z, nz); a = z; da = z * nz;
  } else {
    sigmoids<FAST>(v, z, nz); a = v * z; da = fmaf(a, nz, z);
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
