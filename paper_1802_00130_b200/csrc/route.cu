// Routing to experts: scores, the choice of k experts, their weights; and the backward pass.
//
// A warp has a row of logits in registers, V neighbouring experts to a lane, so that the lowest lane that holds the largest value holds the lowest expert that
// has it.  The k largest are taken one after the other: a warp's maximum of 32-bit keys is one instruction, and only the lane that gives an
// expert away looks for its next best.  16384 rows of 256 FP32 logits are 17 MB, 2.8 us of the memory's time; the instructions of
// the choice bound the kernel, not the bytes.
//
// The order of two experts has to be that of their values, whatever FP32 makes of them.  Without a bias it is the order of the logits, which are at hand.
// With one, and for sums of a group's two best, the values are computed in FP32 with a bound on what they may be off; where two neighbours in the
// order are nearer than that (and not the same logit with the same bias, which are equal in any arithmetic), the row is done again in FP64.
//
// The backward pass reads a whole row only where the scores are shares of all experts; else the chosen logits alone.
#include <math.h>

#include "op_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int kRouteWarps = 8, kRouteExperts = 1024, kRouteChoices = 32;
struct RouteParams {
  int64_t tokens; int experts, k, softmax, renormalise, groups, each, top, best, vec;
  float scale;
  const void* logits; int64_t ld;
  const float* bias;
  int* index; float* weight;
  const float* dweight; void* dlogits; int64_t ld_d;
};

// Keys that order as the values do; NaN below every number, and 0 is nobody.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);             // (-0 is 0)
  return v != v ? 1u : u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return v != v ? 1u : u >> 63 ? ~u : u | 0x8000000000000000u;
}
__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(0xffffffffu, k); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
  const uint32_t high = warp_max((uint32_t)(k >> 32));
  const uint32_t low = warp_max((uint32_t)(k >> 32) == high ? (uint32_t)k : 0u);
  return (uint64_t)high << 32 | low;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

// This lane's V logits of a row; -inf where there is no expert.
template <int V, class T>
__device__ __forceinline__ void load_row(const T* row, int lane, int experts, bool vec, float (&l)[V]) {
  const int e0 = lane * V;
  constexpr int BYTES = V * (int)sizeof(T);
  if (vec) {                         // (experts is a multiple of V, and V elements lie in one piece on a boundary of their own size, or of 16 bytes)
    if (e0 >= experts) {
#pragma unroll
      for (int v = 0; v < V; ++v) l[v] = -__int_as_float(0x7f800000);
      return;
    }
    if constexpr (BYTES >= 16) {
#pragma unroll
      for (int q = 0; q < BYTES / 16; ++q) {
        Pack<T> p;
        p.w = *(reinterpret_cast<const uint4*>(row + e0) + q);
#pragma unroll
        for (int i = 0; i < Pack<T>::V; ++i) l[q * Pack<T>::V + i] = p.get(i);
      }
      return;
    } else if constexpr (BYTES == 8) {
      const uint2 w = *reinterpret_cast<const uint2*>(row + e0);
      Pack<T> p;
      p.w = make_uint4(w.x, w.y, 0u, 0u);
#pragma unroll
      for (int v = 0; v < V; ++v) l[v] = p.get(v);
      return;
    } else if constexpr (BYTES == 4) {
      Pack<T> p;
      p.w = make_uint4(*reinterpret_cast<const uint32_t*>(row + e0), 0u, 0u, 0u);
#pragma unroll
      for (int v = 0; v < V; ++v) l[v] = p.get(v);
      return;
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) l[v] = e0 + v < experts ? to_f(row[e0 + v]) : -__int_as_float(0x7f800000);
}

// What lane j < k has of the j-th chosen expert.
struct Chosen { int index; float logit; };

// Scores of this lane's experts.  A row of -inf alone has zeros.
template <int V, class F>
__device__ __forceinline__ void scores_of(const float (&l)[V], bool softmax, int lane, int experts, F (&s)[V]) {
  if (softmax) {
    float top = l[0];
#pragma unroll
    for (int v = 1; v < V; ++v) top = max_nan(top, l[v]);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -__int_as_float(0x7f800000)) top = 0.f;
    F sum = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) { s[v] = exp_of((F)l[v] - (F)top); sum += s[v]; }
    sum = warp_sum(sum);
    if (sum == (F)0) sum = 1;
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] /= sum;
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = (F)1 / ((F)1 + exp_of(-(F)l[v]));
  }
}

// The choice in arithmetic F.  ORDERED: by the logits, without groups.  Returns whether it is certain (always in FP64).
template <class F, int V, bool ORDERED>
__device__ __forceinline__ bool choose(const RouteParams& p, const float (&l)[V], const float* bias, F* stage, int lane, Chosen& c) {
  using Key = decltype(key_of(F()));
  constexpr bool EXACT = sizeof(F) == 8;
  constexpr float E = 5.9604645e-8f;                       // 2^-24
  F s[V];
  float b[V];
  Key key[V];
  if constexpr (!ORDERED) {
    scores_of<V, F>(l, p.softmax, lane, p.experts, s);
#pragma unroll
    for (int v = 0; v < V; ++v) b[v] = bias && lane * V + v < p.experts ? bias[lane * V + v] : 0.f;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (ORDERED) key[v] = key_of((F)l[v]);
    else key[v] = bias ? key_of(s[v] + (F)b[v]) : key_of((F)l[v]);
    if (lane * V + v >= p.experts) key[v] = 0;
  }
  bool certain = true;
  if (!ORDERED && p.groups > 1) {
    // Values of the groups, a lane each; rows of the stage are an odd number of elements apart.
    const int pitch = p.each | 1;
    const bool by_logit = p.best == 1 && !bias;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int x = lane * V + v;
      if (x < p.experts) stage[x / p.each * pitch + x % p.each] = by_logit ? (F)l[v] : s[v] + (F)b[v];
    }
    __syncwarp();
    // (NaN, as a group's best, is below every number: it loses against the -inf that a sum starts from)
    const F low = -(F)__int_as_float(0x7f800000);
    F first = low, second = low;
    int i1 = 0, i2 = 0;
    bool any = false;                // an element that is no NaN
    if (lane < p.groups)
      for (int i = 0; i < p.each; ++i) {
        const F x = stage[lane * pitch + i];
        if (x > first) { second = first; first = x; i2 = i1; i1 = i; } else if (x > second) { second = x; i2 = i; }
        any |= x == x;
      }
    __syncwarp();
    F value = p.best == 2 && p.each > 1 ? first + second : first;
    if (EXACT && p.best == 2 && p.each > 1) {
      // Scores and biases by themselves: two groups that have the same ones in other pairs are equal, which roundings of four different values might not show.
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int x = lane * V + v;
        if (x < p.experts) stage[x / p.each * pitch + x % p.each] = s[v];
      }
      __syncwarp();
      if (lane < p.groups && first > low && second > low) {
        const int e0 = lane * p.each;
        value = (stage[lane * pitch + i1] + stage[lane * pitch + i2]) + (bias ? (F)bias[e0 + i1] + (F)bias[e0 + i2] : (F)0);
      }
      __syncwarp();
    }
    Key g = lane < p.groups ? (any ? key_of(value) : (Key)1) : (Key)0;
    uint32_t kept = 0;
    F last = 0;
    for (int j = 0; j <= p.top && j < p.groups; ++j) {
      const Key m = warp_max(g);
      const int from = __ffs(__ballot_sync(0xffffffffu, g == m)) - 1;
      const F mine = __shfl_sync(0xffffffffu, value, from);
      if (j == p.top) {
        // two sums of two scores, each score off by 150 steps of itself at most (see below), and the biases' roundings
        const float gap = (float)(last - mine), bound = E * (300.f * 2.f + 4.f * (fabsf((float)last) + fabsf((float)mine)));
        if (!EXACT && !by_logit && gap <= bound) certain = false;
      } else {
        kept |= 1u << from;
        last = mine;
        if (lane == from) g = 0;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (!(kept >> (min(lane * V + v, p.experts - 1) / p.each) & 1)) key[v] = 0;
  }

  Key best;
  int at;
  const auto look = [&] {
    best = key[0]; at = 0;
#pragma unroll
    for (int v = 1; v < V; ++v)
      if (key[v] > best) { best = key[v]; at = v; }
  };
  look();
  c = Chosen{-1, 0.f};
  // ORDERED, and without a bias, the keys are the values; else the first one behind the last that is not its equal is looked at too.
  const bool sure = ORDERED || EXACT || !bias;
  float last_l = 0.f, last_s = 0.f, last_b = 0.f;
  for (int j = 0; j < p.k || !sure; ++j) {
    const Key m = warp_max(best);
    if (m == 0) break;                                     // (nobody is left)
    const int from = __ffs(__ballot_sync(0xffffffffu, best == m)) - 1;
    float mine_l = l[0], mine_s = 0.f, mine_b = 0.f;
    if constexpr (!ORDERED) { mine_s = (float)s[0]; mine_b = b[0]; }
#pragma unroll
    for (int v = 1; v < V; ++v)
      if (at == v) {
        mine_l = l[v];
        if constexpr (!ORDERED) { mine_s = (float)s[v]; mine_b = b[v]; }
      }
    const int index = __shfl_sync(0xffffffffu, lane * V + at, from);
    const float logit = __shfl_sync(0xffffffffu, mine_l, from);
    if (!sure) {
      const float score = __shfl_sync(0xffffffffu, mine_s, from), by = __shfl_sync(0xffffffffu, mine_b, from);
      const bool same = logit == last_l && by == last_b;
      // A score is off by at most 150 steps of itself: the sum of up to 1024 exponentials by 5 + 32 + 2 of them, an exponential by 2 and, with its argument's
      // rounding, as many as the argument is large, 103 before it is zero; the division by 1.  A value by its own rounding besides.
      const float value = score + by, last = last_s + last_b;
      if (j > 0 && !same && last - value <= E * (150.f * (last_s + score) + fabsf(last) + fabsf(value))) { certain = false; break; }
      if (j >= p.k && !same) break;
      last_l = logit; last_s = score; last_b = by;
    }
    if (lane == j && j < p.k) { c.index = index; c.logit = logit; }
    if (lane == from) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (at == v) key[v] = 0;
      look();
    }
  }
  return certain;
}

// (by itself, so that the usual case keeps its registers)
template <int V>
__device__ __noinline__ Chosen choose_exactly(const RouteParams& p, const float (&l)[V], const float* bias, double* stage, int lane) {
  Chosen c;
  choose<double, V, false>(p, l, bias, stage, lane, c);
  return c;
}

template <class T, int V, bool ORDERED>
__global__ void __launch_bounds__(32 * kRouteWarps) route_kernel(const __grid_constant__ RouteParams p) {
  extern __shared__ double stages[];                       // (groups: an element for each expert and for each group)
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double* const stage = stages + warp * (p.experts + p.groups);
  const T* const logits = (const T*)dep(p.logits);
  const float* const bias = dep(p.bias);
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.tokens; t += (int64_t)gridDim.x * kRouteWarps) {
    float l[V];
    load_row<V, T>(logits + t * p.ld, lane, p.experts, p.vec, l);
    Chosen c;
    if (!choose<float, V, ORDERED>(p, l, bias, reinterpret_cast<float*>(stage), lane, c)) {
      if constexpr (!ORDERED) {
        float copy[V];               // (of which the call takes an address)
#pragma unroll
        for (int v = 0; v < V; ++v) copy[v] = l[v];
        c = choose_exactly<V>(p, copy, bias, stage, lane);
      }
    }
    float w;
    const bool mine = lane < p.k;
    if (p.softmax) {
      float top = l[0], sum = 0.f;
#pragma unroll
      for (int v = 1; v < V; ++v) top = max_nan(top, l[v]);
#pragma unroll
      for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (top == -__int_as_float(0x7f800000)) top = 0.f;
      w = mine ? expf(c.logit - top) : 0.f;
      if (p.renormalise) {
        sum = w;
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) sum += expf(l[v] - top);
      }
      sum = warp_sum(sum);
      w = sum == 0.f ? 0.f : w / sum;
    } else {
      w = mine ? 1.f / (1.f + expf(-c.logit)) : 0.f;
      if (p.renormalise) {
        const float sum = warp_sum(w);
        w = sum == 0.f ? 0.f : w / sum;
      }
    }
    if (mine) {
      p.index[t * p.k + lane] = c.index;
      p.weight[t * p.k + lane] = w * p.scale;
    }
  }
}

// WHOLE: softmax over all experts; else what is not chosen has no gradient.
template <class T, int V, bool WHOLE>
__global__ void __launch_bounds__(32 * kRouteWarps) route_grad_kernel(const __grid_constant__ RouteParams p) {
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* const logits = (const T*)dep(p.logits);
  const int* const index = dep(p.index);
  const float* const dweight = dep(p.dweight);
  const float NONE = -__int_as_float(0x7f800000);
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.tokens; t += (int64_t)gridDim.x * kRouteWarps) {
    const T* const row = logits + t * p.ld;
    T* const out = (T*)p.dlogits + t * p.ld_d;
    int at = -1;
    float u = 0.f, z = NONE;
    if (lane < p.k) {
      at = index[t * p.k + lane];
      u = dweight[t * p.k + lane] * p.scale;
    }
    const bool in = at >= 0 && at < p.experts;             // (an expert that there is not takes no part)
    if (in) z = to_f(row[at]);
    float s = 0.f, l[V], top = 0.f, sum = 1.f;
    if (p.softmax) {
      top = z;
      if constexpr (WHOLE) {
        load_row<V, T>(row, lane, p.experts, p.vec, l);
#pragma unroll
        for (int v = 0; v < V; ++v) top = max_nan(top, l[v]);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (top == NONE) top = 0.f;
      s = in ? expf(z - top) : 0.f;
      if constexpr (WHOLE) {
        sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) { l[v] = expf(l[v] - top); sum += l[v]; }
        sum = warp_sum(sum);
        sum = sum == 0.f ? 0.f : 1.f / sum;
        s *= sum;
      }
    } else if (in) {
      s = 1.f / (1.f + expf(-z));
    }
    float d;                         // dL/dlogit of this lane's expert, of this choice alone
    float dot = 0.f;
    if (p.renormalise) {
      const float total = warp_sum(s), share = total == 0.f ? 0.f : s / total;
      dot = warp_sum(in ? u * share : 0.f);
      const float g = share * (u - dot);
      d = p.softmax ? g : g / (1.f + expf(z));             // (share (1 - s) (u - dot); 1 - s = 1 / (1 + exp(z)))
      dot = 0.f;
    } else if (p.softmax) {
      dot = warp_sum(in ? u * s : 0.f);
      d = s * u;
    } else {
      d = s * u / (1.f + expf(z));
    }
    if (!in) d = 0.f;
    // what is chosen twice has both
    float all = 0.f;
    for (int j = 0; j < p.k; ++j) {
      const int other = __shfl_sync(0xffffffffu, at, j);
      const float theirs = __shfl_sync(0xffffffffu, d, j);
      if (other == at) all += theirs;
    }
    if (p.vec) {
      constexpr int BYTES = V * (int)sizeof(T);
      if (lane * V < p.experts) {
        float o[V];
#pragma unroll
        for (int v = 0; v < V; ++v) o[v] = WHOLE ? -(l[v] * sum) * dot : 0.f;
        if constexpr (BYTES >= 16) {
#pragma unroll
          for (int q = 0; q < BYTES / 16; ++q) {
            Pack<T> w;
            float part[Pack<T>::V];
#pragma unroll
            for (int i = 0; i < Pack<T>::V; ++i) part[i] = o[q * Pack<T>::V + i];
            w.set(part);
            *(reinterpret_cast<uint4*>(out + lane * V) + q) = w.w;
          }
        } else {
#pragma unroll
          for (int v = 0; v < V; ++v) out[lane * V + v] = from_f<T>(o[v]);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (lane * V + v < p.experts) out[lane * V + v] = from_f<T>(WHOLE ? -(l[v] * sum) * dot : 0.f);
    }
    __syncwarp();                    // (the row is written before the chosen elements are)
    if (in) out[at] = from_f<T>(all - s * dot);
  }
}

template <class T, int V>
cudaError_t launch_route(const RouteParams& p, bool grad, cudaStream_t st) {
  const int64_t want = (p.tokens + kRouteWarps - 1) / kRouteWarps, most = (int64_t)num_sms() * 8;
  const int grid = (int)(want < most ? want : most);
  if (grad) return launch_pdl(p.softmax && !p.renormalise ? route_grad_kernel<T, V, true> : route_grad_kernel<T, V, false>, grid, 32 * kRouteWarps, 0, st, p);
  if (!p.bias && p.groups == 1) return launch_pdl(route_kernel<T, V, true>, grid, 32 * kRouteWarps, 0, st, p);
  const int smem = p.groups > 1 ? kRouteWarps * (p.experts + p.groups) * 8 : 0;
  auto* const kernel = route_kernel<T, V, false>;
  static std::atomic<signed char> ready[64];
  if (!once_per_device(ready, [&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRouteWarps * (kRouteExperts + 32) * 8) == cudaSuccess;
      }))
    return cudaErrorInvalidDevice;
  return launch_pdl(kernel, grid, 32 * kRouteWarps, smem, st, p);
}

template <class T>
cudaError_t run_route(RouteParams p, bool grad, cudaStream_t st) {
  int v = 1;
  while (32 * v < p.experts) v *= 2;
  // pieces of v elements, or of 16 bytes of them
  const auto whole = [&](const void* q, int64_t ld) {
    const int piece = v * (int)sizeof(T) < 16 ? v * (int)sizeof(T) : 16;
    return ((uintptr_t)q % (uintptr_t)piece) == 0 && ld * (int)sizeof(T) % piece == 0;
  };
  p.vec = p.experts % v == 0 && whole(p.logits, p.ld) && (!grad || whole(p.dlogits, p.ld_d));
  switch (v) {
    case 1: return launch_route<T, 1>(p, grad, st);
    case 2: return launch_route<T, 2>(p, grad, st);
    case 4: return launch_route<T, 4>(p, grad, st);
    case 8: return launch_route<T, 8>(p, grad, st);
    case 16: return launch_route<T, 16>(p, grad, st);
    default: return launch_route<T, 32>(p, grad, st);
  }
}

const char* route_args(int type, int score, int64_t tokens, int experts, int k, double scale) {
  if (!type_ok(type)) return "type is not a gn_dtype";
  if (score != GN_SOFTMAX && score != GN_SIGMOID) return "score is not a gn_score";
  if (tokens < 0 || tokens >= (int64_t(1) << 31)) return "tokens must be in [0, 2^31)";
  if (experts < 1 || experts > kRouteExperts) return "experts must be in [1, 1024]";
  if (k < 1 || k > kRouteChoices || k > experts) return "k must be in [1, 32] and not above the number of experts";
  if (!(fabs(scale) <= 3.402823466e38)) return "scale must be a finite FP32 number";
  return nullptr;
}
bool words_ok(const void* p) { return p && ((uintptr_t)p & 3) == 0; }

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" gn_status gn_route(gn_dtype type, gn_score score, int64_t tokens, int32_t experts, int32_t k, const void* d_logits, int64_t ld,
                              const float* d_bias, int32_t groups, int32_t top_groups, int32_t group_best, int32_t renormalise, double scale,
                              int32_t* d_index, float* d_weight, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = route_args(type, score, tokens, experts, k, scale);
  if (!why) {
    if (groups < 1 || groups > 32 || experts % groups) why = "groups must be in [1, 32] and divide the experts";
    else if (top_groups < 1 || top_groups > groups) why = "top_groups must be in [1, groups]";
    else if (group_best != 1 && group_best != 2) why = "group_best must be 1 or 2";
    else if (k > experts / groups * top_groups) why = "k must not be above the experts of top_groups groups";
    else if ((uintptr_t)d_bias & 3) why = "bias is not aligned to 4 bytes";
    else if (tokens > 0) {
      if (!mat_ok(d_logits, ld, experts, type)) why = "logits: null, misaligned, or a leading dimension below the number of experts";
      else if (!words_ok(d_index) || !words_ok(d_weight)) why = "index or weight: null or misaligned";
    }
  }
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  if (tokens == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  RouteParams p = {};
  p.tokens = tokens; p.experts = experts; p.k = k; p.softmax = score == GN_SOFTMAX; p.renormalise = renormalise != 0;
  // (all groups are kept: there is nothing to choose between)
  p.groups = top_groups == groups ? 1 : groups; p.each = experts / p.groups; p.top = top_groups; p.best = group_best; p.scale = (float)scale;
  p.logits = d_logits; p.ld = ld; p.bias = d_bias; p.index = d_index; p.weight = d_weight;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return op_done(type == GN_F32 ? run_route<float>(p, false, st) : type == GN_BF16 ? run_route<__nv_bfloat16>(p, false, st) : run_route<__half>(p, false, st),
                 errbuf, errbuf_len);
}

extern "C" gn_status gn_route_grad(gn_dtype type, gn_score score, int64_t tokens, int32_t experts, int32_t k, const float* d_dweight,
                                   const void* d_logits, int64_t ld, const int32_t* d_index, int32_t renormalise, double scale, void* d_dlogits,
                                   int64_t ld_d, void* cuda_stream, char* errbuf, int64_t errbuf_len) {
  const char* why = route_args(type, score, tokens, experts, k, scale);
  if (!why && tokens > 0) {
    if (!mat_ok(d_logits, ld, experts, type)) why = "logits: null, misaligned, or a leading dimension below the number of experts";
    else if (!mat_ok(d_dlogits, ld_d, experts, type)) why = "dlogits: null, misaligned, or a leading dimension below the number of experts";
    else if (d_dlogits == d_logits) why = "dlogits must not be in the place of the logits";
    else if (!words_ok(d_index) || !words_ok(d_dweight)) why = "index or dweight: null or misaligned";
  }
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  if (tokens == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  RouteParams p = {};
  p.tokens = tokens; p.experts = experts; p.k = k; p.softmax = score == GN_SOFTMAX; p.renormalise = renormalise != 0; p.groups = 1; p.each = experts;
  p.scale = (float)scale; p.logits = d_logits; p.ld = ld; p.index = const_cast<int*>(d_index); p.dweight = d_dweight; p.dlogits = d_dlogits; p.ld_d = ld_d;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return op_done(type == GN_F32 ? run_route<float>(p, true, st) : type == GN_BF16 ? run_route<__nv_bfloat16>(p, true, st) : run_route<__half>(p, true, st),
                 errbuf, errbuf_len);
}
