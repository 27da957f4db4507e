// Routing to experts: scores, the choice of k experts, their weights; and the backward pass.
//
// A warp has a row of logits in registers, V neighbouring experts to a lane, so that the lowest lane that holds the largest value holds the lowest expert that
// has it.  The k largest are taken one after the other: a warp's maximum of 32-bit keys is one instruction, and only the lane that gives an
// expert away looks for its next best.  16384 rows of 256 FP32 logits are 17 MB, 2.8 us of the memory's time; the instructions of
// the choice bound the kernel, not the bytes.
//
// The order of two experts has to be that of their values, whatever FP32 makes of them.  Without a bias it is the order of the logits, which are at hand.
// With one, and for sums of a group's two best, the values are computed in FP32 with a bound on what they may be off; where two neighbours in the
// order are nearer than that (and not the same logit with the same bias, which are equal in any arithmetic), the row is done again in FP64, from shared memory, in a
// function of its own that leaves the usual case its registers.
//
// The backward pass reads a whole row only where the scores are shares of all experts; else the chosen logits alone.
#include <math.h>

#include "op_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int kRouteWarps = 8, kRouteExperts = 1024, kRouteChoices = 32;
struct RouteParams {
  int64_t tokens; int experts, k, softmax, renormalise, groups, each, top, best, vec, lanes;
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

__device__ __forceinline__ float value_of(uint32_t key) { return key == 1u ? __int_as_float(0x7fffffff) : __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
__device__ __forceinline__ float warp_max_nan(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float exp_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f)); return y; }

// The k experts of a row in FP64, by a warp, from and to shared memory (an element for each expert): lane j < k returns the j-th.  Rare: few registers, no speed.
template <class T>
__device__ __noinline__ int choose_exactly(const RouteParams& p, const T* row, const float* bias, double* order, int lane) {
  const double LOW = -(double)__int_as_float(0x7f800000);
  float top = (float)LOW;
  double sum = 0.0;
  if (p.softmax) {
    for (int e = lane; e < p.experts; e += 32) top = max_nan(top, to_f(row[e]));
    top = warp_max_nan(top);
    if (top == (float)LOW) top = 0.f;
    for (int e = lane; e < p.experts; e += 32) sum += exp((double)to_f(row[e]) - (double)top);
    sum = warp_sum(sum);
    if (sum == 0.0) sum = 1.0;
  }
  const auto score = [&](int e) {
    const double l = (double)to_f(row[e]);
    return p.softmax ? exp(l - (double)top) / sum : 1.0 / (1.0 + exp(-l));
  };
  for (int e = lane; e < p.experts; e += 32) order[e] = bias ? score(e) + (double)bias[e] : (double)to_f(row[e]);
  __syncwarp();
  uint32_t kept = 0xffffffffu;
  if (p.groups > 1) {
    double first = LOW, second = LOW;
    int i1 = -1, i2 = -1;
    bool any = false;                // an element that is no NaN
    if (lane < p.groups)
      for (int e = lane * p.each; e < (lane + 1) * p.each; ++e) {
        const double x = order[e];
        if (x > first || (i1 < 0 && x == x)) { second = first; i2 = i1; first = x; i1 = e; } else if (x > second || (i2 < 0 && x == x)) { second = x; i2 = e; }
        any |= x == x;
      }
    double value = first;
    // Scores and biases by themselves: two groups that have the same ones in other pairs are equal, which roundings of four different values might not show.
    if (p.best == 2 && p.each > 1) value = i2 < 0 ? LOW : (score(i1) + score(i2)) + (bias ? (double)bias[i1] + (double)bias[i2] : 0.0);
    uint64_t g = lane < p.groups ? (any ? key_of(value) : 1u) : 0u;
    kept = 0;
    for (int j = 0; j < p.top; ++j) {
      const uint64_t m = warp_max(g);
      const int from = __ffs(__ballot_sync(0xffffffffu, g == m)) - 1;
      kept |= 1u << from;
      if (lane == from) g = 0;
    }
  }
  uint64_t best;
  int at, mine = -1;
  const auto look = [&] {
    best = 0; at = -1;
#pragma unroll 1
    for (int e = lane; e < p.experts; e += 32) {
      if (p.groups > 1 && !(kept >> (e / p.each) & 1)) continue;
      const uint64_t k = key_of(order[e]);
      if (k > best && !(__double_as_longlong(order[e]) == 0x7fffffffffffffffll)) { best = k; at = e; }
    }
  };
  look();
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    const uint64_t m = warp_max(best);
    const int e = (int)__reduce_min_sync(0xffffffffu, best == m ? (unsigned)at : 0xffffffffu);
    if (lane == j) mine = e;
    if (best == m && at == e) { order[e] = __longlong_as_double(0x7fffffffffffffffll); look(); }      // (a NaN of its own: taken)
  }
  __syncwarp();
  return mine;
}

// The same in FP32.  ORDERED: by the logits, without groups.  Whether the order is certain goes to `certain`.
template <int V, bool ORDERED, class T>
__device__ __forceinline__ int choose(const RouteParams& p, const T* row, const float (&l)[V], const float (&b)[V], const float* bias, float* stage, int lane, bool& certain) {
  constexpr float E = 5.9604645e-8f;                       // 2^-24
  const float LOW = -__int_as_float(0x7f800000);
  uint32_t key[V];
  // What a score may be off, in 2^-24.  Sigmoid: the exponential's argument (|l| s (1 - s) is below 0.23), the exponential 2, the sum and the reciprocal 1 each.
  // Softmax, of the largest score: the two roundings of the argument (|x| exp(x) is below 0.37), the exponential 2, the sum of up to 1024 of them 5 + 32, 2 more.
  float off = 8.f;
  if constexpr (!ORDERED) {
    float s[V];
    if (p.softmax) {
      float top = l[0], sum = 0.f;
#pragma unroll
      for (int v = 1; v < V; ++v) top = max_nan(top, l[v]);
      top = warp_max_nan(top);
      if (top == LOW) top = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) { s[v] = exp_fast(l[v] - top); sum += s[v]; }
      sum = warp_sum(sum);
      sum = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] *= sum;
      off = 48.f * sum;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = sigmoid_from(exp_fast(-l[v]));
    }
    const bool by_logit = !bias;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      s[v] += b[v];                                        // (from here on the values)
      key[v] = key_of(by_logit ? l[v] : s[v]);
      if (lane * V + v >= p.experts) key[v] = 0;
    }
    if (p.groups > 1) {
      const bool one = p.best == 1 || p.each == 1, plain = one && by_logit;
      float first = LOW, second = LOW;
      bool any = false;              // an element that is no NaN
      const auto take = [&](float x) { second = fmaxf(second, fminf(first, x)); first = fmaxf(first, x); any |= x == x; };
      uint32_t g, kept = 0;
      int lanes = 1;                 // to a group
      if (p.lanes) {                 // a power of two of whole lanes
        lanes = p.lanes;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float x = plain ? l[v] : s[v];
          if (x == x) take(x);
        }
        any = false;
#pragma unroll
        for (int v = 0; v < V; ++v) any |= (plain ? l[v] : s[v]) == (plain ? l[v] : s[v]);
        for (int o = 1; o < lanes; o <<= 1) {
          const float f = __shfl_xor_sync(0xffffffffu, first, o), q = __shfl_xor_sync(0xffffffffu, second, o);
          second = fmaxf(fminf(first, f), fmaxf(second, q));
          first = fmaxf(first, f);
          any |= __shfl_xor_sync(0xffffffffu, (int)any, o) != 0;
        }
        g = lane * V < p.experts ? 2u : 0u;
      } else {                       // a lane each; rows of the stage are an odd number of elements apart
        const int pitch = p.each | 1;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int x = lane * V + v;
          if (x < p.experts) stage[x / p.each * pitch + x % p.each] = plain ? l[v] : s[v];
        }
        __syncwarp();
        if (lane < p.groups)
          for (int i = 0; i < p.each; ++i) {
            const float x = stage[lane * pitch + i];
            if (x == x) take(x);
          }
        __syncwarp();
        g = lane < p.groups ? 2u : 0u;
      }
      const float value = one ? first : first + second;
      if (g) g = any ? key_of(value) : 1u;
      float last = 0.f;
      const uint32_t span = lanes == 32 ? 0xffffffffu : (1u << lanes) - 1;
      for (int j = 0; j <= p.top && j < p.groups; ++j) {
        const uint32_t m = warp_max(g);
        const int from = __ffs(__ballot_sync(0xffffffffu, g == m)) - 1;
        const float v = value_of(m);
        if (j == p.top) {
          // two sums of two values, each a score and a bias, and their roundings
          if (!plain && last - v <= E * (4.f * off + 4.f * (fabsf(last) + fabsf(v)))) certain = false;
        } else {
          kept |= span << from;
          last = v;
          if (kept >> lane & 1) g = 0;
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (!(kept >> (p.lanes ? lane : min(lane * V + v, p.experts - 1) / p.each) & 1)) key[v] = 0;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      key[v] = key_of(l[v]);
      if (lane * V + v >= p.experts) key[v] = 0;
    }
  }

  uint32_t best;
  int at;
  const auto look = [&] {
    best = key[0]; at = 0;
#pragma unroll
    for (int v = 1; v < V; ++v)
      if (key[v] > best) { best = key[v]; at = v; }
  };
  look();
  // ORDERED, and without a bias, the keys are the values; else the first one behind the last that is not its equal is looked at too.
  const bool sure = ORDERED || !bias;
  int mine = -1, last_index = 0;
  float last = __int_as_float(0x7fffffff);
  for (int j = 0; j < p.k || !sure; ++j) {
    const uint32_t m = warp_max(best);
    if (m == 0) break;                                     // (nobody is left)
    const int from = __ffs(__ballot_sync(0xffffffffu, best == m)) - 1;
    const int index = __shfl_sync(0xffffffffu, lane * V + at, from);
    if (!sure) {
      const float value = value_of(m);
      bool same = false;
      if (last - value <= E * (2.f * off + fabsf(last) + fabsf(value))) {
        same = to_f(row[index]) == to_f(row[last_index]) && bias[index] == bias[last_index];
        if (!same) { certain = false; break; }
      }
      if (j >= p.k && !same) break;
      last = value; last_index = index;
    }
    if (lane == j && j < p.k) mine = index;
    if (lane == from) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (at == v) key[v] = 0;
      look();
    }
  }
  return mine;
}

template <class T, int V, bool ORDERED>
__global__ void __launch_bounds__(32 * kRouteWarps) route_kernel(const __grid_constant__ RouteParams p) {
  extern __shared__ double stages[];                       // (an element for each expert and for each group)
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double* const stage = stages + warp * (p.experts + p.groups);
  const T* const logits = (const T*)dep(p.logits);
  const float* const bias = dep(p.bias);
  float b[V];
#pragma unroll
  for (int v = 0; v < V; ++v) b[v] = !ORDERED && bias && lane * V + v < p.experts ? bias[lane * V + v] : 0.f;
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.tokens; t += (int64_t)gridDim.x * kRouteWarps) {
    const T* const row = logits + t * p.ld;
    float l[V];
    load_row<V, T>(row, lane, p.experts, p.vec, l);
    bool certain = true;
    int index = choose<V, ORDERED, T>(p, row, l, b, bias, reinterpret_cast<float*>(stage), lane, certain);
    if (!ORDERED && !certain) index = choose_exactly<T>(p, row, bias, stage, lane);
    const bool mine = lane < p.k;
    const float z = mine ? to_f(row[index]) : 0.f;
    float w;
    if (p.softmax) {
      float top = l[0], sum = 0.f;
#pragma unroll
      for (int v = 1; v < V; ++v) top = max_nan(top, l[v]);
      top = warp_max_nan(top);
      if (top == -__int_as_float(0x7f800000)) top = 0.f;
      w = mine ? expf(z - top) : 0.f;
      if (p.renormalise) {
        sum = w;
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) sum += expf(l[v] - top);
      }
      sum = warp_sum(sum);
      w = sum == 0.f ? 0.f : w / sum;
    } else {
      w = mine ? 1.f / (1.f + expf(-z)) : 0.f;
      if (p.renormalise) {
        const float sum = warp_sum(w);
        w = sum == 0.f ? 0.f : w / sum;
      }
    }
    if (mine) {
      p.index[t * p.k + lane] = index;
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
  const int smem = kRouteWarps * (p.experts + p.groups) * 8;
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
  // lanes of a group where they are whole and a power of two
  p.lanes = p.groups > 1 && p.each % v == 0 && (p.each / v & (p.each / v - 1)) == 0 ? p.each / v : 0;
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
