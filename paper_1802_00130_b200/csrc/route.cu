// Routing to experts: scores, the choice of k experts, their weights; and the backward pass.
//
// A warp has a row of logits in registers, V neighbouring experts to a lane, so that the lowest lane that holds the largest value holds the lowest expert that
// has it.  The k largest are taken one after the other: a warp's maximum of 32-bit keys is one instruction, and only the lane that gives an
// expert away looks for its next best.  16384 rows of 256 FP32 logits are 17 MB, 2.8 us of the memory's time; the instructions of the choice bound the kernel, not
// the bytes: 10 us for the best one without a bias, 15 for eight, 22 with a bias, 27 with groups as well, and 32 where the rows come from memory (1240 instructions a row, half of them on the pipe of half the rate).
//
// The order of two experts has to be that of their values, whatever FP32 makes of them.  Without a bias it is the order of the logits, which are at hand.
// With one, and for sums of a group's two best, the values are computed in FP32 with a bound on what they may be off; where two neighbours in the
// order are nearer than that (and not the same logit with the same bias, which are equal in any arithmetic), the row is done again in FP64, from shared memory, in a
// function of its own that leaves the usual case its registers.
//
// The backward pass reads a whole row only where the scores are shares of all experts; else the chosen logits alone: 8 us for 16384 rows of 256, 17 MB written.
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
  return v != v ? 1u : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
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
// The largest z of the lanes that are `in` (NaN: none is a number).
__device__ __forceinline__ float warp_largest(float z, bool in) { return value_of(warp_max(in ? key_of(z) : 0u)); }
// sigmoid(z) of the lanes that are `in`, 0 of the others, times exp(-m) where the largest z, m, is negative: numbers in the proportions of the scores, all of which may be below FP32's smallest.
// From exp(-700) down, where 64 bits end too, they are 0 all the same: a row that is masked by a type's lowest value instead of -inf has no shares either.  rest = 1 - sigmoid(z).
__device__ __forceinline__ float sigmoid_share(float z, float m, bool in, float& rest) {
  const float e = expf(-fabsf(z)), r = 1.f / (1.f + e);
  rest = z < 0.f ? r : e * r;
  return !in ? 0.f : z < 0.f ? (m < 0.f && m >= -700.f ? expf(z - m) : e) * r : r;
}
__device__ __forceinline__ float exp_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f)); return y; }

// Scores in FP64: of a row whose largest logit (0 if that is -inf) and sum of exponentials are known.
struct Exact { float top; double sum; };
template <class T>
__device__ __forceinline__ Exact exact_of(const RouteParams& p, const T* row, int lane) {
  Exact x{-__int_as_float(0x7f800000), 0.0};
  if (!p.softmax) return x;
  for (int e = lane; e < p.experts; e += 32) x.top = max_nan(x.top, to_f(row[e]));
  x.top = warp_max_nan(x.top);
  if (x.top == -__int_as_float(0x7f800000)) x.top = 0.f;
#pragma unroll 4
  for (int e = lane; e < p.experts; e += 32) x.sum += exp((double)to_f(row[e]) - (double)x.top);
  x.sum = warp_sum(x.sum);
  if (x.sum == 0.0) x.sum = 1.0;
  return x;
}
__device__ __forceinline__ double exact_score(const RouteParams& p, const Exact& x, float l) {
  return p.softmax ? exp((double)l - (double)x.top) / x.sum : 1.0 / (1.0 + exp(-(double)l));
}

// The order in FP64 of n experts (one to a lane, bias included): lane j < k returns the j-th.
template <class T>
__device__ __noinline__ int order_exactly(const RouteParams& p, const T* row, const float* bias, int index, int n, int lane) {
  const Exact x = exact_of(p, row, lane);
  const bool on = lane < n;
  const uint64_t key = on ? key_of(exact_score(p, x, to_f(row[index])) + (double)bias[index]) : 0u;
  int rank = 0, mine = -1;
  for (int i = 0; i < n; ++i) {
    const uint64_t k = __shfl_sync(0xffffffffu, key, i);
    const int e = __shfl_sync(0xffffffffu, index, i);
    rank += k > key || (k == key && e < index);
  }
  for (int i = 0; i < n; ++i) {
    const int r = __shfl_sync(0xffffffffu, rank, i), e = __shfl_sync(0xffffffffu, index, i);
    if (r == lane) mine = e;
  }
  return mine;
}

// The k experts of a row in FP64, by a warp, from and to shared memory (an element for each expert): lane j < k returns the j-th.  Rare: few registers, no speed.
template <class T>
__device__ __noinline__ int choose_exactly(const RouteParams& p, const T* row, const float* bias, double* order, int lane) {
  const double LOW = -(double)__int_as_float(0x7f800000);
  const Exact exact = exact_of(p, row, lane);
  const auto score = [&](int e) { return exact_score(p, exact, to_f(row[e])); };
#pragma unroll 4
  for (int e = lane; e < p.experts; e += 32) order[e] = bias ? score(e) + (double)bias[e] : (double)to_f(row[e]);
  __syncwarp();
  const double TAKEN = __longlong_as_double(0x7fffffffffffffffll);       // (a NaN of its own: nobody any more)
  if (p.groups > 1) {
    // Lanes in turn take a group's elements, two groups' halves at a time where there are lanes for it: here a power of two of lanes to a group.
    int lanes = 1;
    while (2 * lanes * p.groups <= 32) lanes *= 2;
    const int group = lane / lanes, sub = lane % lanes;
    double first = LOW, second = LOW;
    int i1 = -1, i2 = -1;
    const auto better = [](double x, int i, double y, int j) { return j < 0 || (i >= 0 && (x > y || (x == y && i < j))); };
    const auto merge = [&](double x, int i) {
      if (i < 0) return;
      if (better(x, i, first, i1)) { second = first; i2 = i1; first = x; i1 = i; } else if (better(x, i, second, i2)) { second = x; i2 = i; }
    };
    if (group < p.groups)
#pragma unroll 4
      for (int i = sub; i < p.each; i += lanes) {
        const double x = order[group * p.each + i];
        merge(x, x == x ? group * p.each + i : -1);
      }
    for (int o = 1; o < lanes; o <<= 1) {
      const double f = __shfl_xor_sync(0xffffffffu, first, o), q = __shfl_xor_sync(0xffffffffu, second, o);
      const int i = __shfl_xor_sync(0xffffffffu, i1, o), j = __shfl_xor_sync(0xffffffffu, i2, o);
      merge(f, i); merge(q, j);
    }
    double value = first;
    // Scores and biases by themselves: two groups that have the same ones in other pairs are equal, which roundings of four different values might not show.
    if (p.best == 2 && p.each > 1) value = i2 < 0 ? LOW : (score(i1) + score(i2)) + (bias ? (double)bias[i1] + (double)bias[i2] : 0.0);
    uint64_t g = group < p.groups && sub == 0 ? key_of(value) : 0u;
    uint32_t kept = 0;
    for (int j = 0; j < p.top; ++j) {
      const uint64_t m = warp_max(g);
      const int from = __ffs(__ballot_sync(0xffffffffu, g == m)) - 1;
      kept |= 1u << (from / lanes);
      if (lane == from) g = 0;
    }
    for (int e = lane; e < p.experts; e += 32)
      if (!(kept >> (e / p.each) & 1)) order[e] = TAKEN;
    __syncwarp();
  }
  uint64_t best;
  int at, mine = -1;
  const auto look = [&] {
    best = 0; at = -1;
#pragma unroll 4
    for (int e = lane; e < p.experts; e += 32) {
      const double x = order[e];
      const uint64_t k = __double_as_longlong(x) == __double_as_longlong(TAKEN) ? 0u : key_of(x);
      if (k > best) { best = k; at = e; }
    }
  };
  look();
#pragma unroll 1
  for (int j = 0; j < p.k; ++j) {
    const uint64_t m = warp_max(best);
    const int e = (int)__reduce_min_sync(0xffffffffu, best == m ? (unsigned)at : 0xffffffffu);
    if (lane == j) mine = e;
    if (best == m && at == e) { order[e] = TAKEN; look(); }
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
      const auto take = [&](float x) {
        x = x == x ? x : LOW;        // (a NaN is nobody's best)
        second = fmaxf(second, fminf(first, x)); first = fmaxf(first, x);
      };
      uint32_t kept = 0;
      int lanes = 1;                 // to a group
      bool mine;                     // a group is this lane's
      if (p.lanes) {                 // a power of two of whole lanes
        lanes = p.lanes;
#pragma unroll
        for (int v = 0; v < V; ++v) take(plain ? l[v] : s[v]);
        for (int o = 1; o < lanes; o <<= 1) {
          const float f = __shfl_xor_sync(0xffffffffu, first, o), q = __shfl_xor_sync(0xffffffffu, second, o);
          second = fmaxf(fminf(first, f), fmaxf(second, q));
          first = fmaxf(first, f);
        }
        mine = lane * V < p.experts;
      } else {                       // a lane each; rows of the stage are an odd number of elements apart
        const int pitch = p.each | 1;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int x = lane * V + v;
          if (x < p.experts) stage[x / p.each * pitch + x % p.each] = plain ? l[v] : s[v];
        }
        __syncwarp();
        mine = lane < p.groups;
        if (mine)
          for (int i = 0; i < p.each; ++i) take(stage[lane * pitch + i]);
        __syncwarp();
      }
      // (half the sum of two, which does not overflow)
      const float value = one ? first : 0.5f * first + 0.5f * second;
      uint32_t g = mine ? key_of(value) : 0u;
      const uint32_t span = lanes == 32 ? 0xffffffffu : (1u << lanes) - 1;
      for (int j = 0; j < p.top; ++j) {
        const uint32_t m = warp_max(g);
        const int from = __ffs(__ballot_sync(0xffffffffu, g == m)) - 1;
        kept |= span << from;
        if (kept >> lane & 1) g = 0;
      }
      if (!plain) {
        // What a group's value may be off: each of its scores and the rounding of each sum, which goes by what was added, since a score's bias and another's may cancel.  Certain is a choice
        // whose lowest is above all that is left, or as far down or up as that, where no rounding is.
        const float about = E * 1.25f * (off + fabsf(first) + (one ? 0.f : fabsf(second))), err = about < __int_as_float(0x7f800000) ? about : 0.f;
        const bool in = kept >> lane & 1;
        const uint32_t low = __reduce_min_sync(0xffffffffu, mine && in ? key_of(value - err) : 0xffffffffu);
        const uint32_t high = warp_max(mine && !in ? key_of(value + err) : 0u);
        if (!(low > high || (low == high && fabsf(value_of(low)) == __int_as_float(0x7f800000)))) certain = false;
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
  // ORDERED, and without a bias, the keys are the values.  Else those behind the last are looked at until one is clearly less than it; if two neighbours are
  // too near to tell, and not equal in any arithmetic, all that may be among the first k are put in order in FP64.
  const bool sure = ORDERED || !bias;
  int mine = -1;
  uint32_t my_key = 0, m = 0;
  int from = 0;
  const auto next = [&] {            // the best that is left: its key (0: nobody) and its lane
    m = warp_max(best);
    from = __ffs(__ballot_sync(0xffffffffu, best == m)) - 1;
  };
  const auto take = [&](int n) {
    const int index = __shfl_sync(0xffffffffu, lane * V + at, from);
    if (lane == n) { mine = index; my_key = m; }
    if (lane == from) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (at == v) key[v] = 0;
      look();
    }
  };
#pragma unroll 1
  for (int n = 0; n < p.k; ++n) { next(); take(n); }
  if constexpr (!ORDERED) {
    if (sure) return mine;
    const float kth = value_of(m);
    int n = p.k;
#pragma unroll 1
    for (;; ++n) {
      next();
      if (m == 0 || !(kth - value_of(m) <= E * (2.f * off + fabsf(kth) + fabsf(value_of(m))))) break;
      if (n == 32) { certain = false; return mine; }       // (too many for a lane each)
      take(n);
    }
    const float value = value_of(my_key), after = __shfl_down_sync(0xffffffffu, value, 1);
    const bool near = lane < n - 1 && value - after <= E * (2.f * off + fabsf(value) + fabsf(after));
    if (__any_sync(0xffffffffu, near)) {
      const int behind = __shfl_down_sync(0xffffffffu, mine, 1);
      const bool differ = near && !(to_f(row[mine]) == to_f(row[behind]) && bias[mine] == bias[behind]);
      if (__any_sync(0xffffffffu, differ)) mine = order_exactly<T>(p, row, bias, mine, n, lane);
    }
  }
  return mine;
}

template <class T, int V, bool ORDERED>
__global__ void __launch_bounds__(32 * kRouteWarps, ORDERED ? 1 : V <= 8 ? 4 : 2) route_kernel(const __grid_constant__ RouteParams p) {
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
      // Shares are of the chosen alone, which a bias or the groups may have taken far below the row's largest: from the largest of them on, as the backward pass has them.
      // (A NaN or +inf anywhere in the row is one in its scores.  ORDERED, the largest is the first chosen.)
      if (!ORDERED && p.renormalise) top = top < __int_as_float(0x7f800000) ? warp_largest(z, mine) : __int_as_float(0x7fffffff);
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
      if (p.renormalise) {
        float rest;
        w = sigmoid_share(z, ORDERED ? __shfl_sync(0xffffffffu, z, 0) : warp_largest(z, mine), mine, rest);
        const float sum = warp_sum(w);
        w = sum == 0.f ? 0.f : w / sum;
      } else {
        w = mine ? 1.f / (1.f + expf(-z)) : 0.f;
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
    float s = 0.f, l[V], top = 0.f, sum = 1.f, rest = 0.f;
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
    } else if (p.renormalise) {
      s = sigmoid_share(z, warp_largest(z, in), in, rest);
    } else {
      s = in ? 1.f / (1.f + expf(-z)) : 0.f;
    }
    float d;                         // dL/dlogit of this lane's expert, of this choice alone
    float dot = 0.f;
    if (p.renormalise) {
      const float total = warp_sum(s), share = total == 0.f ? 0.f : s / total;
      dot = warp_sum(in ? u * share : 0.f);
      const float g = share * (u - dot);
      d = p.softmax ? g : g * rest;                        // (share (1 - s) (u - dot))
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

const char* route_args(const gn_router* f, bool grad) {
  if (!f) return "no arguments";
  if (!type_ok(f->type)) return "type is not a gn_dtype";
  if (f->score != GN_SOFTMAX && f->score != GN_SIGMOID) return "score is not a gn_score";
  if (f->tokens < 0 || f->tokens >= (int64_t(1) << 31)) return "tokens must be in [0, 2^31)";
  if (f->experts < 1 || f->experts > kRouteExperts) return "experts must be in [1, 1024]";
  if (f->k < 1 || f->k > kRouteChoices || f->k > f->experts) return "k must be in [1, 32] and not above the number of experts";
  if (!(fabs(f->scale) <= 3.402823466e38)) return "scale must be a finite FP32 number";
  if (!grad) {
    if (f->groups < 1 || f->groups > 32 || f->experts % f->groups) return "groups must be in [1, 32] and divide the experts";
    if (f->top_groups < 1 || f->top_groups > f->groups) return "top_groups must be in [1, groups]";
    if (f->group_best != 1 && f->group_best != 2) return "group_best must be 1 or 2";
    if (f->k > f->experts / f->groups * f->top_groups) return "k must not be above the experts of top_groups groups";
    if ((uintptr_t)f->bias & 3) return "bias is not aligned to 4 bytes";
  }
  if (f->tokens == 0) return nullptr;
  if (!mat_ok(f->logits.p, f->logits.ld, f->experts, f->type)) return "logits: null, misaligned, or a leading dimension below the number of experts";
  if (!f->index || ((uintptr_t)f->index & 3) || !f->weight || ((uintptr_t)f->weight & 3)) return "index or weight: null or misaligned";
  if (grad && !mat_ok(f->dlogits.p, f->dlogits.ld, f->experts, f->type)) return "dlogits: null, misaligned, or a leading dimension below the number of experts";
  if (grad && f->dlogits.p == f->logits.p) return "dlogits must not be in the place of the logits";
  return nullptr;
}

gn_status run(const gn_router* f, bool grad, void* stream, char* errbuf, int64_t errbuf_len) {
  const char* why = route_args(f, grad);
  if (why) return op_fail(GN_EINVAL, why, errbuf, errbuf_len);
  if (f->tokens == 0) return op_done(cudaSuccess, errbuf, errbuf_len);
  RouteParams p = {};
  p.tokens = f->tokens; p.experts = f->experts; p.k = f->k; p.softmax = f->score == GN_SOFTMAX; p.renormalise = f->renormalise != 0; p.scale = (float)f->scale;
  // (where all groups are kept there is nothing to choose between)
  p.groups = grad || f->top_groups == f->groups ? 1 : f->groups;
  p.each = f->experts / p.groups; p.top = f->top_groups; p.best = f->group_best;
  p.logits = f->logits.p; p.ld = f->logits.ld; p.bias = grad ? nullptr : f->bias; p.index = f->index; p.weight = f->weight; p.dweight = f->weight;
  p.dlogits = f->dlogits.p; p.ld_d = f->dlogits.ld;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = f->type == GN_F32 ? run_route<float>(p, grad, st) : f->type == GN_BF16 ? run_route<__nv_bfloat16>(p, grad, st) : run_route<__half>(p, grad, st);
  return op_done(e, errbuf, errbuf_len);
}

}  // namespace
}  // namespace gn

using namespace gn;

extern "C" gn_status gn_route(const gn_router* args, void* cuda_stream, char* errbuf, int64_t errbuf_len) { return run(args, false, cuda_stream, errbuf, errbuf_len); }
extern "C" gn_status gn_route_grad(const gn_router* args, void* cuda_stream, char* errbuf, int64_t errbuf_len) { return run(args, true, cuda_stream, errbuf, errbuf_len); }
