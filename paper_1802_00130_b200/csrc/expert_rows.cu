// What a mixture of experts does with rows beside its products: the order of the pairs by expert, tokens to their slots, the pairs' results back to tokens.
//
// The order is a counting sort that keeps the pairs of an expert in their own order, so that every sum has one order: a block counts the experts of its pairs;
// then each block adds up what the blocks before it have counted, and places its own.  Up to 1024 pairs are one block and one launch.  Bound by latency: 4 and 8 us for 32768 pairs
// of 64 experts, 5 for 64 pairs.
#include "expert_kernels.h"
#include "op_common.cuh"
#include "tc_common.cuh"

namespace gn {
namespace {

constexpr int kPlanThreads = 1024, kPlanWarps = 32;

// Sum of a over the threads before this one, and over all of them (n_warps full warps).
__device__ __forceinline__ int before_me(int a, int* warps, int n_warps, int& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = a;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
  __syncthreads();
  if (lane == 31) warps[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int s = lane < n_warps ? warps[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += y; }
    warps[lane] = s;
  }
  __syncthreads();
  all = warps[31];
  return x - a + (warp ? warps[warp - 1] : 0);
}

struct PlanParams { const int* index; ExpertPlan plan; int64_t chunk; int height; };

__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const __grid_constant__ PlanParams p) {
  __shared__ int count[kMostExperts];
  grid_dep_wait();
  grid_dep_launch();
  const int* const index = dep(p.index);
  const int E = p.plan.experts;
  for (int e = threadIdx.x; e < E; e += kPlanThreads) count[e] = 0;
  __syncthreads();
  const int64_t from = blockIdx.x * p.chunk, to = min(from + p.chunk, p.plan.pairs);
  for (int64_t i = from + threadIdx.x; i < to; i += kPlanThreads) {
    const int e = index[i];
    if ((unsigned)e < (unsigned)E) atomicAdd(&count[e], 1);        // (a count: the order of additions does not matter)
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kPlanThreads) p.plan.hist[(int64_t)blockIdx.x * E + e] = count[e];
}

// ONE: the grid is one block of up to kPlanThreads pairs, which counts for itself.
template <bool ONE>
__global__ void __launch_bounds__(kPlanThreads) plan_place_kernel(const __grid_constant__ PlanParams p) {
  extern __shared__ uint16_t of_warp[];          // [warps][experts]: pairs of a round's warps, then of the warps before
  __shared__ int base[kMostExperts], warps[kPlanWarps];
  grid_dep_wait();
  grid_dep_launch();
  const int* const index = dep(p.index);
  const int E = p.plan.experts, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = ONE ? (int)blockDim.x : kPlanThreads, n_warps = threads >> 5;
  const int64_t from = ONE ? 0 : blockIdx.x * p.chunk, to = ONE ? p.plan.pairs : min(from + p.chunk, p.plan.pairs);
  int before = 0, mine = 0;                      // thread e: pairs of expert e in the blocks before, in all
  const auto round = [&](int64_t i0, auto first) {
    for (int i = threadIdx.x; i < n_warps * E; i += threads) of_warp[i] = 0;
    __syncthreads();
    const int64_t i = i0 + threadIdx.x;
    int e = i < to ? index[i] : -1;
    if ((unsigned)e >= (unsigned)E) e = -1;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    const int rank = __popc(same & ((1u << lane) - 1));
    if (e >= 0 && rank == 0) of_warp[warp * E + e] = (uint16_t)__popc(same);
    __syncthreads();
    int sum = 0;
    if (threadIdx.x < E)
      for (int w = 0; w < n_warps; ++w) {
        const int n = of_warp[w * E + threadIdx.x];
        of_warp[w * E + threadIdx.x] = (uint16_t)sum;
        sum += n;
      }
    first(sum);
    __syncthreads();
    if (i < to) {
      const int slot = e < 0 ? -1 : base[e] + of_warp[warp * E + e] + rank;
      p.plan.slot_of[i] = slot;
      if (slot >= 0) p.plan.pair_of[slot] = (int)i;
    }
    __syncthreads();
    if (threadIdx.x < E) base[threadIdx.x] += sum;
  };
  const auto lay_out = [&] {
    int slots, tiles;
    const int padded = (mine + kSlots - 1) / kSlots * kSlots, n = (mine + p.height - 1) / p.height;
    const int start = before_me(padded, warps, n_warps, slots), tile = before_me(n, warps, n_warps, tiles);
    if (threadIdx.x < E) base[threadIdx.x] = start + before;
    if (blockIdx.x == 0) {
      if (threadIdx.x < E) {
        const int e = threadIdx.x;
        p.plan.start[e] = start; p.plan.count[e] = mine;
        for (int i = mine; i < padded; ++i) p.plan.pair_of[start + i] = -1;
        for (int i = 0; i < n; ++i)
          p.plan.tiles[tile + i] = ExpertTile{e, start + i * p.height, min(p.height, mine - i * p.height), min(p.height, padded - i * p.height)};
      }
      if (threadIdx.x == 0) *p.plan.n_tiles = tiles;
    }
    __syncthreads();
  };
  if (ONE) {
    round(0, [&](int sum) { mine = sum; lay_out(); });
    return;
  }
  if (threadIdx.x < E) {
    const int* const hist = dep(p.plan.hist) + threadIdx.x;
#pragma unroll 8
    for (int b = 0; b < gridDim.x; ++b) {
      const int n = hist[(int64_t)b * E];
      mine += n;
      if (b < blockIdx.x) before += n;
    }
  }
  lay_out();
  for (int64_t i0 = from; i0 < to; i0 += kPlanThreads) round(i0, [](int) {});
}

// Blocks of a plan: of 1024 pairs at least, and no more of them than SMs, since each reads what all have counted.
int64_t plan_chunk(int64_t pairs) {
  const int64_t rounds = (pairs + kPlanThreads - 1) / kPlanThreads, each = (rounds + 147) / 148;
  return (each > 0 ? each : 1) * kPlanThreads;
}

// ---- tokens to slots ----------------------------------------------------------------------------
constexpr int kCopies = 2;
struct CopyParams {
  RowCopy c[kCopies]; int vec[kCopies];
  int64_t tokens; int k, row_bytes, zero, units;           // zero: experts whose empty slots are written
  ExpertPlan plan;
};
// Bound by its bytes: 8192 tokens of 2048 BF16 columns to 4 slots each, 168 MB, 27 us (6.3 TB/s).
// A warp takes 1 KB of a token's row at a time (two 16-byte units a lane) and writes it to the token's k slots; the warps behind the tokens' zero the experts' empty slots (where
// they are terms of a sum).
__global__ void __launch_bounds__(256) to_slots_kernel(const __grid_constant__ CopyParams p) {
  grid_dep_wait();
  grid_dep_launch();
  const RowCopy& c = p.c[blockIdx.y];
  const bool vec = p.vec[blockIdx.y] != 0;
  const int* const slot_of = dep(p.plan.slot_of);
  const int lane = threadIdx.x & 31;
  const int64_t work = (p.tokens + p.zero) * p.units;
  for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < work; w += (int64_t)gridDim.x * 8) {
    const int64_t t = w / p.units;
    const int unit = (int)(w - t * p.units), at = unit * 1024 + lane * 16;
    char* const dst = (char*)c.dst;
    const int64_t ld = c.ld_dst * 2;
    if (t >= p.tokens) {
      const int e = (int)(t - p.tokens), n = p.plan.count[e], end = (n + kSlots - 1) / kSlots * kSlots;
      for (int i = n; i < end; ++i) {
        char* const to = dst + (p.plan.start[e] + i) * ld + at;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (at + h * 512 < p.row_bytes) *reinterpret_cast<uint4*>(to + h * 512) = make_uint4(0u, 0u, 0u, 0u);
      }
      continue;
    }
    const char* const src = (const char*)dep(c.src) + t * c.ld * 2 + at;
    uint4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v[h] = make_uint4(0u, 0u, 0u, 0u);
      const int left = p.row_bytes - at - h * 512;
      if (left <= 0) continue;
      if (vec && left >= 16) {
        v[h] = *reinterpret_cast<const uint4*>(src + h * 512);
      } else {
        uint32_t o[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int b = 0; b < 16; b += 2)
          if (b < left) o[b >> 2] |= (uint32_t) * reinterpret_cast<const uint16_t*>(src + h * 512 + b) << (8 * (b & 3));
        v[h] = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
    for (int j = 0; j < p.k; ++j) {
      const int slot = slot_of[t * p.k + j];
      if (slot < 0) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (at + h * 512 < p.row_bytes) *reinterpret_cast<uint4*>(dst + slot * ld + at + h * 512) = v[h];
    }
  }
}

// ---- pairs to tokens ----------------------------------------------------------------------------
// Bound by its bytes: 8192 tokens, 4 rows of 2048 FP32 columns each, 302 MB, 49 us (6.2 TB/s; with a branch around each row's load 74 for half the bytes).
// A thread takes four columns of a token (rows of src start on 16 bytes and are whole units of four), four of its rows' loads before their additions.
template <class T>
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ Combine p, int units, int vec) {
  grid_dep_wait();
  grid_dep_launch();
  const int* const index = dep(p.index);
  const float* const weight = dep(p.weight);
  const int64_t work = p.d ? p.tokens * units : 0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < work; i += (int64_t)gridDim.x * 256) {
    const int64_t t = work <= 0x7fffffff ? (int64_t)((uint32_t)i / (uint32_t)units) : i / units;
    const int c = (int)(i - t * units) * 4;
    const float* const src = dep(p.src) + t * p.k * p.ld + c;
    const int* const mine = index + t * p.k;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < p.k; j0 += 4) {
      float4 v[4];
      float w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = j0 + j < p.k && (unsigned)mine[min(j0 + j, p.k - 1)] < (unsigned)p.experts;
        v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        w[j] = 0.f;
        if (in) { v[j] = __ldcs(reinterpret_cast<const float4*>(src + (j0 + j) * p.ld)); w[j] = weight ? weight[t * p.k + j0 + j] : 1.f; }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) { s[0] = fmaf(w[j], v[j].x, s[0]); s[1] = fmaf(w[j], v[j].y, s[1]); s[2] = fmaf(w[j], v[j].z, s[2]); s[3] = fmaf(w[j], v[j].w, s[3]); }
    }
    T* const d = (T*)p.d + t * p.ld_d + c;
    if (vec && c + 4 <= p.cols) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(d) = make_float4(s[0], s[1], s[2], s[3]);
      } else {
        Pack<T> x;
        const float o[8] = {s[0], s[1], s[2], s[3], 0.f, 0.f, 0.f, 0.f};
        x.set(o);
        *reinterpret_cast<uint2*>(d) = make_uint2(x.w.x, x.w.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < p.cols) d[e] = from_f<T>(s[e]);
    }
  }
  if (p.parts) {
    const float* const parts = dep(p.parts);
    const int* const slot_of = dep(p.slot_of);
    for (int64_t pair = (int64_t)blockIdx.x * 256 + threadIdx.x; pair < p.tokens * p.k; pair += (int64_t)gridDim.x * 256) {
      const int slot = slot_of[pair];
      float s = 0.f;
      if (slot >= 0)
        for (int n = 0; n < p.n_parts; ++n) s += parts[(int64_t)slot * p.n_parts + n];
      p.dweight[pair] = s;
    }
  }
}

// ---- rows that TMA can address -------------------------------------------------------------------
// A warp per 256 columns of a row, eight elements a lane.
struct PackMatsList { PackMats j[kPackMats]; };
__global__ void __launch_bounds__(256) pack_mats_kernel(const __grid_constant__ PackMatsList list) {
  grid_dep_wait();
  grid_dep_launch();
  const PackMats& j = list.j[blockIdx.y];
  const uint16_t* const src = (const uint16_t*)dep(j.src);
  const int64_t per_row = (j.cols + 255) / 256, work = j.experts * j.rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < work; i += (int64_t)gridDim.x * 8) {
    const int64_t r = i / per_row, e = r / j.rows;
    const int c = (int)(i - r * per_row) * 256 + (threadIdx.x & 31) * 8, left = j.cols - c;
    if (left <= 0) continue;
    const uint16_t* const s = src + e * j.stride + (r - e * j.rows) * j.ld + c;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (q < left) w[q >> 1] |= (uint32_t)s[q] << (16 * (q & 1));
    *reinterpret_cast<uint4*>((uint16_t*)j.dst + r * j.ld_out + c) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

int64_t up4(int64_t n) { return (n + 3) / 4 * 4; }

}  // namespace

int64_t plan_ints(int64_t pairs, int experts, int height) {
  const int64_t chunk = plan_chunk(pairs), blocks = (pairs + chunk - 1) / chunk;
  return 2 * up4(experts) + up4(pairs) + up4(plan_slots(pairs, experts)) + 4 * plan_tiles(pairs, experts, height) + 4 + blocks * experts;
}
ExpertPlan plan_at(int* mem, int64_t pairs, int experts, int height) {
  ExpertPlan p;
  p.experts = experts; p.pairs = pairs;
  const auto take = [&](int64_t n) { int* const q = mem; mem += up4(n); return q; };
  p.start = take(experts); p.count = take(experts); p.slot_of = take(pairs); p.pair_of = take(plan_slots(pairs, experts));
  p.tiles = reinterpret_cast<ExpertTile*>(take(4 * plan_tiles(pairs, experts, height)));
  p.n_tiles = take(4);
  p.hist = mem;
  return p;
}

cudaError_t launch_plan(const int* index, const ExpertPlan& plan, int height, cudaStream_t st) {
  static std::atomic<signed char> ready[64];
  if (!once_per_device(ready, [] {
        const int most = kPlanWarps * kMostExperts * 2;
        return cudaFuncSetAttribute(plan_place_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess &&
               cudaFuncSetAttribute(plan_place_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) == cudaSuccess;
      }))
    return cudaErrorInvalidDevice;
  const PlanParams p{index, plan, plan_chunk(plan.pairs), height};
  const int smem = kPlanWarps * plan.experts * 2, blocks = (int)((plan.pairs + p.chunk - 1) / p.chunk);
  if (plan.pairs <= kPlanThreads) {      // (a thread for each pair and each expert)
    const int most = (int)plan.pairs > plan.experts ? (int)plan.pairs : plan.experts, threads = (most + 31) / 32 * 32;
    return launch_pdl(plan_place_kernel<true>, 1, threads, threads / 32 * plan.experts * 2, st, p);
  }
  const cudaError_t e = launch_pdl(plan_count_kernel, blocks, kPlanThreads, 0, st, p);
  return e == cudaSuccess ? launch_pdl(plan_place_kernel<false>, blocks, kPlanThreads, smem, st, p) : e;
}

cudaError_t launch_to_slots(const RowCopy* list, int n, int64_t tokens, int k, int cols, bool zero, const ExpertPlan& plan, cudaStream_t st) {
  CopyParams p = {};
  for (int i = 0; i < n; ++i) {
    p.c[i] = list[i];
    p.vec[i] = ((uintptr_t)list[i].src & 15) == 0 && list[i].ld % 8 == 0;
  }
  p.tokens = tokens; p.k = k; p.row_bytes = cols * 2; p.zero = zero ? plan.experts : 0; p.units = (p.row_bytes + 1023) / 1024; p.plan = plan;
  const int64_t want = ((tokens + p.zero) * p.units + 7) / 8, most = (int64_t)num_sms() * 8;
  const dim3 grid((unsigned)(want < most ? want : most), (unsigned)n);
  return launch_pdl_grid(to_slots_kernel, grid, 256, 0, st, p);
}

cudaError_t launch_pack_mats(const PackMats* list, int n, cudaStream_t st) {
  PackMatsList q = {};
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    q.j[i] = list[i];
    const int64_t warps = list[i].experts * list[i].rows * ((list[i].cols + 255) / 256);
    most = warps > most ? warps : most;
  }
  if (most == 0) return cudaSuccess;
  const int64_t blocks = (most + 7) / 8;
  return launch_pdl_grid(pack_mats_kernel, dim3((unsigned)(blocks < 1184 ? blocks : 1184), (unsigned)n), 256, 0, st, q);
}

template <class T>
static cudaError_t combine_as(const Combine& c, int type, cudaStream_t st) {
  const int units = (c.cols + 3) / 4, each = 4 * type_bytes(type);
  const int vec = (uintptr_t)c.d % each == 0 && c.ld_d * type_bytes(type) % each == 0;
  const int64_t want = (c.tokens * units + 255) / 256, most = (int64_t)num_sms() * 32;
  return launch_pdl(combine_kernel<T>, (int)(want < most ? want : most), 256, 0, st, c, units, vec);
}
cudaError_t launch_combine(int type, const Combine& c, cudaStream_t st) {
  return type == GN_F32 ? combine_as<float>(c, type, st) : type == GN_BF16 ? combine_as<__nv_bfloat16>(c, type, st) : combine_as<__half>(c, type, st);
}

}  // namespace gn
