// es_route and es_combine: tokens to experts and back.
#include <cfloat>

#include "es_attention.cuh"
#include "es_project_internal.h"

namespace esopt {
namespace {

constexpr int kRouteWarps = 16, kAloneWarps = 32;  // of a block among others, and of one alone
constexpr int kRouteGrid = 304;  // two blocks an SM

struct RouteArgs {
  const void* scores;
  int32_t* chosen;
  float* weights;
  int32_t* start;
  int32_t* rows;
  int32_t* places;
  uint64_t stride;
  int tokens, experts, top, normalise;
  int share;  // tokens of a warp
};

// Order-preserving code of a score; 0 for one that is never chosen. Zeros of both signs are equal scores: 0 added to
// the negative one makes it the other.
__device__ __forceinline__ uint32_t code_of(float x) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t w = __float_as_uint(fminf(x, FLT_MAX) + 0.0f);
  return w & 0x80000000u ? ~w : w | 0x80000000u;
}
__device__ __forceinline__ float score_of_code(uint32_t c) {
  return __uint_as_float(c & 0x80000000u ? c & 0x7FFFFFFFu : ~c);
}

// kTokens tokens by one warp, together so that their chains of reductions run beside one another: lane j
// gets the j-th choice of each (its expert or -1, its weight).
template <int kPerLane, bool kBf16, int kTokens>
__device__ __forceinline__ void choose(const RouteArgs& a, const int64_t (&token)[kTokens], int lane, int (&expert)[kTokens],
                                       float (&weight)[kTokens]) {
  uint32_t code[kTokens][kPerLane];
#pragma unroll
  for (int n = 0; n < kTokens; ++n)
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      const int e = i * 32 + lane;
      code[n][i] = 0;
      if (e < a.experts) {
        const uint64_t at = token[n] * a.stride + e;
        code[n][i] = code_of(kBf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.scores)[at]) << 16)
                                   : static_cast<const float*>(a.scores)[at]);
      }
    }
  uint32_t best[kTokens], mine[kTokens];
  float top[kTokens], all[kTokens];
#pragma unroll
  for (int n = 0; n < kTokens; ++n) {
    best[n] = mine[n] = 0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) best[n] = max(best[n], code[n][i]);
    const uint32_t first = __reduce_max_sync(0xFFFFFFFFu, best[n]);
    top[n] = first != 0 ? score_of_code(first) : 0.0f;
    all[n] = 0.0f;
    expert[n] = -1;
    if (!a.normalise) {
#pragma unroll
      for (int i = 0; i < kPerLane; ++i)
        if (code[n][i] != 0) all[n] += expf(score_of_code(code[n][i]) - top[n]);
    }
  }
  if constexpr (kPerLane <= 4) {
    // A lane keeps its scores in order (equal ones by the lower expert), so only their first takes part, and the
    // reduction for the lowest expert is left for scores that several lanes have.
    int of[kTokens][kPerLane];
#pragma unroll
    for (int n = 0; n < kTokens; ++n) {
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) of[n][i] = i * 32 + lane;
#pragma unroll
      for (int end = kPerLane - 1; end > 0; --end)
#pragma unroll
        for (int i = 0; i < end; ++i)
          if (code[n][i + 1] > code[n][i]) {
            const uint32_t c = code[n][i];
            code[n][i] = code[n][i + 1];
            code[n][i + 1] = c;
            const int o = of[n][i];
            of[n][i] = of[n][i + 1];
            of[n][i + 1] = o;
          }
    }
    for (int j = 0; j < a.top; ++j) {
#pragma unroll
      for (int n = 0; n < kTokens; ++n) {
        const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, code[n][0]);
        const bool has = code[n][0] == most;
        const uint32_t those = __ballot_sync(0xFFFFFFFFu, has);
        int at = __shfl_sync(0xFFFFFFFFu, of[n][0], __ffs(those) - 1);
        if (those & (those - 1)) at = static_cast<int>(__reduce_min_sync(0xFFFFFFFFu, has ? static_cast<uint32_t>(of[n][0]) : 0xFFFFFFFFu));
        if (lane == j && most != 0) {
          expert[n] = at;
          mine[n] = most;
        }
        if (has && of[n][0] == at) {
#pragma unroll
          for (int i = 0; i + 1 < kPerLane; ++i) {
            code[n][i] = code[n][i + 1];
            of[n][i] = of[n][i + 1];
          }
          code[n][kPerLane - 1] = 0;
        }
      }
    }
  } else {
    for (int j = 0; j < a.top; ++j) {
      uint32_t most[kTokens], at[kTokens];
#pragma unroll
      for (int n = 0; n < kTokens; ++n) most[n] = __reduce_max_sync(0xFFFFFFFFu, best[n]);
#pragma unroll
      for (int n = 0; n < kTokens; ++n) {
        at[n] = 0xFFFFFFFFu;
#pragma unroll
        for (int i = kPerLane - 1; i >= 0; --i)
          if (code[n][i] == most[n]) at[n] = i * 32 + lane;
        at[n] = __reduce_min_sync(0xFFFFFFFFu, at[n]);
      }
#pragma unroll
      for (int n = 0; n < kTokens; ++n) {
        best[n] = 0;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
          if (static_cast<uint32_t>(i * 32 + lane) == at[n]) code[n][i] = 0;
          best[n] = max(best[n], code[n][i]);
        }
        if (lane == j && most[n] != 0) {
          expert[n] = static_cast<int>(at[n]);
          mine[n] = most[n];
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < kTokens; ++n) {
    weight[n] = expert[n] >= 0 ? expf(score_of_code(mine[n]) - top[n]) : 0.0f;
    if (a.normalise) all[n] = weight[n];
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) all[n] += __shfl_xor_sync(0xFFFFFFFFu, all[n], m);
    if (expert[n] >= 0) weight[n] = weight[n] / all[n];
  }
}

// Walks the pairs [begin, end) of one warp in order: next[e] is the place of the next pair of
// expert e. kPlace: writes places and rows; else it only counts.
template <bool kPlace>
__device__ __forceinline__ void walk(const RouteArgs& a, int begin, int end, int32_t* next, int lane) {
  for (int p0 = begin; p0 < end; p0 += 32) {
    const int p = p0 + lane;
    const int e = p < end ? a.chosen[p] : -1;
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, e);
    const int before = __popc(same & ((1u << lane) - 1));
    const int base = e >= 0 ? next[e] : 0;
    __syncwarp();
    if (e >= 0 && before == 0) next[e] = base + __popc(same);
    __syncwarp();
    if (kPlace && p < end) {
      a.places[p] = e >= 0 ? base + before : -1;
      if (e >= 0) a.rows[base + before] = p / a.top;
    }
  }
}

// Sum over the block's threads before this one; total: over all.
template <int kWarps>
__device__ __forceinline__ int scan_before(int x, int* shared, int& total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int sum = x;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, sum, m);
    if (lane >= m) sum += y;
  }
  if (lane == 31) shared[warp] = sum;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += shared[w];
    total += shared[w];
  }
  __syncthreads();
  return before + sum - x;
}

// Chooses the experts of the block's tokens and counts them: counts[expert][block]. With one
// block (kAll) it goes on to the places itself.
//
// A warp has a token's scores in registers, as order-preserving codes, and takes the largest
// `top` times (one reduction for the value, one for the lowest index). Pairs are then placed
// by a counting sort: a warp's pairs are a range of their own, so a pair's place is its
// expert's start, the pairs of earlier blocks and warps, and those before it in the warp
// (__match_any_sync), whatever the timing.
template <int kPerLane, bool kBf16, bool kAll>
__global__ void __launch_bounds__((kAll ? kAloneWarps : kRouteWarps) * 32)
choose_kernel(const RouteArgs a, int32_t* counts) {
  constexpr int kWarps = kAll ? kAloneWarps : kRouteWarps;
  extern __shared__ int32_t next[];  // [warp][expert]
  __shared__ int sums[kWarps];
  wait_for_previous();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t t0 = min((static_cast<int64_t>(blockIdx.x) * kWarps + warp) * a.share, static_cast<int64_t>(a.tokens));
  const int64_t t1 = min(t0 + a.share, static_cast<int64_t>(a.tokens));
  int32_t* mine = next + warp * a.experts;
  for (int e = lane; e < a.experts; e += 32) mine[e] = 0;
  __syncwarp();
  constexpr int kTokens = kPerLane <= 4 ? 2 : 1;
  for (int64_t t = t0; t < t1; t += kTokens) {
    int64_t token[kTokens];
    int expert[kTokens];
    float weight[kTokens];
#pragma unroll
    for (int n = 0; n < kTokens; ++n) token[n] = min(t + n, t1 - 1);
    choose<kPerLane, kBf16, kTokens>(a, token, lane, expert, weight);
#pragma unroll
    for (int n = 0; n < kTokens; ++n) {
      if (lane < a.top && t + n < t1) {
        a.chosen[(t + n) * a.top + lane] = expert[n];
        a.weights[(t + n) * a.top + lane] = weight[n];
        if (expert[n] >= 0) ++mine[expert[n]];  // a token's experts differ
      }
      __syncwarp();
    }
  }
  __syncthreads();
  if (!kAll) {
    for (int e = threadIdx.x; e < a.experts; e += kWarps * 32) {
      int sum = 0;
      for (int w = 0; w < kWarps; ++w) sum += next[w * a.experts + e];
      counts[e * kRouteGrid + blockIdx.x] = sum;
    }
    return;
  }
  int base = 0;
  for (int e0 = 0; e0 < a.experts; e0 += kWarps * 32) {
    const int e = e0 + threadIdx.x;
    int sum = 0;
    if (e < a.experts)
      for (int w = 0; w < kWarps; ++w) sum += next[w * a.experts + e];
    int total;
    int at = base + scan_before<kWarps>(sum, sums, total);
    if (e < a.experts) {
      a.start[e] = at;
      for (int w = 0; w < kWarps; ++w) {
        const int n = next[w * a.experts + e];
        next[w * a.experts + e] = at;
        at += n;
      }
    }
    base += total;
  }
  if (threadIdx.x == 0) a.start[a.experts] = base;
  __syncthreads();
  walk<true>(a, static_cast<int>(t0) * a.top, static_cast<int>(t1) * a.top, mine, lane);
}

// Places the pairs of the block's tokens, with the counts of all blocks.
__global__ void __launch_bounds__(kRouteWarps * 32)
place_kernel(const RouteArgs a, const int32_t* counts) {
  extern __shared__ int32_t next[];
  __shared__ int sums[kRouteWarps], whole[ES_MAX_EXPERTS], earlier[ES_MAX_EXPERTS];
  wait_for_previous();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t t0 = min((static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp) * a.share, static_cast<int64_t>(a.tokens));
  const int64_t t1 = min(t0 + a.share, static_cast<int64_t>(a.tokens));
  int32_t* mine = next + warp * a.experts;
  for (int e = lane; e < a.experts; e += 32) mine[e] = 0;
  __syncwarp();
  walk<false>(a, static_cast<int>(t0) * a.top, static_cast<int>(t1) * a.top, mine, lane);
  // each expert's pairs, in all blocks and in those before this one
#pragma unroll 4
  for (int e = warp; e < a.experts; e += kRouteWarps) {
    int sum = 0, before = 0;
#pragma unroll
    for (int i = 0; i < (kRouteGrid + 31) / 32; ++i) {
      const int b = i * 32 + lane;
      const int n = b < static_cast<int>(gridDim.x) ? counts[e * kRouteGrid + b] : 0;
      sum += n;
      before += b < static_cast<int>(blockIdx.x) ? n : 0;
    }
    sum = __reduce_add_sync(0xFFFFFFFFu, sum);
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    if (lane == 0) {
      whole[e] = sum;
      earlier[e] = before;
    }
  }
  __syncthreads();
  int base = 0;
  for (int e0 = 0; e0 < a.experts; e0 += kRouteWarps * 32) {
    const int e = e0 + threadIdx.x;
    int total;
    int at = base + scan_before<kRouteWarps>(e < a.experts ? whole[e] : 0, sums, total);
    if (e < a.experts) {
      if (blockIdx.x == 0) a.start[e] = at;
      at += earlier[e];
      for (int w = 0; w < kRouteWarps; ++w) {
        const int n = next[w * a.experts + e];
        next[w * a.experts + e] = at;
        at += n;
      }
    }
    base += total;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.start[a.experts] = base;
  __syncthreads();
  walk<true>(a, static_cast<int>(t0) * a.top, static_cast<int>(t1) * a.top, mine, lane);
}

template <int kPerLane, bool kBf16>
cudaError_t route(RouteArgs a, int32_t* counts, cudaStream_t stream) {
  const size_t alone = sizeof(int32_t) * kAloneWarps * a.experts, shared = sizeof(int32_t) * kRouteWarps * a.experts;
  auto one = choose_kernel<kPerLane, kBf16, true>;
  auto many = choose_kernel<kPerLane, kBf16, false>;
  if (alone + sizeof(int) * kAloneWarps > 48 * 1024) {  // with what the kernel declares itself
    // The limit is the kernel's, in all threads: each call sets the same one, that of the most experts.
    constexpr int kMostAlone = sizeof(int32_t) * kAloneWarps * ES_MAX_EXPERTS, kMost = sizeof(int32_t) * kRouteWarps * ES_MAX_EXPERTS;
    cudaError_t err = cudaFuncSetAttribute(one, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostAlone);
    if (err == cudaSuccess) err = cudaFuncSetAttribute(many, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (err == cudaSuccess) err = cudaFuncSetAttribute(place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (err != cudaSuccess) {
      cudaGetLastError();
      return err;
    }
  }
  if (a.tokens <= 8 * kAloneWarps) {
    a.share = (a.tokens + kAloneWarps - 1) / kAloneWarps;
    return launch_early(one, 1, kAloneWarps * 32, alone, stream, a, counts);
  }
  a.share = (a.tokens + kRouteWarps * kRouteGrid - 1) / (kRouteWarps * kRouteGrid);
  const int grid = (a.tokens + kRouteWarps * a.share - 1) / (kRouteWarps * a.share);
  const cudaError_t err = launch_early(many, grid, kRouteWarps * 32, shared, stream, a, counts);
  if (err != cudaSuccess) return err;
  return launch_early(place_kernel, grid, kRouteWarps * 32, shared, stream, a, static_cast<const int32_t*>(counts));
}

struct CombineArgs {
  const uint16_t* y;
  const int32_t* places;
  const float* weights;
  const uint16_t* add;
  uint16_t* out;
  uint64_t y_stride, add_stride, out_stride;
  int slots, tokens, top, features;
};

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// A thread has eight features of a token. Bound by memory.
__global__ void __launch_bounds__(256)
combine_kernel(const CombineArgs a) {
  wait_for_previous();
  const int width = a.features / 8;
  const int64_t all = static_cast<int64_t>(a.tokens) * width;
  for (int64_t n = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; n < all;
       n += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t t = n / width;
    const int f = static_cast<int>(n - t * width) * 8;
    float sum[8] = {};
#pragma unroll 4
    for (int j = 0; j < a.top; ++j) {
      const int place = a.places[t * a.top + j];
      if (static_cast<unsigned>(place) >= static_cast<unsigned>(a.slots)) continue;
      const float w = a.weights[t * a.top + j];
      const uint4 v = *reinterpret_cast<const uint4*>(a.y + place * a.y_stride + f);
      const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[2 * i] = fmaf(w, bf16_low(word[i]), sum[2 * i]);
        sum[2 * i + 1] = fmaf(w, bf16_high(word[i]), sum[2 * i + 1]);
      }
    }
    if (a.add != nullptr) {
      const uint4 v = *reinterpret_cast<const uint4*>(a.add + t * a.add_stride + f);
      const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[2 * i] += bf16_low(word[i]);
        sum[2 * i + 1] += bf16_high(word[i]);
      }
    }
    *reinterpret_cast<uint4*>(a.out + t * a.out_stride + f) =
        make_uint4(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]), pack_bf16(sum[4], sum[5]), pack_bf16(sum[6], sum[7]));
  }
}

}  // namespace

uint64_t route_workspace_bytes(int, int experts, int) { return sizeof(int32_t) * kRouteGrid * experts; }

cudaError_t launch_route(const es_route_t& r, void* workspace, cudaStream_t stream) {
  const RouteArgs a{r.scores, r.chosen, r.weights, r.start, r.rows, r.places, r.scores_stride,
                    r.tokens, r.experts, r.top, r.normalise, 0};
  int32_t* counts = static_cast<int32_t*>(workspace);
  const bool b = r.dtype == ES_BF16;
  const int n = (r.experts + 31) / 32;
  if (n <= 1) return b ? route<1, true>(a, counts, stream) : route<1, false>(a, counts, stream);
  if (n <= 2) return b ? route<2, true>(a, counts, stream) : route<2, false>(a, counts, stream);
  if (n <= 4) return b ? route<4, true>(a, counts, stream) : route<4, false>(a, counts, stream);
  if (n <= 8) return b ? route<8, true>(a, counts, stream) : route<8, false>(a, counts, stream);
  return b ? route<32, true>(a, counts, stream) : route<32, false>(a, counts, stream);
}

cudaError_t launch_combine(const es_combine_t& c, cudaStream_t stream) {
  const CombineArgs a{static_cast<const uint16_t*>(c.y), c.places, c.weights, static_cast<const uint16_t*>(c.add),
                      static_cast<uint16_t*>(c.out), c.y_stride, c.add_stride, c.out_stride, c.slots, c.tokens, c.top, c.features};
  const int64_t blocks = (static_cast<int64_t>(c.tokens) * (c.features / 8) + 255) / 256;
  return launch_early(combine_kernel, static_cast<int>(blocks < 152 * 64 ? blocks : 152 * 64), 256, 0, stream, a);
}

}  // namespace esopt
