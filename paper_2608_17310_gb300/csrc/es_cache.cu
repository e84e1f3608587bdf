// es_cache_append and es_cache_read: whole head vectors, 8 elements (16 bytes of bf16)
// per lane, a vector in the 8 or 16 lanes of one warp that its head_dim takes.
#include <cuda_runtime.h>

#include <cfloat>

#include "es_rollout_internal.h"

namespace esopt {
namespace {

constexpr int kThreads = 256;
constexpr float kE4m3Max = 448.0f;

__device__ __forceinline__ float2 unpack_bf16(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack_bf16(u[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                    pack_bf16(x[6], x[7]));
}

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return static_cast<uint32_t>(lo) | static_cast<uint32_t>(hi) << 16;
}

// Four E4M3 codes as floats; every code is an f16 number.
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(w >> (16 * i))));
    asm("{\n .reg .f16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}"
        : "=f"(x[2 * i]), "=f"(x[2 * i + 1])
        : "r"(h));
  }
}

// The sequence whose rows hold token t, and the token's position; false where it has
// none (a row past the last sequence, or more new tokens than the sequence has).
__device__ __forceinline__ bool locate(const BatchView& b, int t, int& seq, int& pos) {
  seq = t;
  if (b.start != nullptr) {
    int lo = 0, hi = b.sequences - 1;  // the last sequence whose start is at most t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (b.start[mid] <= t) lo = mid; else hi = mid - 1;
    }
    seq = lo;
  }
  int begin, count, base;
  new_tokens(b, seq, begin, count, base);
  if (t < begin || t >= begin + count) return false;
  pos = base + (t - begin);
  return pos >= 0;
}

// Where a token's keys and values go or come from.
struct Place {
  int pos;   // in the sequence, -1 where it has none
  int page;  // -1 where there is none
  int slot;
};

__device__ __forceinline__ Place place_of(const CacheView& cache, const BatchView& batch, int t) {
  Place p{-1, -1, 0};
  int seq, pos;
  if (t < batch.tokens && locate(batch, t, seq, pos)) {
    p.pos = pos;
    p.page = page_of(cache, batch, seq, pos);
    p.slot = pos & ((1 << cache.page_shift) - 1);
  }
  return p;
}

// A block takes kTokens tokens. Their places are found once; then each group of lanes takes
// whole vectors, kBatch of them with all loads in flight. Neighbouring groups take the same
// head of neighbouring tokens, whose vectors lie side by side in the page.
//
// Bound by HBM on large calls and by the latency of one chain of loads on small ones.
// Measured (GB300): append of 16,383 tokens of 40 + 2 x 8 heads of 128, bf16, 85 us, 5.6 TB/s,
// 84 % of the copy rate (a vector to each group, its place and its row of the rope table
// found each time: 170 us; a token's row once: 140; the next batch's loads ahead: 86), at 67 %
// of the issue slots; of 16,333 ragged tokens into FP8 81 us, 4.6 TB/s, at 71 % of them;
// read of 213,000 FP8 tokens of 8 heads 208 us, 6.4 TB/s, 96 %. Batches of 4 take 14 %
// longer, 16 tokens a block 10 %, 4 tokens 5 %.
constexpr int kBatch = 2;

template <int D, bool kFp8, int kTokens>
__global__ void __launch_bounds__(kThreads)
append_kernel(const CacheView cache, const BatchView batch, const AppendArgs a) {
  constexpr int kLanes = D / 8, kGroups = kThreads / kLanes;
  __shared__ Place places[kTokens];
  __shared__ int turns[kTokens];  // row of the rope table, -1 where it has none
  wait_for_previous();
  const int t0 = blockIdx.x * kTokens;
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, e = lane * 8;
  const int heads = a.q_heads + 2 * cache.kv_heads, vectors = kTokens * heads;
  // A group stays with one token, its heads kGroups / kTokens apart.
  static_assert(kGroups % kTokens == 0, "a group's vectors are of one token");
  const int own = group % kTokens, t = t0 + own;
  auto load = [&](uint4 (&to)[kBatch], int v0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int v = v0 + b * kGroups + group;
      to[b] = make_uint4(0, 0, 0, 0);
      if (v < vectors && t < batch.tokens)
        to[b] = *reinterpret_cast<const uint4*>(a.qkv + t * a.qkv_stride + static_cast<uint64_t>(v / kTokens) * D + e);
    }
  };
  uint4 next[kBatch];
  load(next, 0);
  if (threadIdx.x < kTokens) {
    const int t = t0 + threadIdx.x;
    const Place p = place_of(cache, batch, t);
    int turn = p.pos;
    if (a.positions != nullptr && t < batch.tokens) turn = a.positions[t];
    places[threadIdx.x] = p;
    turns[threadIdx.x] = turn >= 0 && static_cast<uint64_t>(turn) < a.rope_rows ? turn : -1;
  }
  const int half = a.rotary_dim / 2;
  const float nan = __int_as_float(0x7FC00000);
  uint4 weight[2] = {};  // of queries and keys, this lane's elements
  if (a.q_weight != nullptr) weight[0] = *reinterpret_cast<const uint4*>(a.q_weight + e);
  if (a.k_weight != nullptr) weight[1] = *reinterpret_cast<const uint4*>(a.k_weight + e);
  __syncthreads();

  // This token's (cos, sin) of the lane's elements: of 8 pairs, or of 4 where pairs are neighbours.
  const bool turning = e < a.rotary_dim, low = e < half;
  const int turn = turns[own];
  const Place p = places[own];
  float4 cs[4] = {make_float4(nan, nan, nan, nan), make_float4(nan, nan, nan, nan), make_float4(nan, nan, nan, nan),
                  make_float4(nan, nan, nan, nan)};
  if (turning && turn >= 0) {
    const int first = a.interleaved ? e : 2 * (low ? e : e - half);
    const float4* row = reinterpret_cast<const float4*>(a.rope + static_cast<uint64_t>(turn) * a.rotary_dim + first);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < 2 || !a.interleaved) cs[i] = row[i];
  }
  for (int v0 = 0; v0 < vectors; v0 += kGroups * kBatch) {  // the same for all lanes: they shuffle
    uint4 raw[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) raw[b] = next[b];
    if (v0 + kGroups * kBatch < vectors) load(next, v0 + kGroups * kBatch);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (v0 + b * kGroups >= vectors) break;
      const int v = v0 + b * kGroups + group, h = v / kTokens;
      const bool here = v < vectors && t < batch.tokens;
      const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + cache.kv_heads;
      float x[8];
      unpack8(raw[b], x);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
      for (int m = kLanes / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, m);
      if (!is_v && (is_q ? a.q_weight : a.k_weight) != nullptr) {
        float w[8];
        unpack8(is_q ? weight[0] : weight[1], w);
        const float r = rsqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
      }

      if (half > 0 && a.interleaved) {
        if (!is_v && turning) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float c = i % 2 == 0 ? cs[i / 2].x : cs[i / 2].z, n = i % 2 == 0 ? cs[i / 2].y : cs[i / 2].w;
            const float y = x[2 * i] * c - x[2 * i + 1] * n;
            x[2 * i + 1] = x[2 * i + 1] * c + x[2 * i] * n;
            x[2 * i] = y;
          }
        }
      } else if (half > 0) {
        // the partner of each element is in the lane half / 8 away
        const int self = threadIdx.x & 31, from = turning ? (low ? self + half / 8 : self - half / 8) : self;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xFFFFFFFFu, x[i], from);
        if (!is_v && turning) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[2 * i] = low ? x[2 * i] * cs[i].x - y[2 * i] * cs[i].y : x[2 * i] * cs[i].x + y[2 * i] * cs[i].y;
            x[2 * i + 1] = low ? x[2 * i + 1] * cs[i].z - y[2 * i + 1] * cs[i].w : x[2 * i + 1] * cs[i].z + y[2 * i + 1] * cs[i].w;
          }
        }
      }

      float scale = 1.0f;
      if (kFp8 && __any_sync(0xFFFFFFFFu, !is_q)) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float m = fabsf(x[i]);
          top = m <= FLT_MAX ? fmaxf(top, m) : top;
        }
#pragma unroll
        for (int m = kLanes / 2; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
        scale = fmaxf(top / kE4m3Max, FLT_MIN);
      }
      if (!here) continue;
      if (is_q) {
        *reinterpret_cast<uint4*>(a.q_out + t * a.q_out_stride + static_cast<uint64_t>(h) * D + e) = pack8(x);
        continue;
      }
      if (p.page < 0) continue;
      const int kv = is_v ? h - a.q_heads - cache.kv_heads : h - a.q_heads;
      const uint64_t row = (static_cast<uint64_t>(kv) << cache.page_shift) + p.slot;
      const uint64_t at = p.page * cache.page_stride + row * D + e;
      if (kFp8) {
        // by the reciprocal: a code on the border of two can fall to either side, as with any
        // fp32 rounding of x / scale, for an eighth of the time of eight divisions
        const float inv = 1.0f / scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inv;
        uint8_t* to = static_cast<uint8_t*>(is_v ? cache.v : cache.k) + at;
        *reinterpret_cast<uint2*>(to) = make_uint2(pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7]));
        if (lane == 0) (is_v ? cache.v_scale : cache.k_scale)[p.page * cache.scale_stride + row] = scale;
      } else {
        uint16_t* to = static_cast<uint16_t*>(is_v ? cache.v : cache.k) + at;
        *reinterpret_cast<uint4*>(to) = pack8(x);
      }
    }
  }
}

// Keys' heads, then values', of a block's tokens; outputs are contiguous rows. A lane takes 16
// bytes of a vector: 8 elements, or 16 codes.
template <int D, bool kFp8, int kTokens>
__global__ void __launch_bounds__(kThreads)
read_kernel(const CacheView cache, const BatchView batch, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out) {
  constexpr int kEach = kFp8 ? 16 : 8, kLanes = D / kEach, kGroups = kThreads / kLanes;
  __shared__ Place places[kTokens];
  wait_for_previous();
  const int t0 = blockIdx.x * kTokens;
  if (threadIdx.x < kTokens) places[threadIdx.x] = place_of(cache, batch, t0 + threadIdx.x);
  const int group = threadIdx.x / kLanes, e = threadIdx.x % kLanes * kEach;
  const int vectors = kTokens * 2 * cache.kv_heads;
  __syncthreads();
  for (int v0 = group; v0 < vectors; v0 += kGroups * kBatch) {
    uint4 raw[kBatch];
    float scale[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int v = v0 + b * kGroups, h2 = v / kTokens;
      raw[b] = make_uint4(0, 0, 0, 0);
      scale[b] = 0.0f;
      if (v >= vectors) continue;
      const bool is_v = h2 >= cache.kv_heads;
      const Place p = places[v % kTokens];
      if (p.page < 0 || (is_v ? v_out : k_out) == nullptr) continue;
      const uint64_t row = (static_cast<uint64_t>(is_v ? h2 - cache.kv_heads : h2) << cache.page_shift) + p.slot;
      const char* from = static_cast<const char*>(is_v ? cache.v : cache.k) + (p.page * cache.page_stride + row * D + e) * (kFp8 ? 1 : 2);
      raw[b] = __ldg(reinterpret_cast<const uint4*>(from));
      if (kFp8) scale[b] = __ldg((is_v ? cache.v_scale : cache.k_scale) + p.page * cache.scale_stride + row);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int v = v0 + b * kGroups, t = t0 + v % kTokens, h2 = v / kTokens;
      const bool is_v = h2 >= cache.kv_heads;
      uint16_t* out = is_v ? v_out : k_out;
      if (v >= vectors || t >= batch.tokens || out == nullptr) continue;
      uint4* to = reinterpret_cast<uint4*>(out + (static_cast<uint64_t>(t) * cache.kv_heads + (is_v ? h2 - cache.kv_heads : h2)) * D + e);
      if (kFp8) {
        const uint32_t u[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[4];
          unpack_e4m3(u[i], f);
          w[2 * i] = pack_bf16(f[0] * scale[b], f[1] * scale[b]);
          w[2 * i + 1] = pack_bf16(f[2] * scale[b], f[3] * scale[b]);
        }
        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
      } else {
        to[0] = raw[b];
      }
    }
  }
}

// Blocks of 8 tokens where there are enough of them to fill the card, of one token else.
constexpr int kManyTokens = 2048;

template <class K, class... A>
cudaError_t launch_tokens(K kernel, int tokens, int per_block, cudaStream_t stream, const A&... args) {
  return launch_early(kernel, (tokens + per_block - 1) / per_block, kThreads, 0, stream, args...);
}

template <int D, bool kFp8>
cudaError_t append(const CacheView& cache, const BatchView& batch, const AppendArgs& args, cudaStream_t stream) {
  if (batch.tokens >= kManyTokens) return launch_tokens(append_kernel<D, kFp8, 8>, batch.tokens, 8, stream, cache, batch, args);
  return launch_tokens(append_kernel<D, kFp8, 1>, batch.tokens, 1, stream, cache, batch, args);
}

template <int D, bool kFp8>
cudaError_t read(const CacheView& cache, const BatchView& batch, uint16_t* k_out, uint16_t* v_out, cudaStream_t stream) {
  if (batch.tokens >= kManyTokens) return launch_tokens(read_kernel<D, kFp8, 8>, batch.tokens, 8, stream, cache, batch, k_out, v_out);
  return launch_tokens(read_kernel<D, kFp8, 1>, batch.tokens, 1, stream, cache, batch, k_out, v_out);
}

}  // namespace

cudaError_t launch_append(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                          const AppendArgs& args, cudaStream_t stream) {
  auto f = head_dim == 128 ? (fp8 ? append<128, true> : append<128, false>) : (fp8 ? append<64, true> : append<64, false>);
  return f(cache, batch, args, stream);
}

cudaError_t launch_read(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                        uint16_t* k_out, uint16_t* v_out, cudaStream_t stream) {
  auto f = head_dim == 128 ? (fp8 ? read<128, true> : read<128, false>) : (fp8 ? read<64, true> : read<64, false>);
  return f(cache, batch, k_out, v_out, stream);
}

}  // namespace esopt
