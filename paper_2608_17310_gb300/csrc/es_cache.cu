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

// Norm, rotation and cache write in one pass: each vector is read once and written
// once. Bound by HBM on large calls and by the latency of one load - reduce - store
// chain on small ones, so every vector has its own lanes, and the loads of a vector
// and of its token's place do not wait for one another.
template <int D, bool kFp8>
__global__ void __launch_bounds__(kThreads)
append_kernel(const CacheView cache, const BatchView batch, const AppendArgs a) {
  wait_for_previous();
  constexpr int kLanes = D / 8;
  const int heads = a.q_heads + 2 * cache.kv_heads;
  const int64_t vectors = static_cast<int64_t>(batch.tokens) * heads;
  const int64_t id = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / kLanes;
  const int lane = threadIdx.x % kLanes;
  const bool here = id < vectors;
  // lanes without a vector follow vector 0 through the shuffles and write nothing
  const int t = here ? static_cast<int>(id / heads) : 0;
  const int h = here ? static_cast<int>(id - static_cast<int64_t>(t) * heads) : 0;
  const int e = lane * 8;
  const bool is_q = h < a.q_heads, is_v = h >= a.q_heads + cache.kv_heads;

  const uint4 raw = *reinterpret_cast<const uint4*>(a.qkv + t * a.qkv_stride +
                                                    static_cast<uint64_t>(h) * D + e);
  int seq = 0, pos = -1;
  const bool placed = locate(batch, t, seq, pos);
  float x[8];
  unpack8(raw, x);
  const uint16_t* weight = is_q ? a.q_weight : a.k_weight;
  if (is_v) weight = nullptr;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
  for (int m = kLanes / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, m);
  if (weight != nullptr) {
    float w[8];
    unpack8(*reinterpret_cast<const uint4*>(weight + e), w);
    const float r = rsqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
  }

  const int half = a.rotary_dim / 2;
  const int turn = a.positions != nullptr && a.rotary_dim > 0 ? a.positions[t] : pos;
  const bool known = turn >= 0 && static_cast<uint64_t>(turn) < a.rope_rows && (placed || a.positions != nullptr);
  const float nan = __int_as_float(0x7FC00000);
  if (half > 0 && a.interleaved) {
    if (!is_v && e < a.rotary_dim) {
      float cs[8];
      if (known) {
        const float4* row = reinterpret_cast<const float4*>(a.rope + static_cast<uint64_t>(turn) * a.rotary_dim + e);
        reinterpret_cast<float4*>(cs)[0] = row[0];
        reinterpret_cast<float4*>(cs)[1] = row[1];
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float c = known ? cs[i] : nan, s = known ? cs[i + 1] : nan;
        const float y = x[i] * c - x[i + 1] * s;
        x[i + 1] = x[i + 1] * c + x[i] * s;
        x[i] = y;
      }
    }
  } else if (half > 0) {
    // the partner of each element is in the lane half / 8 away
    const int away = half / 8;
    const bool turns = e < a.rotary_dim, low = e < half;
    const int self = threadIdx.x & 31;
    const int from = turns ? (low ? self + away : self - away) : self;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xFFFFFFFFu, x[i], from);
    if (!is_v && turns) {
      float cs[16];
      if (known) {
        const float4* row = reinterpret_cast<const float4*>(
            a.rope + static_cast<uint64_t>(turn) * a.rotary_dim + 2 * (low ? e : e - half));
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(cs)[i] = row[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = known ? cs[2 * i] : nan, s = known ? cs[2 * i + 1] : nan;
        x[i] = low ? x[i] * c - y[i] * s : x[i] * c + y[i] * s;
      }
    }
  }

  if (is_q) {
    if (here)
      *reinterpret_cast<uint4*>(a.q_out + t * a.q_out_stride + static_cast<uint64_t>(h) * D + e) = pack8(x);
  }
  float scale = 1.0f;
  if (kFp8) {
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
  if (is_q || !here || !placed) return;
  const int page = page_of(cache, batch, seq, pos);
  if (page < 0) return;
  const int kv = is_v ? h - a.q_heads - cache.kv_heads : h - a.q_heads;
  const uint64_t row = (static_cast<uint64_t>(kv) << cache.page_shift) + (pos & ((1 << cache.page_shift) - 1));
  const uint64_t at = page * cache.page_stride + row * D + e;
  if (kFp8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] / scale;
    uint8_t* to = static_cast<uint8_t*>(is_v ? cache.v : cache.k) + at;
    *reinterpret_cast<uint2*>(to) = make_uint2(pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7]));
    if (lane == 0) (is_v ? cache.v_scale : cache.k_scale)[page * cache.scale_stride + row] = scale;
  } else {
    uint16_t* to = static_cast<uint16_t*>(is_v ? cache.v : cache.k) + at;
    *reinterpret_cast<uint4*>(to) = pack8(x);
  }
}

// Vectors [token][key or value][head]; outputs are contiguous rows.
template <int D, bool kFp8>
__global__ void __launch_bounds__(kThreads)
read_kernel(const CacheView cache, const BatchView batch, uint16_t* __restrict__ k_out,
            uint16_t* __restrict__ v_out) {
  wait_for_previous();
  constexpr int kLanes = D / 8;
  const int heads = 2 * cache.kv_heads;
  const int64_t id = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / kLanes;
  if (id >= static_cast<int64_t>(batch.tokens) * heads) return;
  const int e = (threadIdx.x % kLanes) * 8;
  const int t = static_cast<int>(id / heads);
  int h = static_cast<int>(id - static_cast<int64_t>(t) * heads);
  const bool is_v = h >= cache.kv_heads;
  if (is_v) h -= cache.kv_heads;
  uint16_t* out = is_v ? v_out : k_out;
  if (out == nullptr) return;
  int seq, pos, page = -1;
  if (locate(batch, t, seq, pos)) page = page_of(cache, batch, seq, pos);
  uint4 w = make_uint4(0, 0, 0, 0);
  if (page >= 0) {
    const uint64_t row = (static_cast<uint64_t>(h) << cache.page_shift) + (pos & ((1 << cache.page_shift) - 1));
    const uint64_t at = page * cache.page_stride + row * D + e;
    if (kFp8) {
      const float scale = (is_v ? cache.v_scale : cache.k_scale)[page * cache.scale_stride + row];
      const uint2 codes = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(is_v ? cache.v : cache.k) + at);
      float a[4], b[4];
      unpack_e4m3(codes.x, a);
      unpack_e4m3(codes.y, b);
      w = make_uint4(pack_bf16(a[0] * scale, a[1] * scale), pack_bf16(a[2] * scale, a[3] * scale),
                     pack_bf16(b[0] * scale, b[1] * scale), pack_bf16(b[2] * scale, b[3] * scale));
    } else {
      w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(is_v ? cache.v : cache.k) + at);
    }
  }
  *reinterpret_cast<uint4*>(out + (static_cast<uint64_t>(t) * cache.kv_heads + h) * D + e) = w;
}

template <class K, class... A>
cudaError_t launch_vectors(K kernel, int64_t vectors, int head_dim, cudaStream_t stream, const A&... args) {
  const int64_t per_block = kThreads / (head_dim / 8);
  const int64_t blocks = (vectors + per_block - 1) / per_block;
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_early(kernel, static_cast<int>(blocks), kThreads, 0, stream, args...);
}

}  // namespace

cudaError_t launch_append(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                          const AppendArgs& args, cudaStream_t stream) {
  const int64_t n = static_cast<int64_t>(batch.tokens) * (args.q_heads + 2 * cache.kv_heads);
  auto kernel = head_dim == 128 ? (fp8 ? append_kernel<128, true> : append_kernel<128, false>)
                                : (fp8 ? append_kernel<64, true> : append_kernel<64, false>);
  return launch_vectors(kernel, n, head_dim, stream, cache, batch, args);
}

cudaError_t launch_read(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                        uint16_t* k_out, uint16_t* v_out, cudaStream_t stream) {
  const int64_t n = static_cast<int64_t>(batch.tokens) * 2 * cache.kv_heads;
  auto kernel = head_dim == 128 ? (fp8 ? read_kernel<128, true> : read_kernel<128, false>)
                                : (fp8 ? read_kernel<64, true> : read_kernel<64, false>);
  return launch_vectors(kernel, n, head_dim, stream, cache, batch, k_out, v_out);
}

}  // namespace esopt
