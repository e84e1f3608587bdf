// es_attention: attention of the new tokens over a paged cache.
//
// The rows of a (sequence, key head) are its new tokens times the query heads that share
// the key head, token by token, so a tile of rows reads its keys once for the whole group
// and spans few positions. With m the running maximum of a row's scores (in units of
// log 2) and l the running sum, a tile of keys does
//   m' = max(m, max x),  o = o 2^(m - m') + sum 2^(x - m') v,  l = l 2^(m - m') + sum 2^(x - m').
#include <cuda_runtime.h>

#include <cfloat>

#include "es_attention.cuh"
#include "es_rollout_internal.h"

namespace esopt {
namespace {

constexpr int kTile = 64;  // keys per tile
constexpr int kRows = 64;  // rows per block, 16 per warp

// One block for 64 rows of a (sequence, key head), one warp for 16 of them, keys in tiles
// of 64 through shared memory.
template <int D, bool kFp8>
__global__ void __launch_bounds__(128)
attention_kernel(const CacheView cache, const BatchView batch, const AttentionArgs a) {
  __shared__ __align__(16) uint16_t ks[kTile * D];
  __shared__ __align__(16) uint16_t vs[kTile * D];
  __shared__ float k_scale[kTile], v_scale[kTile];
  __shared__ unsigned long long absent, poisoned;
  __shared__ int range[2];

  const int seq = blockIdx.z, head = blockIdx.y;
  const int length = sequence_length(batch, seq);
  int begin, count, base;
  new_tokens(batch, seq, begin, count, base);
  const int row0 = blockIdx.x * kRows;
  if (row0 >= count * a.group) return;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, quad = lane / 4, pair = lane % 4;

  if (threadIdx.x == 0) {
    range[0] = INT32_MAX;
    range[1] = 0;
  }
  __syncthreads();
  Row row[2];
  float slope[2];
  const uint16_t* q_row[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = row0 + warp * 16 + quad + 8 * i;
    row[i] = row_of(batch, a, begin, count, base, length, r);
    const int h = head * a.group + r % a.group;
    slope[i] = a.slopes != nullptr ? a.slopes[h] : 0.0f;
    q_row[i] = row[i].token < 0 ? nullptr : a.q + row[i].token * a.q_stride + static_cast<uint64_t>(h) * D;
    if (row[i].hi > row[i].lo) {
      atomicMin(&range[0], row[i].lo);
      atomicMax(&range[1], row[i].hi);
    }
  }
  __syncthreads();
  const int lo = range[0], hi = range[1];

  uint32_t qf[D / 16][4];
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t* p = q_row[i & 1];
      qf[k][i] = p == nullptr ? 0u : *reinterpret_cast<const uint32_t*>(p + k * 16 + (i >> 1) * 8 + pair * 2);
    }
  float o[D / 8][4] = {};
  float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f};

  for (int j0 = lo & ~(kTile - 1); j0 < hi; j0 += kTile) {
    __syncthreads();
    if (threadIdx.x == 0) absent = poisoned = 0;
    __syncthreads();
    constexpr int kChunks = D / 8;  // 16 bytes of bf16 each
    for (int c = threadIdx.x; c < kTile * kChunks; c += 128) {
      const int key = c / kChunks, chunk = c % kChunks, j = j0 + key;
      uint4 kw = make_uint4(0, 0, 0, 0), vw = kw;
      float sk = 0.0f, sv = 0.0f;
      const int page = j >= lo && j < hi ? page_of(cache, batch, seq, j) : -1;
      if (page >= 0) {
        const uint64_t r = (static_cast<uint64_t>(head) << cache.page_shift) + (j & ((1 << cache.page_shift) - 1));
        const uint64_t at = page * cache.page_stride + r * D + chunk * 8;
        bool bad = false;
        if (kFp8) {
          sk = cache.k_scale[page * cache.scale_stride + r];
          sv = cache.v_scale[page * cache.scale_stride + r];
          const uint2 kc = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(cache.k) + at);
          const uint2 vc = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(cache.v) + at);
          kw = make_uint4(bf16_of_e4m3(kc.x), bf16_of_e4m3(kc.x >> 16), bf16_of_e4m3(kc.y), bf16_of_e4m3(kc.y >> 16));
          vw = make_uint4(bf16_of_e4m3(vc.x), bf16_of_e4m3(vc.x >> 16), bf16_of_e4m3(vc.y), bf16_of_e4m3(vc.y >> 16));
          bad = !(fabsf(sv) <= FLT_MAX);
        } else {
          kw = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(cache.k) + at);
          vw = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(cache.v) + at);
        }
        bad = bad || has_nonfinite(vw.x) || has_nonfinite(vw.y) || has_nonfinite(vw.z) || has_nonfinite(vw.w);
        if (bad) atomicOr(&poisoned, 1ull << key);
      } else if (chunk == 0) {
        atomicOr(&absent, 1ull << key);
      }
      const int at = key * D + ((chunk ^ (key & 7)) * 8);
      *reinterpret_cast<uint4*>(ks + at) = kw;
      *reinterpret_cast<uint4*>(vs + at) = vw;
      if (kFp8 && chunk == 0) {
        k_scale[key] = sk;
        v_scale[key] = sv;
      }
    }
    __syncthreads();
    unsigned long long bad = poisoned;
    if (bad != 0) {  // their values reach only the rows that see them, below
      for (int c = threadIdx.x; c < kTile * kChunks; c += 128)
        if (bad >> (c / kChunks) & 1) {
          *reinterpret_cast<uint4*>(vs + c * 8) = make_uint4(0, 0, 0, 0);
        }
      __syncthreads();
      if (kFp8 && threadIdx.x < kTile && (bad >> threadIdx.x & 1)) v_scale[threadIdx.x] = 0.0f;
      __syncthreads();
    }

    float s[kTile / 8][4] = {};
#pragma unroll
    for (int n = 0; n < kTile / 8; ++n) {
#pragma unroll
      for (int k = 0; k < D / 16; k += 2) {
        uint32_t b[4];
        const int key = n * 8 + lane % 8, chunk = k * 2 + lane / 8;
        load_matrices(b, shared_address(ks + key * D + ((chunk ^ (key & 7)) * 8)));
        mma_bf16(s[n], qf[k], b[0], b[1]);
        mma_bf16(s[n], qf[k + 1], b[2], b[3]);
      }
    }
    const unsigned long long gone = absent;
    float best[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < kTile / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = n * 8 + pair * 2 + (i & 1), j = j0 + key;
        const Row& r = row[i >> 1];
        const float x = score_of(a, s[n][i] * (kFp8 ? k_scale[key] : 1.0f) * a.scale, slope[i >> 1], r.pos - j);
        s[n][i] = j >= r.lo && j < r.hi && !(gone >> key & 1) ? x : -INFINITY;
        // NaN scores are kept by the sum, not by the maximum
        best[i >> 1] = fmaxf(best[i >> 1], s[n][i]);
      }
    float keep[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      best[i] = fmaxf(best[i], __shfl_xor_sync(0xFFFFFFFFu, best[i], 1));
      best[i] = fmaxf(best[i], __shfl_xor_sync(0xFFFFFFFFu, best[i], 2));
      const float next = fmaxf(top[i], best[i]);
      keep[i] = top[i] == -INFINITY ? 0.0f : exp2_approx(top[i] - next);
      top[i] = next;
      sum[i] *= keep[i];
    }
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] *= keep[i >> 1];
    const float zero[2] = {top[0] == -INFINITY ? 0.0f : top[0], top[1] == -INFINITY ? 0.0f : top[1]};
#pragma unroll
    for (int n = 0; n < kTile / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][i] = exp2_approx(s[n][i] - zero[i >> 1]);
        sum[i >> 1] += s[n][i];
      }
    if (bad != 0) {
      for (int key = 0; key < kTile; ++key) {
        if (!(bad >> key & 1)) continue;
        const int j = j0 + key;
        const uint64_t r = (static_cast<uint64_t>(head) << cache.page_shift) + (j & ((1 << cache.page_shift) - 1));
        const int page = page_of(cache, batch, seq, j);
        if (page < 0) continue;
        float p[2] = {0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < kTile / 8; ++n)
          if (n == key / 8)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if ((i & 1) == (key & 1)) p[i >> 1] = s[n][i];
#pragma unroll
        for (int i = 0; i < 2; ++i) p[i] = __shfl_sync(0xFFFFFFFFu, p[i], (lane & ~3) | (key % 8 / 2));
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint64_t at = page * cache.page_stride + r * D + n * 8 + pair * 2 + (i & 1);
            float v;
            if (kFp8) {
              v = __uint_as_float(bf16_of_e4m3(static_cast<const uint8_t*>(cache.v)[at]) << 16) *
                  cache.v_scale[page * cache.scale_stride + r];
            } else {
              v = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(cache.v)[at]) << 16);
            }
            const Row& w = row[i >> 1];
            if (j >= w.lo && j < w.hi) o[n][i] += p[i >> 1] * v;
          }
      }
    }
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k) {
      uint32_t p[4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = s[2 * k + h][2 * i], y = s[2 * k + h][2 * i + 1];
          if (kFp8) {
            x *= v_scale[(2 * k + h) * 8 + pair * 2];
            y *= v_scale[(2 * k + h) * 8 + pair * 2 + 1];
          }
          p[h * 2 + i] = pack_bf16(x, y);
        }
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t b[4];
        const int key = k * 16 + lane % 16, chunk = n + lane / 16;
        load_matrices_transposed(b, shared_address(vs + key * D + ((chunk ^ (key & 7)) * 8)));
        mma_bf16(o[n], p, b[0], b[1]);
        mma_bf16(o[n + 1], p, b[2], b[3]);
      }
    }
  }

#pragma unroll
  for (int i = 0; i < 2; ++i) {
    sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], 1);
    sum[i] += __shfl_xor_sync(0xFFFFFFFFu, sum[i], 2);
    if (row[i].token < 0) continue;
    const int h = head * a.group + (row0 + warp * 16 + quad + 8 * i) % a.group;
    const bool some = top[i] > -INFINITY || sum[i] != sum[i];
    const float inv = some ? 1.0f / sum[i] : 0.0f;
    uint16_t* to = a.out + row[i].token * a.out_stride + static_cast<uint64_t>(h) * D;
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
      *reinterpret_cast<uint32_t*>(to + n * 8 + pair * 2) =
          some ? pack_bf16(o[n][2 * i] * inv, o[n][2 * i + 1] * inv) : 0u;
    if (a.lse != nullptr && pair == 0)
      a.lse[static_cast<uint64_t>(row[i].token) * a.q_heads + h] = some ? top[i] * kLn2 + logf(sum[i]) : -INFINITY;
  }
}

}  // namespace

uint64_t attention_workspace_bytes(int head_dim, int) { return few_rows_workspace_bytes(head_dim); }

cudaError_t launch_attention(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                             const AttentionArgs& args, void* workspace, cudaStream_t stream) {
  if (static_cast<int64_t>(batch.max_new) * args.group <= 16)
    return launch_few_rows(cache, fp8, head_dim, batch, args, workspace, stream);
  const int64_t tiles = (static_cast<int64_t>(batch.max_new) * args.group + kRows - 1) / kRows;
  if (tiles > INT32_MAX) return cudaErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(cache.kv_heads),
                  static_cast<unsigned>(batch.sequences));
  auto kernel = head_dim == 128 ? (fp8 ? attention_kernel<128, true> : attention_kernel<128, false>)
                                : (fp8 ? attention_kernel<64, true> : attention_kernel<64, false>);
  kernel<<<grid, 128, 0, stream>>>(cache, batch, args);
  return cudaGetLastError();
}

}  // namespace esopt
