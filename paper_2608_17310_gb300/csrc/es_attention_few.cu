// es_attention of up to 16 rows per (sequence, key head): single tokens, and a few drafted
// or queued ones.
//
// What bounds it is reading the cache once: 4 D bytes a key and head in bf16, 2 D + 8 in
// FP8, against 2 D operations a byte at most for the tensor cores. So the keys go from
// memory straight into the registers that the products take them from, without shared
// memory:
//   S^T = K Q^T   m16n8k16, 16 keys x 8 rows; the order of the D products of a dot is free,
//                 so a lane loads 16 bytes of a key and pairs them with the same elements of q;
//   O^T = V^T P^T 16 elements of v x 8 rows over 16 keys; the order of the elements is free
//                 too, so a lane loads 16 bytes of four keys and packs pairs of keys
//                 with byte permutes.
// P^T comes out of S^T by transposing 8 x 8 blocks within the warp. FP8 codes become f16,
// which holds them exactly, and the products run in f16 with q and p v_scale scaled by powers of
// two into its range: q by its row's largest element, p v_scale by the row's largest so far.
//
// The tiles of all (sequence, key head) units lie end to end and are cut into one range per
// block, all of one length, whatever the sequences' lengths. A unit that several blocks
// share is joined by the last of them to finish, from the parts in the order of the blocks,
// so results do not depend on who is last.
//
// Measured (GB300; 4 or 5 rows of 8 key heads of 128): 96 bf16 caches of 200 to 9,000 tokens
// 280 us, 6.6 TB/s, 98 % of the card's copy rate; three FP8 caches of 90,000 to 131,071 tokens
// 127 us, 5.7 TB/s, 85 %, where converting and packing codes keeps the integer pipe 47 % busy and
// the loads in flight are what registers hold (16 warps of 4 KB an SM); one cache of 777
// tokens 8.1 us, 15,500 cycles of latency (lengths, pages, keys, a part's way through
// memory, the join) in code that each launch reads anew.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "es_attention.cuh"
#include "es_rollout_internal.h"

namespace esopt {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

template <bool kFp8>
struct Shape {
  // 16-key blocks that a warp takes at a time. Two for FP8, with 12 warps an SM in place of 16,
  // measured 141 us against 132 (three caches of up to 131,071 tokens).
  static constexpr int subs = 1;
  static constexpr int warp_keys = 16 * subs;
  static constexpr int tile = kWarps * warp_keys;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool kFp8>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (kFp8) mma_f16(c, a, b0, b1); else mma_bf16(c, a, b0, b1);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t w) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(w));
  return y;
}

// 2^n for n in [-126, 127]
__device__ __forceinline__ float power_of_two(int n) { return __int_as_float((n + 127) << 23); }

// The power of two at or below x > 0, as an exponent within [-126, 127].
__device__ __forceinline__ int exponent_of(float x) { return max((__float_as_int(x) >> 23 & 0xFF) - 127, -126); }

// FP8: exp(x) v_scale becomes f16 in units of 2^(u - 14), where u is this of the row's largest such
// product (log 2 of a bound within a factor of 2): the largest is at least 2^12 then and below 2^14, so
// products keep 11 bits down to 2^-28 of it and are off by 2^-37 of it below. Units that go by the scales
// alone would leave nothing of a key with all of the weight and a scale 2^-40 of another's.
__device__ __forceinline__ float unit_of(float largest) { return ceilf(fminf(fmaxf(largest, -112.0f), 127.0f)); }

// An exponent e with |scale| < 2^e <= 2 |scale|, for scales that are finite and not tiny.
__device__ __forceinline__ float size_bound(float scale) {
  const int e = __float_as_int(scale) >> 23 & 0xFF;
  return e == 255 ? -INFINITY : static_cast<float>(e - 126);
}

template <int kBytes> struct Bytes;
template <> struct Bytes<16> { using type = uint4; };
template <> struct Bytes<8> { using type = uint2; };

// A warp's 16 keys and values of one head, as loaded. A lane (g, t) = (lane / 4, lane % 4)
// holds elements of keys g and g + 8, and of values 2t, 2t + 1, 2t + 8, 2t + 9.
template <int D, bool kFp8>
struct Block {
  static constexpr int kk = kFp8 ? D / 64 : D / 32;  // 16-byte pieces of a key
  static constexpr int vbytes = kFp8 && D == 64 ? 8 : 16;
  static constexpr int vv = kFp8 ? 1 : D / 64;       // pieces of a value
  using V = typename Bytes<vbytes>::type;
  uint4 k[2][kk];
  V v[4][vv];
  float k_scale[2], v_scale[2];

  // From a page that exists; what the page's place in the sequence does not hold is masked
  // by the caller.
  __device__ __forceinline__ void load_keys(const CacheView& c, int page, uint32_t row, int lane) {
    const int g = lane / 4, t = lane % 4;
    const char* from = static_cast<const char*>(c.k) +
                       (page * c.page_stride + row * D + g * D + t * (kFp8 ? 16 : 8)) * (kFp8 ? 1 : 2);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int p = 0; p < kk; ++p)
        k[i][p] = __ldg(reinterpret_cast<const uint4*>(from + i * 8 * D * (kFp8 ? 1 : 2) + p * 64));
    if (kFp8) {
      const uint64_t s = page * c.scale_stride + row + g;
      k_scale[0] = __ldg(c.k_scale + s);
      k_scale[1] = __ldg(c.k_scale + s + 8);
    }
  }

  __device__ __forceinline__ void load_values(const CacheView& c, int page, uint32_t row, int lane) {
    const int g = lane / 4, t = lane % 4;
    const char* from = static_cast<const char*>(c.v) +
                       (page * c.page_stride + row * D + 2 * t * D) * (kFp8 ? 1 : 2) + g * vbytes;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int p = 0; p < vv; ++p)
        v[i][p] = __ldg(reinterpret_cast<const V*>(from + ((i & 1) + 8 * (i >> 1)) * D * (kFp8 ? 1 : 2) + p * 128));
    if (kFp8) {  // as the scores lie: keys g and g + 8
      const uint64_t s = page * c.scale_stride + row + g;
      v_scale[0] = __ldg(c.v_scale + s);
      v_scale[1] = __ldg(c.v_scale + s + 8);
    }
  }

  __device__ __forceinline__ uint32_t key_word(int i, int w) const {
    const uint4& x = k[i][w / 4];
    return w % 4 == 0 ? x.x : w % 4 == 1 ? x.y : w % 4 == 2 ? x.z : x.w;
  }
  __device__ __forceinline__ uint32_t value_word(int i, int w) const {
    const V& x = v[i][w / (vbytes / 4)];
    if constexpr (vbytes == 16) {
      const int u = w % 4;
      return u == 0 ? x.x : u == 1 ? x.y : u == 2 ? x.z : x.w;
    } else {
      return w % 2 == 0 ? x.x : x.y;
    }
  }
  __device__ __forceinline__ void clear_value(int i) {
#pragma unroll
    for (int p = 0; p < vv; ++p) v[i][p] = V{};
  }
  // Whether value i of this lane holds an infinity or NaN.
  __device__ __forceinline__ bool bad_value(int i) const {
    bool bad = false;
#pragma unroll
    for (int w = 0; w < vv * vbytes / 4; ++w) {
      const uint32_t x = value_word(i, w);
      if (kFp8) bad = bad || (((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
      else bad = bad || has_nonfinite(x);
    }
    return bad;
  }
  // The products' A operands: 16 keys x 16 elements, and 16 elements x 16 keys.
  __device__ __forceinline__ void key_operand(int s, uint32_t (&a)[4]) const {
    if (kFp8) {
      const uint32_t lo = key_word(0, s), hi = key_word(1, s);
      a[0] = f16_of_e4m3(lo);
      a[1] = f16_of_e4m3(hi);
      a[2] = f16_of_e4m3(lo >> 16);
      a[3] = f16_of_e4m3(hi >> 16);
    } else {
      a[0] = key_word(0, 2 * s);
      a[1] = key_word(1, 2 * s);
      a[2] = key_word(0, 2 * s + 1);
      a[3] = key_word(1, 2 * s + 1);
    }
  }
  __device__ __forceinline__ void value_operand(int m, uint32_t (&a)[4]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t x, y;
      if (kFp8) {
        x = f16_of_e4m3(value_word(2 * h, m / 2) >> (16 * (m % 2)));
        y = f16_of_e4m3(value_word(2 * h + 1, m / 2) >> (16 * (m % 2)));
      } else {
        x = value_word(2 * h, m);
        y = value_word(2 * h + 1, m);
      }
      a[2 * h] = __byte_perm(x, y, 0x5410);
      a[2 * h + 1] = __byte_perm(x, y, 0x7632);
    }
  }
};

// A row's interval, position and slope (as bits). The kernel keeps them in shared memory,
// since only the blocks at the ends of the intervals and biased scores need them: in
// registers they would cost the loads in flight.
__device__ __forceinline__ int4 row_info(const int4* p) {
  int4 r;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "r"(shared_address(p)));
  return r;
}

// The element of a head that row g of product m of a lane stands for (g + 8: the next one).
template <int D, bool kFp8>
__device__ __forceinline__ int element_of(int m, int g) {
  if (kFp8) return g * (D / 8) + 2 * m;
  return m / 4 * 64 + g * 8 + m % 4 * 2;
}

// What a sequence's rows see: their count, and the union and the common part of their
// intervals of the cache. Called by whole warps.
struct Span {
  int begin, count, base, length;
  int lo, hi;          // some row sees nothing outside
  int in_lo, in_hi;    // every row sees all inside
};

__device__ __forceinline__ Span span_of(const BatchView& b, const AttentionArgs& a, int seq, int lane) {
  Span s;
  s.length = sequence_length(b, seq);
  new_tokens(b, seq, s.begin, s.count, s.base);
  if (b.max_new == 1) {  // every lane works out the one token: 20 shuffles less before the first load
    const Row r = row_of(b, a, s.begin, s.count, s.base, s.length, 0);
    s.lo = s.in_lo = r.lo;
    s.hi = s.in_hi = r.hi;
    return s;
  }
  int lo = INT32_MAX, hi = 0, in_lo = 0, in_hi = INT32_MAX;
  if (lane < s.count) {
    const Row r = row_of(b, a, s.begin, s.count, s.base, s.length, lane * a.group);
    if (r.hi > r.lo) {
      lo = r.lo;
      hi = r.hi;
    }
    in_lo = r.lo;
    in_hi = r.hi;
  }
#pragma unroll
  for (int m = 8; m > 0; m >>= 1) {  // at most 16 rows
    lo = min(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, m));
    hi = max(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, m));
    in_lo = max(in_lo, __shfl_xor_sync(0xFFFFFFFFu, in_lo, m));
    in_hi = min(in_hi, __shfl_xor_sync(0xFFFFFFFFu, in_hi, m));
  }
  s.lo = __shfl_sync(0xFFFFFFFFu, lo, 0);
  s.hi = __shfl_sync(0xFFFFFFFFu, hi, 0);
  s.in_lo = __shfl_sync(0xFFFFFFFFu, in_lo, 0);
  s.in_hi = __shfl_sync(0xFFFFFFFFu, in_hi, 0);
  if (s.hi <= s.lo) s.lo = s.hi = 0;
  return s;
}

// Tiles of one key head of a sequence; one at least where there are rows, so that rows which
// see nothing are written too.
__device__ __forceinline__ int tiles_of(int count, int lo, int hi, int tile) {
  if (count == 0) return 0;
  return max(1, (hi - (lo & ~15) + tile - 1) / tile);
}

__device__ __forceinline__ int tiles_of(const BatchView& b, const AttentionArgs& a, int seq, int tile) {
  const int length = sequence_length(b, seq);
  int begin, count, base;
  new_tokens(b, seq, begin, count, base);
  int lo = INT32_MAX, hi = 0;
  for (int i = 0; i < count; ++i) {
    const Row r = row_of(b, a, begin, count, base, length, i * a.group);
    if (r.hi > r.lo) {
      lo = min(lo, r.lo);
      hi = max(hi, r.hi);
    }
  }
  if (hi <= lo) lo = hi = 0;
  return tiles_of(count, lo, hi, tile);
}

// The parts of units that blocks share: block c's first unit, if it began in an earlier block,
// is part 2c, and its last one, if it began here, part 2c + 1.
template <int D>
struct Part {
  float o[16][D];
  float top[16], sum[16];
};

constexpr int kMinTiles = 1;  // of a block's range
constexpr int kMaxParts = 2 * kCounters;  // two for each block

template <int D, bool kFp8, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks == 1 ? (kFp8 ? 4 : 3) : 2)
few_rows_kernel(const CacheView cache, const BatchView batch, const AttentionArgs a, uint32_t* counters,
                Part<D>* parts) {
  using S = Shape<kFp8>;
  constexpr int kSubs = S::subs;
  constexpr int kRows = 8 * kBlocks;
  __shared__ float o_of[kWarps][kRows][D + 4];
  __shared__ float top_of[kWarps][kRows], sum_of[kWarps][kRows];
  __shared__ int64_t warp_tiles[kWarps];
  __shared__ int64_t first_tile;
  __shared__ int first_seq;
  __shared__ bool is_last;
  __shared__ __align__(16) int4 info[kWarps][kRows];

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;

  wait_for_previous();
  // This block's range of tiles: every thread counts a run of sequences.
  const int run = (batch.sequences + kThreads - 1) / kThreads;
  const int run0 = threadIdx.x * run, run1 = min(run0 + run, batch.sequences);
  int64_t mine = 0;
  for (int s = run0; s < run1; ++s) mine += tiles_of(batch, a, s, S::tile);
  mine *= cache.kv_heads;
  int64_t upto = mine;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const int64_t x = __shfl_up_sync(0xFFFFFFFFu, upto, m);
    if (lane >= m) upto += x;
  }
  if (lane == 31) warp_tiles[warp] = upto;
  __syncthreads();
  int64_t all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) upto += warp_tiles[w];
    all += warp_tiles[w];
  }
  const int64_t share = all <= UINT32_MAX - gridDim.x ? (static_cast<uint32_t>(all) + gridDim.x - 1) / gridDim.x
                                                     : (all + gridDim.x - 1) / gridDim.x;
  const int64_t per = max(share, static_cast<int64_t>(kMinTiles));
  const int64_t begin = blockIdx.x * per, end = min(begin + per, all);
  if (begin >= end) return;  // which lets the next kernel start too
  if (begin >= upto - mine && begin < upto) {
    int64_t at = upto - mine;
    for (int s = run0;; ++s) {
      const int64_t n = static_cast<int64_t>(tiles_of(batch, a, s, S::tile)) * cache.kv_heads;
      if (begin < at + n) {
        first_seq = s;
        first_tile = at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();

  int seq = first_seq;
  int64_t seq_tile = first_tile;  // the sequence's first tile in the space of all
  Span span = span_of(batch, a, seq, lane);
  int tiles = tiles_of(span.count, span.lo, span.hi, S::tile);
  for (int64_t at = begin; at < end;) {
    while (at >= seq_tile + static_cast<int64_t>(tiles) * cache.kv_heads) {
      seq_tile += static_cast<int64_t>(tiles) * cache.kv_heads;
      ++seq;
      span = span_of(batch, a, seq, lane);
      tiles = tiles_of(span.count, span.lo, span.hi, S::tile);
    }
    const int64_t into = at - seq_tile;
    const int head = into <= UINT32_MAX ? static_cast<int>(static_cast<uint32_t>(into) / static_cast<uint32_t>(tiles))
                                        : static_cast<int>(into / tiles);
    const int64_t unit0 = seq_tile + static_cast<int64_t>(head) * tiles, unit1 = unit0 + tiles;
    const int tile0 = static_cast<int>(at - unit0);
    const int tile1 = static_cast<int>(min(unit1, end) - unit0);

    // --- the unit's rows: 8 n + 2 t, + 1 in the products' columns of this lane
    float factor[kBlocks][2];  // of a dot product, for a score in units of log 2 (plain scores)
    uint32_t q[kBlocks][D / 16][2];
    const bool plain = a.softcap <= 0.0f && a.slopes == nullptr;
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      float q_unit = 1.0f;
      const int r = 8 * n + g;  // the row whose elements this lane holds for the products
      const uint16_t* from = r < span.count * a.group
          ? a.q + (span.begin + r / a.group) * a.q_stride + static_cast<uint64_t>(head * a.group + r % a.group) * D
          : nullptr;
      if (kFp8) {
        float x[D / 64][16];
        float most = 0.0f;
#pragma unroll
        for (int p = 0; p < D / 64; ++p)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 w = from ? *reinterpret_cast<const uint4*>(from + p * 64 + t * 16 + h * 8) : make_uint4(0, 0, 0, 0);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[p][h * 8 + 2 * i] = __uint_as_float(u[i] << 16);
              x[p][h * 8 + 2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
              most = fmaxf(most, fmaxf(fabsf(x[p][h * 8 + 2 * i]), fabsf(x[p][h * 8 + 2 * i + 1])));
            }
          }
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        // q / 2^e is below 2^15, and a dot with codes below 2^15 D 448: f16 and fp32 hold both. Elements
        // stay exact down to 2^-31 of the row's largest, where f16 numbers are 2^-24 apart.
        const int e = max(min(exponent_of(most), 127) - 14, -126);
        q_unit = power_of_two(e);
        const float inv = power_of_two(-e);
#pragma unroll
        for (int p = 0; p < D / 64; ++p)
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              q[n][p * 4 + s][h] = pack_f16(x[p][s * 4 + 2 * h] * inv, x[p][s * 4 + 2 * h + 1] * inv);
      } else {
#pragma unroll
        for (int p = 0; p < D / 32; ++p) {
          const uint4 w = from ? *reinterpret_cast<const uint4*>(from + p * 32 + t * 8) : make_uint4(0, 0, 0, 0);
          q[n][2 * p][0] = w.x;
          q[n][2 * p][1] = w.y;
          q[n][2 * p + 1][0] = w.z;
          q[n][2 * p + 1][1] = w.w;
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // the unit of row 2 t + i is with the lanes of g = 2 t + i
        factor[n][i] = a.scale * __shfl_sync(0xFFFFFFFFu, q_unit, (2 * t + i) * 4);
        if (plain) factor[n][i] *= kLog2e;
      }
    }

    if (lane < kRows) {
      const Row r = row_of(batch, a, span.begin, span.count, span.base, span.length, lane);
      const float slope = a.slopes != nullptr ? a.slopes[head * a.group + lane % a.group] : 0.0f;
      info[warp][lane] = make_int4(r.lo, r.hi, r.pos, __float_as_int(slope));
    }
    __syncwarp();

    float o[kBlocks][D / 16][4] = {};
    float top[kBlocks][2], sum[kBlocks][2];
    // FP8: log 2 of a bound of the row's largest p |v_scale| so far, with its top, within a factor of 2
    float largest[kBlocks][2];
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      top[n][0] = top[n][1] = -INFINITY;
      sum[n][0] = sum[n][1] = 0.0f;
      largest[n][0] = largest[n][1] = -INFINITY;
    }

    // --- the keys, a block of 16 per sub and warp, loaded one tile ahead
    const int origin = span.lo & ~15;
    auto key_of = [&](int tile, int sub) { return origin + tile * S::tile + warp * S::warp_keys + sub * 16; };
    auto page_at = [&](int tile, int sub) {
      const int j = key_of(tile, sub);
      return tile < tile1 && j < span.hi ? page_of(cache, batch, seq, j) : -1;
    };
    auto row_at = [&](int tile, int sub) {  // of the page's rows of all heads
      return (static_cast<uint32_t>(head) << cache.page_shift) + (key_of(tile, sub) & ((1 << cache.page_shift) - 1));
    };
    Block<D, kFp8> block[kSubs];
    int page[kSubs], next_page[kSubs];  // -1: no tokens, and what is loaded from page 0 instead is masked
#pragma unroll
    for (int u = 0; u < kSubs; ++u) {
      page[u] = page_at(tile0, u);
      block[u].load_keys(cache, max(page[u], 0), row_at(tile0, u), lane);
      block[u].load_values(cache, max(page[u], 0), row_at(tile0, u), lane);
      next_page[u] = page_at(tile0 + 1, u);
    }
    for (int tile = tile0; tile < tile1; ++tile) {
      float s[kSubs][kBlocks][4];
      const bool more = tile + 1 < tile1;
      float best[kBlocks][2];
#pragma unroll
      for (int n = 0; n < kBlocks; ++n) best[n][0] = best[n][1] = -INFINITY;
#pragma unroll
      for (int u = 0; u < kSubs; ++u) {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) s[u][n][0] = s[u][n][1] = s[u][n][2] = s[u][n][3] = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          uint32_t w[4];
          block[u].key_operand(k, w);
#pragma unroll
          for (int n = 0; n < kBlocks; ++n) mma<kFp8>(s[u][n], w, q[n][k][0], q[n][k][1]);
        }
        const int j0 = key_of(tile, u);
        const float k_scale[2] = {kFp8 ? block[u].k_scale[0] : 1.0f, kFp8 ? block[u].k_scale[1] : 1.0f};
        // the next tile's keys are on their way while this one's scores are worked on
        if (more) block[u].load_keys(cache, max(next_page[u], 0), row_at(tile + 1, u), lane);
        const bool whole = page[u] >= 0 && j0 >= span.in_lo && j0 + 16 <= span.in_hi;
        if (plain && whole) {
#pragma unroll
          for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              s[u][n][i] *= kFp8 ? factor[n][i & 1] * k_scale[i >> 1] : factor[n][i & 1];
              best[n][i & 1] = fmaxf(best[n][i & 1], s[u][n][i]);  // a NaN stays with the sum
            }
        } else {
#pragma unroll
          for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int4 r = row_info(&info[warp][8 * n + 2 * t + c]);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int j = j0 + g + 8 * h;
                float x = s[u][n][c + 2 * h] * (kFp8 ? factor[n][c] * k_scale[h] : factor[n][c]);
                if (!plain) x = score_of(a, x, __int_as_float(r.w), r.z - j);
                const bool seen = whole || (page[u] >= 0 && j >= r.x && j < r.y);
                if (!seen) x = -INFINITY;
                s[u][n][c + 2 * h] = x;
                best[n][c] = fmaxf(best[n][c], x);
              }
            }
        }
      }
      // running maxima
      bool grows = false;
      float keep[kBlocks][2], rise[kBlocks][2];
#pragma unroll
      for (int n = 0; n < kBlocks; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int m = 4; m < 32; m <<= 1) best[n][c] = fmaxf(best[n][c], __shfl_xor_sync(0xFFFFFFFFu, best[n][c], m));
          const float next = fmaxf(top[n][c], best[n][c]);
          grows = grows || next > top[n][c];
          rise[n][c] = next > top[n][c] ? next - top[n][c] : 0.0f;
          keep[n][c] = exp2_approx(-rise[n][c]);
          top[n][c] = next;
        }
      if (kFp8) {
        // this tile's products, of this lane's keys; they may need a larger unit
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float zero = top[n][c] == -INFINITY ? 0.0f : top[n][c];
            best[n][c] = -INFINITY;
#pragma unroll
            for (int u = 0; u < kSubs; ++u)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                best[n][c] = fmaxf(best[n][c], s[u][n][c + 2 * h] - zero + size_bound(block[u].v_scale[h]));
            grows = grows || best[n][c] > unit_of(largest[n][c]);
          }
      }
      if (__any_sync(0xFFFFFFFFu, grows)) {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            sum[n][c] *= keep[n][c];
            if (kFp8) {
#pragma unroll
              for (int m = 4; m < 32; m <<= 1) best[n][c] = fmaxf(best[n][c], __shfl_xor_sync(0xFFFFFFFFu, best[n][c], m));
              // by what this row has seen alone, whatever row made the warp come here
              const float unit = unit_of(largest[n][c]);
              if (rise[n][c] > 0.0f || best[n][c] > unit) largest[n][c] = fmaxf(largest[n][c] - rise[n][c], best[n][c]);
              const float step = fminf(fmaxf(unit - unit_of(largest[n][c]), -126.0f), 127.0f);
              keep[n][c] *= power_of_two(static_cast<int>(step));
            }
          }
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][m][i] *= keep[n][i & 1];
        }
      }
      float v_factor[kBlocks][2];
      if (kFp8) {
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) v_factor[n][c] = power_of_two(14 - static_cast<int>(unit_of(largest[n][c])));
      }
#pragma unroll
      for (int u = 0; u < kSubs; ++u) {
        const int j0 = key_of(tile, u);
        uint32_t p[kBlocks][2];
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float zero = top[n][i & 1] == -INFINITY ? 0.0f : top[n][i & 1];
            s[u][n][i] = exp2_approx(s[u][n][i] - zero);
            sum[n][i & 1] += s[u][n][i];
          }
        }
        const bool inside = j0 >= span.in_lo && j0 + 16 <= span.in_hi;
        uint32_t bad = 0;  // keys whose values hold an infinity or NaN that some row does not see
        if (!inside || page[u] < 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = 2 * t + (i & 1) + 8 * (i >> 1), j = j0 + key;
            if (j < span.lo || j >= span.hi || page[u] < 0) block[u].clear_value(i);
            else if (block[u].bad_value(i)) bad |= 1u << key;
          }
          if (kFp8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int j = j0 + g + 8 * h;
              if (j < span.lo || j >= span.hi || page[u] < 0) block[u].v_scale[h] = 0.0f;
              else if (!(fabsf(block[u].v_scale[h]) <= FLT_MAX)) bad |= 1u << (g + 8 * h);
            }
          }
          bad = __reduce_or_sync(0xFFFFFFFFu, bad);
          if (bad != 0) {
            const uint64_t at_row = row_at(tile, u);
            const uint64_t pg = static_cast<uint64_t>(page[u]);
            for (int key = 0; key < 16; ++key) {
              if (!(bad >> key & 1)) continue;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (key == 2 * t + (i & 1) + 8 * (i >> 1)) block[u].clear_value(i);
              const float own = kFp8 ? cache.v_scale[pg * cache.scale_stride + at_row + key] : 1.0f;
#pragma unroll
              for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const float x = key < 8 ? s[u][n][c] : s[u][n][c + 2];
                  const float w = __shfl_sync(0xFFFFFFFFu, x, key % 8 * 4 + t) * own * (kFp8 ? v_factor[n][c] : 1.0f);
                  const int4 r = row_info(&info[warp][8 * n + 2 * t + c]);
                  if (j0 + key < r.x || j0 + key >= r.y) continue;
#pragma unroll
                  for (int m = 0; m < D / 16; ++m)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                      const uint64_t from = pg * cache.page_stride + (at_row + key) * D + element_of<D, kFp8>(m, g) + e;
                      const float v = kFp8
                          ? __uint_as_float(bf16_of_e4m3(static_cast<const uint8_t*>(cache.v)[from]) << 16)
                          : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(cache.v)[from]) << 16);
                      o[n][m][2 * e + c] += w * v;
                    }
                }
            }
            if (kFp8) {
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (bad >> (g + 8 * h) & 1) block[u].v_scale[h] = 0.0f;
            }
          }
        }
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (kFp8) {
              p[n][h] = transpose8x8(pack_f16(s[u][n][2 * h] * block[u].v_scale[h] * v_factor[n][0],
                                              s[u][n][2 * h + 1] * block[u].v_scale[h] * v_factor[n][1]));
            } else {
              p[n][h] = transpose8x8(pack_bf16(s[u][n][2 * h], s[u][n][2 * h + 1]));
            }
          }
#pragma unroll
        for (int m = 0; m < D / 16; ++m) {
          uint32_t w[4];
          block[u].value_operand(m, w);
#pragma unroll
          for (int n = 0; n < kBlocks; ++n) mma<kFp8>(o[n][m], w, p[n][0], p[n][1]);
        }
        if (more) block[u].load_values(cache, max(next_page[u], 0), row_at(tile + 1, u), lane);
        page[u] = next_page[u];
        next_page[u] = page_at(tile + 2, u);
      }
    }

    if (unit0 + tile1 >= end) let_next_start();

    // --- join the warps
#pragma unroll
    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int m = 4; m < 32; m <<= 1) sum[n][c] += __shfl_xor_sync(0xFFFFFFFFu, sum[n][c], m);
        const int r = 8 * n + 2 * t + c;
        const float o_unit = kFp8 ? power_of_two(static_cast<int>(unit_of(largest[n][c])) - 14) : 1.0f;
        if (g == 0) {
          top_of[warp][r] = top[n][c];
          sum_of[warp][r] = sum[n][c];
        }
#pragma unroll
        for (int m = 0; m < D / 16; ++m)
          *reinterpret_cast<float2*>(&o_of[warp][r][element_of<D, kFp8>(m, g)]) =
              make_float2(o[n][m][c] * o_unit, o[n][m][2 + c] * o_unit);
      }
    __syncthreads();

    const int c_first = static_cast<int>(unit0 / per), c_last = static_cast<int>((unit1 - 1) / per);
    const int rows = span.count * a.group;
    constexpr int kCols = D / 4;
    const int self = static_cast<int>(blockIdx.x);
    if (c_first != c_last) {
      Part<D>& part = parts[self == c_first ? 2 * self + 1 : 2 * self];
      for (int i = threadIdx.x; i < rows * kCols; i += kThreads) {
        const int r = i / kCols, col = i % kCols * 4;
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) most = fmaxf(most, top_of[w][r]);
        const float zero = most == -INFINITY ? 0.0f : most;
        float4 x = make_float4(0, 0, 0, 0);
        float l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = exp2_approx(top_of[w][r] - zero);
          const float4 y = *reinterpret_cast<const float4*>(&o_of[w][r][col]);
          x.x += y.x * f;
          x.y += y.y * f;
          x.z += y.z * f;
          x.w += y.w * f;
          l += sum_of[w][r] * f;
        }
        *reinterpret_cast<float4*>(&part.o[r][col]) = x;
        if (col == 0) {
          part.top[r] = most;
          part.sum[r] = l;
        }
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        is_last = count_done(&counters[c_first]) == static_cast<uint32_t>(c_last - c_first);
        if (is_last) counters[c_first] = 0;
      }
      __syncthreads();
    }
    if (c_first == c_last || is_last) {
      // a warp for each row, a lane for D / 32 of its elements
      constexpr int kPer = D / 32;
      for (int r = warp; r < rows; r += kWarps) {
        float most = -INFINITY, l = 0.0f, x[kPer] = {};
        if (c_first == c_last) {
#pragma unroll
          for (int w = 0; w < kWarps; ++w) most = fmaxf(most, top_of[w][r]);
          const float zero = most == -INFINITY ? 0.0f : most;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float f = exp2_approx(top_of[w][r] - zero);
#pragma unroll
            for (int i = 0; i < kPer; ++i) x[i] += o_of[w][r][lane * kPer + i] * f;
            l += sum_of[w][r] * f;
          }
        } else {
          // the parts' maxima and sums a lane each, their elements eight loads at a time
          const int n = c_last - c_first + 1;
          auto part_of = [&](int i) -> const Part<D>& { return parts[2 * (c_first + i) + (i == 0)]; };
          float first_top = -INFINITY, first_sum = 0.0f;  // of the first 32 parts
          if (lane < n) {
            first_top = __ldcg(&part_of(lane).top[r]);
            first_sum = __ldcg(&part_of(lane).sum[r]);
          }
          most = first_top;
          for (int i = lane + 32; i < n; i += 32) most = fmaxf(most, __ldcg(&part_of(i).top[r]));
#pragma unroll
          for (int m = 16; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, m));
          const float zero = most == -INFINITY ? 0.0f : most;
          for (int i0 = 0; i0 < n; i0 += 32) {
            const int some = min(n - i0, 32);
            float f = 0.0f;
            if (lane < some) {
              f = exp2_approx((i0 == 0 ? first_top : __ldcg(&part_of(i0 + lane).top[r])) - zero);
              l += (i0 == 0 ? first_sum : __ldcg(&part_of(i0 + lane).sum[r])) * f;
            }
#pragma unroll 1
            for (int i = 0; i < some; i += 8) {  // eight loads in flight, the last batch's too
              float y[8][kPer];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float* from = &part_of(i0 + min(i + e, some - 1)).o[r][lane * kPer];
                if constexpr (kPer == 4) {
                  const float4 z = __ldcg(reinterpret_cast<const float4*>(from));
                  y[e][0] = z.x;
                  y[e][1] = z.y;
                  y[e][2] = z.z;
                  y[e][3] = z.w;
                } else {
                  const float2 z = __ldcg(reinterpret_cast<const float2*>(from));
                  y[e][0] = z.x;
                  y[e][1] = z.y;
                }
              }
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float g = __shfl_sync(0xFFFFFFFFu, f, min(i + e, 31));
                if (i + e < some)
#pragma unroll
                  for (int j = 0; j < kPer; ++j) x[j] += y[e][j] * g;
              }
            }
          }
#pragma unroll
          for (int m = 16; m > 0; m >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, m);
        }
        const int token = span.begin + r / a.group, h = head * a.group + r % a.group;
        const bool some = most > -INFINITY || l != l;
        const float inv = some ? 1.0f / l : 0.0f;
        uint32_t* to = reinterpret_cast<uint32_t*>(a.out + token * a.out_stride + static_cast<uint64_t>(h) * D + lane * kPer);
        if constexpr (kPer == 4)
          *reinterpret_cast<uint2*>(to) = some ? make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv))
                                               : make_uint2(0, 0);
        else
          *to = some ? pack_bf16(x[0] * inv, x[1] * inv) : 0u;
        if (lane == 0 && a.lse != nullptr)
          a.lse[static_cast<uint64_t>(token) * a.q_heads + h] = some ? most * kLn2 + logf(l) : -INFINITY;
      }
    }
    at = unit0 + tile1;
    if (at < end) __syncthreads();  // the joined rows have been read
  }
}

template <int D, bool kFp8, int kBlocks>
cudaError_t launch(const CacheView& cache, const BatchView& batch, const AttentionArgs& args,
                   char* workspace, uint32_t* counters, cudaStream_t stream) {
  auto kernel = few_rows_kernel<D, kFp8, kBlocks>;
  int device = 0;
  cudaGetDevice(&device);
  // resident blocks of this kernel on each device, kept from its first launch there
  static std::atomic<int> blocks_of[64];
  int resident = device < 64 ? blocks_of[device].load(std::memory_order_relaxed) : 0;
  if (resident == 0) {
    int sms = 0, per_sm = 0;
    cudaError_t err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (err == cudaSuccess) err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, 0);
    if (err != cudaSuccess) {
      cudaGetLastError();
      return err;
    }
    resident = std::max(sms * per_sm, 1);
    if (device < 64) blocks_of[device].store(resident, std::memory_order_relaxed);
  }
  // no more blocks than the longest sequences that the page table allows have work for
  const int64_t longest = (static_cast<int64_t>(batch.capacity) + 15 + Shape<kFp8>::tile - 1) / Shape<kFp8>::tile;
  const int64_t tiles = longest * cache.kv_heads * batch.sequences;
  const int64_t blocks = std::min({static_cast<int64_t>(resident), static_cast<int64_t>(kMaxParts / 2), (tiles + kMinTiles - 1) / kMinTiles});
  return launch_early(kernel, static_cast<int>(blocks), kThreads, 0, stream, cache, batch, args, counters,
                      reinterpret_cast<Part<D>*>(workspace));
}

template <int D, bool kFp8>
cudaError_t launch_rows(const CacheView& cache, const BatchView& batch, const AttentionArgs& args,
                        char* workspace, uint32_t* counters, cudaStream_t stream) {
  return batch.max_new * args.group <= 8 ? launch<D, kFp8, 1>(cache, batch, args, workspace, counters, stream)
                                         : launch<D, kFp8, 2>(cache, batch, args, workspace, counters, stream);
}

}  // namespace

uint64_t few_rows_workspace_bytes(int head_dim) {
  return kMaxParts * (head_dim == 128 ? sizeof(Part<128>) : sizeof(Part<64>));
}

cudaError_t launch_few_rows(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                            const AttentionArgs& args, char* workspace, uint32_t* counters, cudaStream_t stream) {
  auto f = head_dim == 128 ? (fp8 ? launch_rows<128, true> : launch_rows<128, false>)
                           : (fp8 ? launch_rows<64, true> : launch_rows<64, false>);
  return f(cache, batch, args, workspace, counters, stream);
}

}  // namespace esopt
