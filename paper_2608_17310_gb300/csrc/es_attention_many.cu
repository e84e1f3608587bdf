// es_attention of more than 16 rows per (sequence, key head): prompts, and turns of some
// tokens over longer caches.
//
// What bounds it is the tensor cores, 4 D operations a row and key, and the exponentials,
// one a row and key. A block takes 256 rows of a key head as two tiles x = 0, 1 of 128, and
// walks its keys in tiles of 128:
//   S_x = Q_x K^T     tcgen05, Q and K in shared memory, S in tensor memory
//   P_x = 2^(S_x - m) a warpgroup for each x, a thread for each row: S is read from tensor
//                     memory, P written back over it as bf16
//   O_x += P_x V      tcgen05, P in tensor memory, V in shared memory, O in tensor memory
// One thread issues the products in the order P_0 V, Q_0 K', P_1 V, Q_1 K', so that each
// warpgroup's exponentials run beside the other tile's products. The running maximum m only
// moves where a tile's maximum is more than 2^8 above it, which keeps P in bf16's range
// and leaves O in tensor memory alone on almost every tile.
//
// Pages reach shared memory by TMA, each page of a tile by its own copy; FP8 pages then pass
// through six warps that turn codes into bf16, which holds them exactly. The scales go to the
// scores and to P.
//
// The key tiles of all units (sequence, row tile, key head) lie end to end and are cut into
// one range per block, all of one length, so causal triangles and ragged batches leave no
// block idle. A unit that several blocks share is joined by the last of them, from the parts
// in the order of the blocks.
//
// Measured (GB300): a prompt of 8,191 tokens, 32 heads of 128 on 8, 431 us: 1,275 TFLOP/s, 66 % of
// the card's bf16 matrix rate in a burst, the tensor pipe 57 % busy. The chain of a tile of
// rows (product, scores read, maxima, exponentials, P written, product: 2,000 cycles and its
// 1,024 of products) is longer than the 2,048 cycles of products of both. The same inputs pass after pass
// take 414, over an FP8 cache 671, with capped scores 638: more instructions on that chain. Twelve sequences
// with 9 to 130 tokens over FP8 caches, capped, 233 us; packed documents with a bias 81 us, of which a unit
// of four tiles spends two thirds in its tiles. Registers that ptxas spills (up to 80 bytes a thread) are
// touched outside the tiles' loops: 0.05 % of the prompt's instructions, 0.02 % of the turn's.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "es_attention.cuh"
#include "es_rollout_internal.h"
#include "es_tensor.cuh"

namespace esopt {
namespace {

constexpr int kKeys = 128;   // of a tile
constexpr int kRows = 256;   // of a unit
constexpr int kStages = 2;
constexpr int kMaxGrid = 192;
// What a unit costs beside its tiles, in tiles: its queries, the first tile's way through the
// pipeline, its results. Plain bf16 tiles are the quickest, so more of them fit: a prompt of
// 8,191 tokens takes 505 us with 2, 430 with 3, 414 with 4, 424 with 6. Where tiles take longer it
// is 2: over an FP8 cache 772 us with 1, 673 with 2, 680 with 3; with capped scores 745, 638, 643.
template <bool kFp8, bool kPlain>
constexpr int unit_cost() { return kPlain && !kFp8 ? 4 : 2; }
// No block takes less than this of a unit that others share: a part costs its way through
// memory, about as much as two tiles. So a unit of fewer than six tiles stays whole, and where most are, blocks
// differ by a unit. With 1, 2, 3, 4: twelve turns over FP8 caches 190, 190, 193, 195 us, packed
// documents 79, 77, 79, 80, long prompts alike.
constexpr int kLeastShare = 3;
constexpr float kSlack = 8.0f;  // log 2 of how far a score may be above the kept maximum

// Where a block's range begins, from the planning kernel.
struct Start {
  int64_t pair_tile;  // first tile of (seq, row_tile) in the space of all
  int seq, row_tile;
};
struct Plan {
  int64_t all, per;
  int unit_cost;
  Start start[kMaxGrid];
};

// What the rows of (sequence, row tile) see: their tokens, and the union and the common part
// of their intervals of the cache. Rows that see nothing have no part in either: whatever a
// product leaves in them, they are written as zeros.
struct Pair {
  int begin, count, base, length;
  int rows;
  int lo, hi;
  int in_lo, in_hi;
  int tiles;  // one at least where there are rows, so that rows which see nothing are written too
};

__device__ __forceinline__ int row_tiles_of(const BatchView& b, const AttentionArgs& a, int seq) {
  int begin, count, base;
  new_tokens(b, seq, begin, count, base);
  return static_cast<int>((static_cast<int64_t>(count) * a.group + kRows - 1) / kRows);
}

// Called by whole warps, kLanes threads of which (1, 8 or 32) share a pair and are numbered
// `lane`.
template <int kLanes>
__device__ __forceinline__ Pair pair_of(const BatchView& b, const AttentionArgs& a, int seq, int row_tile, int lane) {
  Pair p;
  p.length = sequence_length(b, seq);
  new_tokens(b, seq, p.begin, p.count, p.base);
  const int64_t row0 = static_cast<int64_t>(row_tile) * kRows;
  p.rows = static_cast<int>(min(static_cast<int64_t>(p.count) * a.group - row0, static_cast<int64_t>(kRows)));
  const int i0 = static_cast<int>(row0 / a.group), i1 = static_cast<int>((row0 + p.rows - 1) / a.group);
  int lo = INT32_MAX, hi = 0, in_lo = 0, in_hi = INT32_MAX;
  if (a.first == nullptr && a.last == nullptr) {
    // intervals move with the position
    const Row r0 = row_of(b, a, p.begin, p.count, p.base, p.length, i0 * a.group);
    const Row r1 = row_of(b, a, p.begin, p.count, p.base, p.length, i1 * a.group);
    if (r1.hi > r1.lo) {
      lo = r0.hi > r0.lo ? r0.lo : 0;
      hi = r1.hi;
    }
    in_lo = r1.lo;
    in_hi = r0.hi;
  } else {
#pragma unroll 4
    for (int i = i0 + lane; i <= i1; i += kLanes) {
      const Row r = row_of(b, a, p.begin, p.count, p.base, p.length, i * a.group);
      if (r.hi > r.lo) {
        lo = min(lo, r.lo);
        hi = max(hi, r.hi);
        in_lo = max(in_lo, r.lo);
        in_hi = min(in_hi, r.hi);
      }
    }
#pragma unroll
    for (int m = kLanes / 2; m > 0; m >>= 1) {
      lo = min(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, m));
      hi = max(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, m));
      in_lo = max(in_lo, __shfl_xor_sync(0xFFFFFFFFu, in_lo, m));
      in_hi = min(in_hi, __shfl_xor_sync(0xFFFFFFFFu, in_hi, m));
    }
  }
  if (hi <= lo) lo = hi = 0;
  p.lo = lo;
  p.hi = hi;
  p.in_lo = in_lo;
  p.in_hi = in_hi;
  p.tiles = max(1, (hi - (lo & ~(kKeys - 1)) + kKeys - 1) / kKeys);
  return p;
}

// Counts the tiles of all pairs and finds where each block's range begins. One block: pairs
// are a few thousand at most, and a pair's tiles cost a thread few operations, or with
// `first` or `last` its tokens' entries.
constexpr int kPlanThreads = 1024;

__device__ __forceinline__ int64_t scan_block(int64_t x, int64_t* shared, int64_t& total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int64_t upto = x;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    const int64_t y = __shfl_up_sync(0xFFFFFFFFu, upto, m);
    if (lane >= m) upto += y;
  }
  __syncthreads();
  if (lane == 31) shared[warp] = upto;
  __syncthreads();
  if (warp == 0) {
    int64_t y = shared[lane];
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const int64_t z = __shfl_up_sync(0xFFFFFFFFu, y, m);
      if (lane >= m) y += z;
    }
    shared[lane] = y;
  }
  __syncthreads();
  total = shared[31];
  return upto + (warp > 0 ? shared[warp - 1] : 0) - x;  // of the threads before
}

__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const BatchView batch, const AttentionArgs a, int kv_heads, int grid, int unit_cost, Plan* plan) {
  __shared__ int64_t sums[32];
  __shared__ int first_pair[ES_MAX_SEQUENCES];  // the pairs of a sequence begin here
  __shared__ int tiles[kPlanThreads];
  wait_for_previous();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int64_t pairs = 0;
  for (int s0 = 0; s0 < batch.sequences; s0 += kPlanThreads) {
    const int s = s0 + threadIdx.x;
    const int n = s < batch.sequences ? row_tiles_of(batch, a, s) : 0;
    int64_t more;
    const int64_t before = scan_block(n, sums, more);
    if (s < batch.sequences) first_pair[s] = static_cast<int>(pairs + before);
    pairs += more;
  }
  __syncthreads();
  auto sequence_of = [&](int64_t pair) {  // the last one that begins at or before it
    int lo = 0, hi = batch.sequences - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first_pair[mid] <= pair) lo = mid; else hi = mid - 1;
    }
    return lo;
  };
  int64_t all = 0, per = 1;
  for (int pass = 0; pass < 2; ++pass) {  // the number of tiles, then the blocks' ranges
    int64_t done = 0;
    for (int64_t p0 = 0; p0 < pairs; p0 += kPlanThreads) {
      const int64_t p = p0 + threadIdx.x;
      const int seq = p < pairs ? sequence_of(p) : 0;
      const int row_tile = p < pairs ? static_cast<int>(p - first_pair[seq]) : 0;
      int n = 0;
      if (a.first == nullptr && a.last == nullptr) {
        if (p < pairs) n = pair_of<1>(batch, a, seq, row_tile, 0).tiles;
      } else {
        if (pass == 0 || pairs > kPlanThreads) {
          __syncthreads();
          // eight threads for each pair: its tokens' entries are read side by side
          for (int i = warp * 4; i < kPlanThreads && p0 + i < pairs; i += kPlanThreads / 8) {
            const int mine = i + lane / 8;
            const int64_t at = min(p0 + mine, pairs - 1);
            const int s = sequence_of(at);
            const int of_pair = pair_of<8>(batch, a, s, static_cast<int>(at - first_pair[s]), lane % 8).tiles;
            if (lane % 8 == 0) tiles[mine] = of_pair;
          }
          __syncthreads();
        }
        if (p < pairs) n = tiles[threadIdx.x];
      }
      const int64_t mine = p < pairs ? static_cast<int64_t>(n + unit_cost) * kv_heads : 0;
      int64_t more;
      const int64_t at = done + scan_block(mine, sums, more);
      if (pass == 1)
        for (int64_t c = (at + per - 1) / per; c * per < at + mine; ++c) plan->start[c] = Start{at, seq, row_tile};
      done += more;
    }
    if (pass == 0) {
      all = done;
      per = max((all + grid - 1) / grid, static_cast<int64_t>(1));
      if (threadIdx.x == 0) {
        plan->all = all;
        plan->per = per;
        plan->unit_cost = unit_cost;
      }
    }
  }
}

// --- tensor memory ------------------------------------------------------------------

__device__ __forceinline__ void tensor_store16(uint32_t to, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(to),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// --- the walk over a block's units -----------------------------------------------------

// What the warps of a block need of a unit. One warp walks the units and puts them here, a few
// ahead; kept by every warp for itself they cost registers and a share of each unit's time.
struct Unit {
  int valid;
  int seq, head;
  int tile0, tile1;  // this block's tiles, of the unit's
  int key0;          // first key of tile 0
  int begin, count, base, length;  // of the sequence's new tokens
  int row0, rows;    // of the unit, among the sequence's
  int lo, hi, in_lo, in_hi;
  int c_first, c_last;  // the blocks that share it

  __device__ __forceinline__ int key_of(int tile) const { return key0 + tile * kKeys; }
  // Not every row that sees anything sees all of the tile.
  __device__ __forceinline__ bool edge(int tile) const { return key_of(tile) < in_lo || key_of(tile) + kKeys > in_hi; }
};
constexpr int kUnits = 4;

// 32 keys of a unit (bits of `keys`, from position key0) whose values hold an infinity or NaN that
// not every row sees. A unit's first kBad such pieces are listed; where it has more, all its tiles
// at the ends of intervals are looked through again.
struct Bad {
  int key0;
  uint32_t keys;
};
constexpr uint32_t kBad = 32;

// FP8: codes pass from the pages to the converting warps in pieces of 32 keys or values, four
// and four to a tile, each warp with a place of its own for them. (Four warps that shared each
// piece, a half tile, took 6,000 cycles a tile for 3,000 cycles of work.)
constexpr int kRaw = 6;    // converting warps
constexpr int kPiece = 32;  // keys
constexpr int kPieces = 2 * kKeys / kPiece;

template <int D, bool kFp8>
struct Shared {
  uint16_t q[2][128 * D];
  uint16_t k[kStages][kKeys * D];
  uint16_t v[kStages][kKeys * D];
  uint8_t raw[kFp8 ? kRaw : 1][kFp8 ? kPiece * D : 128];
  // Read with the scores, when the tile's keys may have made room for others: a slot is
  // written again four tiles on, which follows the scores of two tiles on.
  float k_scale[4][kKeys];  // times the scores' factor
  uint32_t absent[4];  // 16-key pieces of the tile whose page does not exist
  float v_scale[kStages][kKeys];
  uint64_t q_full[2], s_full[2], p_full[2], o_done[2];
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], v_fixed[kStages];
  uint64_t group[2], drained;
  uint64_t raw_full[kRaw], raw_empty[kRaw];
  uint64_t unit_full[kUnits], unit_empty[kUnits];
  Unit unit[kUnits];
  uint32_t tensor;           // address of the tensor memory
  int failed;
  CacheView cache;  // for add_bad
  BatchView batch;
  uint32_t bad_count[kUnits];  // of each unit here
  Bad bad[kUnits][kBad];
  int last[2];
};

// Parts of units that blocks share, as in the kernel of few rows: block c's first unit, if it
// began in an earlier block, is part 2c, and its last one, if it began here, part 2c + 1.
// A row belongs to a thread, so 16 bytes of all rows lie together.
template <int D>
struct Part {
  float4 o[D / 4][kRows];
  float top[kRows], sum[kRows];
};

// The four warps of a warpgroup; false as barrier_wait.
template <class Sh>
__device__ __forceinline__ bool group_sync(Sh& sh, const Watch& watch, int x, uint32_t& phase, int lane) {
  warp_arrive(&sh.group[x], lane);
  return warp_wait(&sh.group[x], phase++ & 1, watch);
}

// The units of a block's range, by one warp.
struct Walk {
  int64_t at, end, per, pair_tile;
  int seq, row_tile;
  int unit_cost;
  Pair pair;
  // the unit
  int head, tile0, tile1;
  int64_t unit0;  // of its first tile

  __device__ __forceinline__ Walk(const BatchView& b, const AttentionArgs& a, const Plan* plan, int lane) {
    per = plan->per;
    unit_cost = plan->unit_cost;
    at = blockIdx.x * per;
    end = min(at + per, plan->all);
    if (at < end) {
      const Start& s = plan->start[blockIdx.x];
      pair_tile = s.pair_tile;
      seq = s.seq;
      row_tile = s.row_tile;
      pair = pair_of<32>(b, a, seq, row_tile, lane);
    }
  }
  // The tile of the unit at which a block's range that ends at p does: p itself, or the unit's
  // begin or end where that is near.
  __device__ __forceinline__ int cut(int64_t p) const {
    const int n = pair.tiles;
    const int raw = static_cast<int>(min(max(p - unit0, static_cast<int64_t>(0)), static_cast<int64_t>(n)));
    if (n < 2 * kLeastShare) return 2 * raw < n ? 0 : n;
    return raw < kLeastShare ? 0 : n - raw < kLeastShare ? n : raw;
  }
  __device__ __forceinline__ bool next(const BatchView& b, const AttentionArgs& a, int kv_heads, int lane) {
    while (at < end) {
      while (at >= pair_tile + static_cast<int64_t>(pair.tiles + unit_cost) * kv_heads) {
        pair_tile += static_cast<int64_t>(pair.tiles + unit_cost) * kv_heads;
        ++row_tile;
        while (row_tile >= row_tiles_of(b, a, seq)) {
          ++seq;
          row_tile = 0;
        }
        pair = pair_of<32>(b, a, seq, row_tile, lane);
      }
      const int length = pair.tiles + unit_cost;
      head = static_cast<int>((at - pair_tile) / length);
      const int64_t begin = pair_tile + static_cast<int64_t>(head) * length;
      unit0 = begin + unit_cost;
      tile0 = at <= begin ? 0 : cut(at);
      tile1 = end >= begin + length ? pair.tiles : cut(end);
      at = begin + length;
      if (tile1 > tile0) return true;
    }
    return false;
  }
  // The blocks that have the unit's first tile and its last.
  __device__ __forceinline__ void sharers(int& c_first, int& c_last) const {
    c_first = static_cast<int>((unit0 - unit_cost) / per);
    c_last = static_cast<int>((unit0 + pair.tiles - 1) / per);
    while (c_first < c_last && cut((c_first + 1) * per) == 0) ++c_first;
    while (c_last > c_first && cut(c_last * per) == pair.tiles) --c_last;
  }
};

// The walking warp's side: the next unit into its place; false where there is none (which is
// told as well) or a wait was given up.
template <class Sh>
__device__ __forceinline__ bool tell(Sh& sh, const Watch& watch, Walk& walk, const BatchView& b, const AttentionArgs& a, int kv_heads, uint32_t n, int lane) {
  const bool more = walk.next(b, a, kv_heads, lane);
  if (!warp_wait(&sh.unit_empty[n % kUnits], (n / kUnits & 1) ^ 1, watch)) return false;
  if (lane == 0) {
    Unit& u = sh.unit[n % kUnits];
    u.valid = more;
    sh.bad_count[n % kUnits] = 0;
    if (more) {
      const Pair& p = walk.pair;
      u.seq = walk.seq;
      u.head = walk.head;
      u.tile0 = walk.tile0;
      u.tile1 = walk.tile1;
      u.key0 = p.lo & ~(kKeys - 1);
      u.begin = p.begin;
      u.count = p.count;
      u.base = p.base;
      u.length = p.length;
      u.row0 = walk.row_tile * kRows;
      u.rows = p.rows;
      u.lo = p.lo;
      u.hi = p.hi;
      u.in_lo = p.in_lo;
      u.in_hi = p.in_hi;
      int c_first, c_last;
      walk.sharers(c_first, c_last);
      u.c_first = c_first;
      u.c_last = c_last;
    }
  }
  warp_arrive(&sh.unit_full[n % kUnits], lane);
  return more;
}
// The other warps': waits for unit n; false where there is none.
template <class Sh>
__device__ __forceinline__ bool take(Sh& sh, const Watch& watch, uint32_t n) {
  return warp_wait(&sh.unit_full[n % kUnits], n / kUnits & 1, watch) && sh.unit[n % kUnits].valid;
}
// This warp is done with it.
template <class Sh>
__device__ __forceinline__ void leave(Sh& sh, uint32_t n, int lane) {
  warp_arrive(&sh.unit_empty[n % kUnits], lane);
}

// By a whole warp: unit n's keys key0 + the bits of its lanes are noted.
template <class Sh>
__device__ __forceinline__ void note_bad(Sh& sh, uint32_t n, int key0, uint32_t bits, int lane) {
  const uint32_t keys = __reduce_or_sync(0xFFFFFFFFu, bits);
  if (keys != 0 && lane == 0) {
    const uint32_t at = atomicAdd(&sh.bad_count[n % kUnits], 1u);
    if (at < kBad) sh.bad[n % kUnits][at] = Bad{key0, keys};
  }
}

// Offset in elements of 16-byte piece `piece` of row r, in an operand of 128 rows.
template <int D>
__device__ __forceinline__ int place_of(int r, int piece) {
  return piece / 8 * (128 * 64) + r * 64 + ((piece % 8) ^ (r % 8)) * 8;
}

// --- roles -----------------------------------------------------------------------------

// bf16 pages to shared memory, a lane for each page of the tile.
template <int D>
__device__ void copy_tiles(Shared<D, false>& sh, const Watch& watch, const CacheView& cache, const BatchView& batch, const AttentionArgs& a,
                           const Plan* plan, const CUtensorMap* k_map, const CUtensorMap* v_map, int lane) {
  const int page_size = 1 << cache.page_shift, pages = kKeys >> cache.page_shift;
  uint32_t k_done = 0, v_done = 0;
  bool fine = true;
  Walk walk(batch, a, plan, lane);
  for (uint32_t n = 0; fine && tell(sh, watch, walk, batch, a, cache.kv_heads, n, lane); ++n) {
    const int key0 = walk.pair.lo & ~(kKeys - 1);
    for (int tile = walk.tile0; tile < walk.tile1; ++tile) {
      const int stage = k_done % kStages;
      const uint32_t parity = k_done / kStages & 1;
      const int j = key0 + tile * kKeys + lane * page_size;
      int page = -1;
      if (lane < pages && j < walk.pair.hi) page = page_of(cache, batch, walk.seq, j);
      const uint32_t missing = __ballot_sync(0xFFFFFFFFu, page < 0);
      uint32_t absent = 0;  // in pieces of 16 keys
      for (int i = 0; i < 8; ++i) absent |= (missing >> (i * 16 >> cache.page_shift) & 1) << i;
      // a page past the last one reads as zeros
      const int z = page < 0 ? cache.num_pages : page, y = walk.head << cache.page_shift;
      fine = warp_wait(&sh.k_empty[stage], parity ^ 1, watch);
      if (!fine) break;
      if (lane == 0) {
        sh.absent[k_done % 4] = absent;
        barrier_expect(&sh.k_full[stage], kKeys * D * 2);
      }
      __syncwarp();
      if (lane < pages)
        for (int h = 0; h < D / 64; ++h)
          load_box(k_map, shared_address(sh.k[stage] + h * 128 * 64 + lane * page_size * 64), &sh.k_full[stage], h * 64, y, z);
      ++k_done;
      fine = warp_wait(&sh.v_empty[stage], parity ^ 1, watch);
      if (!fine) break;
      if (lane == 0) barrier_expect(&sh.v_full[stage], kKeys * D * 2);
      __syncwarp();
      if (lane < pages)
        for (int h = 0; h < D / 64; ++h)
          load_box(v_map, shared_address(sh.v[stage] + h * 128 * 64 + lane * page_size * 64), &sh.v_full[stage], h * 64, y, z);
      ++v_done;
    }
  }
  // no copy outlives the block
  for (uint32_t i = k_done > kStages ? k_done - kStages : 0; i < k_done; ++i) barrier_settle(&sh.k_full[i % kStages], i / kStages & 1);
  for (uint32_t i = v_done > kStages ? v_done - kStages : 0; i < v_done; ++i) barrier_settle(&sh.v_full[i % kStages], i / kStages & 1);
}

// bf16 values of tiles at the ends of intervals: those that no row sees become zeros, and
// infinities and NaN too (a product with p = 0 would carry them into rows that do not see them), and
// their keys are noted: the rows that see them get them when the unit is written. Every tile passes here,
// so that the barriers of the stages are never a round ahead.
template <int D>
__device__ void fix_tiles(Shared<D, false>& sh, const Watch& watch, int thread, int lane) {
  uint32_t done = 0;
  for (uint32_t n = 0; take(sh, watch, n); ++n) {
    const Unit& unit = sh.unit[n % kUnits];
    const int tile1 = unit.tile1;
    for (int tile = unit.tile0; tile < tile1; ++tile, ++done) {
      const int stage = done % kStages, j0 = unit.key_of(tile);
      if (!warp_wait(&sh.v_full[stage], done / kStages & 1, watch)) return;
      if (unit.edge(tile)) {
        const int lo = unit.lo, hi = unit.hi;
#pragma unroll 1
        for (int key0 = 0; key0 < kKeys; key0 += 32) {
          constexpr int kSteps = D / 16;  // of 64 pieces, to 32 keys
          auto key_at = [&](int step) { return key0 + (step * 64 + thread) / (D / 8); };
          auto piece_at = [&](int step) { return reinterpret_cast<uint4*>(sh.v[stage] + place_of<D>(key_at(step), thread % (D / 8))); };
          uint4 w[kSteps];
#pragma unroll
          for (int i = 0; i < kSteps; ++i) w[i] = *piece_at(i);
          bool spoiled = false;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            const int j = j0 + key_at(i);
            if (j < lo || j >= hi) *piece_at(i) = make_uint4(0, 0, 0, 0);
            else spoiled = spoiled || has_nonfinite(w[i].x) || has_nonfinite(w[i].y) || has_nonfinite(w[i].z) || has_nonfinite(w[i].w);
          }
          if (!__any_sync(0xFFFFFFFFu, spoiled)) continue;
          uint32_t bad = 0;
#pragma unroll 1
          for (int i = 0; i < kSteps; ++i) {
            uint32_t* u = reinterpret_cast<uint32_t*>(piece_at(i));  // zeros outside [lo, hi) by now
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
              uint32_t x = u[e];
              if (!has_nonfinite(x)) continue;
              if ((x & 0x7F80u) == 0x7F80u) x &= 0xFFFF0000u;
              if ((x & 0x7F800000u) == 0x7F800000u) x &= 0xFFFFu;
              u[e] = x;
              bad |= 1u << (key_at(i) % 32);
            }
          }
          __syncwarp();
          note_bad(sh, n, j0 + key0, bad, lane);
        }
        fence_async();
      }
      warp_arrive(&sh.v_fixed[stage], lane);
    }
    leave(sh, n, lane);
  }
}

// FP8 pages to shared memory as they are: a tile's pieces of keys, then of values, each to the
// next converting warp.
template <int D>
__device__ void copy_codes(Shared<D, true>& sh, const Watch& watch, const CacheView& cache, const BatchView& batch, const AttentionArgs& a,
                           const Plan* plan, const CUtensorMap* k_map, const CUtensorMap* v_map, int lane) {
  const int box = min(1 << cache.page_shift, kPiece), boxes = kPiece / box;  // keys of a copy, copies of a piece
  uint32_t done = 0, tiles = 0;
  bool fine = true;
  Walk walk(batch, a, plan, lane);
  for (uint32_t n = 0; fine && tell(sh, watch, walk, batch, a, cache.kv_heads, n, lane); ++n) {
    const int key0 = walk.pair.lo & ~(kKeys - 1);
    for (int tile = walk.tile0; fine && tile < walk.tile1; ++tile, ++tiles) {
      // lane i's keys are 16 i and up
      const int j = key0 + tile * kKeys + lane * 16;
      const int page = lane < 8 && j < walk.pair.hi ? page_of(cache, batch, walk.seq, j) : -1;
      const uint32_t absent = __ballot_sync(0xFFFFFFFFu, page < 0) & 0xFFu;
#pragma unroll 1
      for (int part = 0; part < kPieces; ++part, ++done) {
        const int slot = done % kRaw, in_tile = part % (kPieces / 2) * kPiece;
        const int mine = __shfl_sync(0xFFFFFFFFu, page, (in_tile + lane * box) / 16 % 8);
        fine = warp_wait(&sh.raw_empty[slot], (done / kRaw & 1) ^ 1, watch);
        if (!fine) break;
        if (lane == 0) {
          if (part == 0) sh.absent[tiles % 4] = absent;
          barrier_expect(&sh.raw_full[slot], kPiece * D);
        }
        __syncwarp();
        if (lane < boxes)
          load_box(part < kPieces / 2 ? k_map : v_map, shared_address(sh.raw[slot] + lane * box * D), &sh.raw_full[slot], 0,
                   (walk.head << cache.page_shift) + ((in_tile + lane * box) & ((1 << cache.page_shift) - 1)),
                   mine < 0 ? cache.num_pages : mine);
      }
    }
  }
  // no copy outlives the block
  for (uint32_t i = done > kRaw ? done - kRaw : 0; i < done; ++i) barrier_settle(&sh.raw_full[i % kRaw], i / kRaw & 1);
}

// One warp's piece of codes to bf16, 8 codes (16 bytes of bf16) to a lane and step, so that the
// eight lanes that write side by side write all of one 128-byte row; eight steps' codes are
// read before any is converted.
// clean: keys outside [lo, hi) become zeros, and NaN codes too; returns the piece's keys of this
// lane that had any.
template <int D>
__device__ __forceinline__ uint32_t convert_piece(const uint8_t* raw, uint16_t* to, int key0, int lane, bool clean, int lo, int hi) {
  constexpr int kSteps = kPiece * D / 8 / 32;
  uint32_t bad_keys = 0;
#pragma unroll 1
  for (int s0 = 0; s0 < kSteps; s0 += 8) {
    uint32_t u[8][2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint2 w = *reinterpret_cast<const uint2*>(raw + ((s0 + i) * 32 + lane) * 8);
      u[i][0] = w.x;
      u[i][1] = w.y;
    }
    if (clean) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = key0 + ((s0 + i) * 32 + lane) / (D / 8);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (key < lo || key >= hi) u[i][e] = 0;
          const uint32_t bad = ((u[i][e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;  // NaN codes
          if (bad != 0) {
            u[i][e] &= ~((bad >> 7) * 0xFFu);
            bad_keys |= 1u << (key - key0);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int piece = (s0 + i) * 32 + lane;
      *reinterpret_cast<uint4*>(to + place_of<D>(key0 + piece / (D / 8), piece % (D / 8))) =
          make_uint4(bf16_of_e4m3(u[i][0]), bf16_of_e4m3(u[i][0] >> 16), bf16_of_e4m3(u[i][1]), bf16_of_e4m3(u[i][1] >> 16));
    }
  }
  return bad_keys;
}

template <int D>
__device__ void convert_tiles(Shared<D, true>& sh, const Watch& watch, const CacheView& cache, const BatchView& batch, const AttentionArgs& a, int warp,
                              int lane) {
  uint32_t done = 0;  // tiles
  uint32_t turns = 0;  // this warp's pieces
  for (uint32_t n = 0; take(sh, watch, n); ++n) {
    const Unit& unit = sh.unit[n % kUnits];
    const int tile1 = unit.tile1;
    for (int tile = unit.tile0; tile < tile1; ++tile, ++done) {
      const int stage = done % kStages, j0 = unit.key_of(tile);
      const uint32_t parity = done / kStages & 1;
      // pieces go round: this warp's first one of the tile, and perhaps another
#pragma unroll 1
      for (uint32_t part = (warp + kRaw - done * kPieces % kRaw) % kRaw; part < kPieces; part += kRaw, ++turns) {
        const bool of_keys = part < kPieces / 2;
        const int key0 = part % (kPieces / 2) * kPiece, j = j0 + key0 + lane;
        // the scale of this lane's key, while the codes are on their way
        const int page = j < unit.hi ? page_of(cache, batch, unit.seq, j) : -1;
        float scale = 0.0f;
        if (page >= 0)
          scale = __ldg((of_keys ? cache.k_scale : cache.v_scale) + page * cache.scale_stride +
                        (static_cast<uint64_t>(unit.head) << cache.page_shift) + (j & ((1 << cache.page_shift) - 1)));
        const bool clean = !of_keys && unit.edge(tile);
        uint32_t bad = 0;
        if (clean) {  // as with NaN codes: only rows that see the key get to know its scale
          if (j < unit.lo || j >= unit.hi) {
            scale = 0.0f;
          } else if (!(fabsf(scale) <= FLT_MAX)) {
            scale = 0.0f;
            bad = 1u << lane;
          }
        }
        if (!warp_wait(of_keys ? &sh.k_empty[stage] : &sh.v_empty[stage], parity ^ 1, watch)) return;
        if (of_keys) sh.k_scale[done % 4][key0 + lane] = scale * a.factor;
        else sh.v_scale[stage][key0 + lane] = scale;
        if (!warp_wait(&sh.raw_full[warp], turns & 1, watch)) return;
        bad |= convert_piece<D>(sh.raw[warp], of_keys ? sh.k[stage] : sh.v[stage], key0, lane, clean, unit.lo - j0, unit.hi - j0);
        if (clean) note_bad(sh, n, j0 + key0, bad, lane);
        // The next codes may come now that these have been used. (After their loads alone have
        // been issued is too early: a copy of zeros can overtake them.)
        warp_arrive(&sh.raw_empty[warp], lane);
        fence_async();
        warp_arrive(of_keys ? &sh.k_full[stage] : &sh.v_full[stage], lane);
      }
    }
    leave(sh, n, lane);
  }
}

// The warp that issues the products.
template <int D, bool kFp8>
__device__ void issue_products(Shared<D, kFp8>& sh, const Watch& watch, int lane) {
  constexpr uint32_t kScores = product_of(kKeys, false), kValues = product_of(D, true);
  const uint32_t tensor = sh.tensor;
  uint32_t k_done = 0, v_done = 0, units = 0, two_units = 0;
  uint32_t p_done = 0, p_done_two = 0;  // of the first tile of rows, and of the second
  // The operands' descriptors: only the address in their low word changes.
  const uint64_t plain_rows = operand(0, 16), value_rows = operand(0, 128 * 128);
  const uint32_t q_at = shared_address(sh.q[0]) >> 4;
  const uint32_t k_at = shared_address(sh.k[0]) >> 4, v_at = shared_address(sh.v[0]) >> 4;
  constexpr uint32_t kOperand = 128 * D * 2 / 16;
  auto scores = [&](uint32_t x, uint32_t stage) {
    const uint64_t q = plain_rows + (q_at + x * kOperand), k = plain_rows + (k_at + stage * kOperand);
    if (elected()) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const uint32_t at = (i / 4 * (128 * 128) + i % 4 * 32) / 16;
        multiply(tensor + x * 128, q + at, k + at, kScores, i > 0);
      }
      commit(&sh.s_full[x]);
      barrier_arrive(&sh.s_full[x]);  // with what this thread has seen: the tile's scales, its absent pages
    }
    __syncwarp();
  };
  auto wait = [&](uint64_t* b, uint32_t parity) { return warp_wait(b, parity, watch); };
  for (uint32_t n = 0; take(sh, watch, n); ++n) {
    const uint32_t count = sh.unit[n % kUnits].rows > 128 ? 2 : 1;
    const int tiles = sh.unit[n % kUnits].tile1 - sh.unit[n % kUnits].tile0;
    leave(sh, n, lane);
    if (!wait(&sh.q_full[0], units & 1)) return;
    if (count == 2 && !wait(&sh.q_full[1], two_units & 1)) return;
    if (!wait(&sh.k_full[k_done % kStages], k_done / kStages & 1)) return;
    fence_after();
    for (uint32_t x = 0; x < count; ++x) scores(x, k_done % kStages);
    if (elected()) commit(&sh.k_empty[k_done % kStages]);
    __syncwarp();
    ++k_done;
    for (int tile = 0; tile < tiles; ++tile, ++v_done) {
      const uint32_t stage = v_done % kStages;
      const bool more = tile + 1 < tiles;
      if (!wait(kFp8 ? &sh.v_full[stage] : &sh.v_fixed[stage], v_done / kStages & 1)) return;
      if (more && !wait(&sh.k_full[k_done % kStages], k_done / kStages & 1)) return;
      for (uint32_t x = 0; x < count; ++x) {
        if (!wait(&sh.p_full[x], (x == 0 ? p_done : p_done_two) & 1)) return;
        fence_after();
        const uint64_t v = value_rows + (v_at + stage * kOperand);
        if (elected()) {
#pragma unroll
          for (int i = 0; i < kKeys / 16; ++i)
            multiply_from_tensor(tensor + 256 + x * 128, tensor + x * 128 + i * 8, v + i * 128, kValues, i > 0 || tile > 0);
          commit(&sh.o_done[x]);
        }
        __syncwarp();
        if (more) scores(x, k_done % kStages);
      }
      if (elected()) {
        commit(&sh.v_empty[stage]);
        if (more) commit(&sh.k_empty[k_done % kStages]);
      }
      __syncwarp();
      if (more) ++k_done;
      ++p_done;
      p_done_two += count == 2;
    }
    ++units;
    two_units += count == 2;
  }
}

__device__ __forceinline__ uint64_t pack(float lo, float hi) {
  uint64_t y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(lo), "f"(hi));
  return y;
}
__device__ __forceinline__ void unpack(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t y;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}

__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Bits n and up of 32; all for n <= 0, none for n >= 32.
__device__ __forceinline__ uint32_t bits_from(int n) { return n >= 32 ? 0u : 0xFFFFFFFFu << max(n, 0); }

// 16 bytes to shared memory without a register in between; zeros where `from` is not to be read.
__device__ __forceinline__ void copy_async(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// This thread's row of a unit, and its query on the way to shared memory.
template <int D, bool kFp8>
__device__ __forceinline__ Row take_row(Shared<D, kFp8>& sh, const BatchView& batch, const AttentionArgs& a, const Unit& unit, int x,
                                        int thread, int& h) {
  const int r = unit.row0 + x * 128 + thread;
  const Row row = row_of(batch, a, unit.begin, unit.count, unit.base, unit.length, r);
  h = unit.head * a.group + r % a.group;
  const uint16_t* from = a.q + static_cast<uint64_t>(max(row.token, 0)) * a.q_stride + static_cast<uint64_t>(h) * D;
#pragma unroll
  for (int i = 0; i < D / 8; ++i) copy_async(shared_address(sh.q[x] + place_of<D>(thread, i)), from + i * 8, row.token >= 0);
  asm volatile("cp.async.commit_group;" ::: "memory");
  return row;
}
template <class Sh>
__device__ __forceinline__ void hand_over(Sh& sh, int x, int lane) {
  asm volatile("cp.async.wait_all;" ::: "memory");
  fence_async();
  warp_arrive(&sh.q_full[x], lane);
}

// Adds the infinities and NaN that unit n's noted keys hold in their values to a row that sees
// [lo, hi): to its results in bf16, or where `part` is given to its part of a shared unit (16 bytes of all
// rows together). 32 elements at a time over all keys, until they are all NaN. Out of line, and with all it
// needs in shared memory: in line it costs FP8 tiles 3 to 6 %.
template <int D, bool kFp8>
__device__ __noinline__ void add_bad(const Shared<D, kFp8>& sh, uint32_t n, int lo, int hi, uint16_t* out, float* part) {
  const CacheView& cache = sh.cache;
  const Unit& unit = sh.unit[n % kUnits];
  const uint32_t bad = sh.bad_count[n % kUnits];
  const bool listed = bad <= kBad;
  const int pieces = listed ? static_cast<int>(bad) : (unit.tile1 - unit.tile0) * (kKeys / 32);
#pragma unroll 1
  for (int c = 0; c < D; c += 32) {
    float sum[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) sum[e] = 0.0f;
    bool more = true;
#pragma unroll 1
    for (int i = 0; more && i < pieces; ++i) {
      Bad piece;
      if (listed) {
        piece = sh.bad[n % kUnits][i];
      } else {
        const int tile = unit.tile0 + i / (kKeys / 32);
        if (!unit.edge(tile)) continue;
        piece = Bad{unit.key_of(tile) + i % (kKeys / 32) * 32, 0xFFFFFFFFu};
      }
      uint32_t keys = piece.keys & bits_from(lo - piece.key0) & ~bits_from(hi - piece.key0);
#pragma unroll 1
      for (; more && keys != 0; keys &= keys - 1) {
        const int j = piece.key0 + __ffs(static_cast<int>(keys)) - 1;
        const int page = page_of(cache, sh.batch, unit.seq, j);
        if (page < 0) continue;
        const uint64_t in_page = (static_cast<uint64_t>(unit.head) << cache.page_shift) + (j & ((1 << cache.page_shift) - 1));
        const uint64_t at = page * cache.page_stride + in_page * D + c;
        const float scale = kFp8 ? cache.v_scale[page * cache.scale_stride + in_page] : 1.0f;
        constexpr int kLoads = kFp8 ? 2 : 4;  // of 16 bytes
        uint4 raw[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
          raw[l] = reinterpret_cast<const uint4*>(static_cast<const char*>(cache.v) + at * (kFp8 ? 1 : 2))[l];
        more = false;
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const uint4& x = raw[e / (32 / kLoads)];
          const int word = e % (32 / kLoads) / (kFp8 ? 4 : 2);
          uint32_t y = word == 0 ? x.x : word == 1 ? x.y : word == 2 ? x.z : x.w;
          if (kFp8) y = bf16_of_e4m3(e % 4 == 0 ? y : y >> 16);
          const float v0 = __uint_as_float(y << 16) * scale, v1 = __uint_as_float(y & 0xFFFF0000u) * scale;
          if (!(fabsf(v0) <= FLT_MAX)) sum[e] += v0;
          if (!(fabsf(v1) <= FLT_MAX)) sum[e + 1] += v1;
          more = more || sum[e] == sum[e] || sum[e + 1] == sum[e + 1];
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      if (fabsf(sum[e]) <= FLT_MAX) continue;
      const int at = c + e;
      if (part != nullptr) part[at / 4 * (4 * kRows) + at % 4] += sum[e];
      else out[at] = static_cast<uint16_t>(pack_bf16(__uint_as_float(static_cast<uint32_t>(out[at]) << 16) + sum[e], 0.0f));
    }
  }
}

// 32 columns of scores in tensor memory, capped, each by its own size. By whole warps, where a chunk
// has a score beyond a quarter of the cap; out of line, since in line it costs the others their place in
// the instruction cache.
template <bool kFp8>
__device__ __noinline__ void cap_chunk(uint32_t at, float cap, float factor, const float* k_scale) {
  const float c1 = -1.0f / 3.0f * cap, c2 = 2.0f / 15.0f * cap, c3 = -17.0f / 315.0f * cap;
  uint32_t w[32];
  tensor_load(w, at);
  tensor_loaded(w);
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const uint64_t u = mul2(pack(__uint_as_float(w[i]), __uint_as_float(w[i + 1])),
                            kFp8 ? *reinterpret_cast<const uint64_t*>(k_scale + i) : pack(factor, factor));
    const uint64_t z = mul2(u, u);
    float lo, hi, lo_small, hi_small;
    unpack(u, lo, hi);
    unpack(mul2(u, fma2(z, fma2(z, fma2(z, pack(c3, c3), pack(c2, c2)), pack(c1, c1)), pack(cap, cap))), lo_small, hi_small);
    constexpr float twice = 2.0f * kLog2e;
    w[i] = __float_as_uint(fabsf(lo) <= 0.25f ? lo_small : fmaf(-2.0f * cap, reciprocal(exp2_approx(lo * twice) + 1.0f), cap));
    w[i + 1] = __float_as_uint(fabsf(hi) <= 0.25f ? hi_small : fmaf(-2.0f * cap, reciprocal(exp2_approx(hi * twice) + 1.0f), cap));
  }
  tensor_store32(at, w);
  tensor_stored();
}

// A warpgroup's rows: a thread for each.
template <int D, bool kFp8, bool kPlain>
__device__ void soften(Shared<D, kFp8>& sh, const Watch& watch, const CacheView& cache, const BatchView& batch, const AttentionArgs& a,
                       uint32_t* counters, Part<D>* parts, int x, int thread, int lane) {
  const uint32_t lanes = static_cast<uint32_t>(thread / 32 * 32) << 16;
  const uint32_t s_at = sh.tensor + lanes + x * 128, o_at = sh.tensor + lanes + 256 + x * 128;
  // Scores in units of log 2. Capped, with u = x / cap: cap tanh(u) is cap u (1 - z / 3 + 2 z^2 / 15 -
  // 17 z^3 / 315), z = u^2, where |u| <= 1 / 4 (the series' next term is 62 z^4 / 2835: off by 3.4e-7 of it
  // at most), else cap (1 - 2 / (2^(2 u log2(e)) + 1)), off by 1e-7 cap. By each score's own size,
  // so that what a row does not see has no part in its last bits.
  const bool capped = a.softcap > 0.0f, biased = a.slopes != nullptr;
  const float cap = a.softcap * kLog2e;
  uint32_t s_done = 0;        // tiles of this warpgroup so far
  uint32_t tiles_before = 0;  // of all units
  uint32_t phase = 0;
  // Unit n is this warpgroup's next one with rows; the tiles of those without are counted.
  uint32_t n = 0;
  auto find = [&](uint32_t& skipped) {
    skipped = 0;
    for (;; ++n) {
      if (!take(sh, watch, n)) return false;
      const Unit& u = sh.unit[n % kUnits];
      if (u.rows > x * 128) return true;
      skipped += u.tile1 - u.tile0;
      leave(sh, n, lane);
    }
  };
  uint32_t skipped;
  bool more = find(skipped);
  Row row_next{};
  int h_next = 0;
  if (more) {
    row_next = take_row<D, kFp8>(sh, batch, a, sh.unit[n % kUnits], x, thread, h_next);
    hand_over(sh, x, lane);
  }
  while (more) {
    bool fetched = false, ended = false;
    const uint32_t mine = n;
    const Unit& unit = sh.unit[mine % kUnits];
    const Row row = row_next;
    const int h = h_next;
    tiles_before += skipped;
    const int tile0 = unit.tile0, tile1 = unit.tile1, key0 = unit.key0;
    const float slope = !kPlain && a.slopes != nullptr ? a.slopes[h] * kLog2e : 0.0f;
    float top = -INFINITY, sum = 0.0f;
    for (int tile = tile0; tile < tile1; ++tile, ++s_done) {
      const uint32_t all_done = tiles_before + (tile - tile0);
      const int stage = all_done % kStages;
      const int j0 = key0 + tile * kKeys;
      if (!warp_wait(&sh.s_full[x], s_done & 1, watch)) return;
      fence_after();
      if (kFp8 && !warp_wait(&sh.v_full[stage], all_done / kStages & 1, watch)) return;
      const uint32_t absent = sh.absent[all_done % 4];
      const bool whole = __all_sync(0xFFFFFFFFu, row.token < 0 || (row.lo <= j0 && row.hi >= j0 + kKeys)) && absent == 0;
      const bool direct = kPlain && whole;
      float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (!direct) {
        // scores that take more than a factor are made here and put back
        const int c_lo = row.lo - j0, c_hi = row.hi - j0;  // the columns that the row sees
        float away = static_cast<float>(row.pos - j0);
#pragma unroll 1
        for (int c = 0; c < kKeys; c += 32) {
          uint32_t w[32];
          tensor_load(w, s_at + c);
          tensor_loaded(w);
          uint64_t y[16];  // pairs of scores
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            ulonglong2 f = make_ulonglong2(pack(a.factor, a.factor), pack(a.factor, a.factor));
            if (kFp8) f = *reinterpret_cast<const ulonglong2*>(&sh.k_scale[all_done % 4][c + 2 * i]);
            y[i] = mul2(pack(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])), f.x);
            y[i + 1] = mul2(pack(__uint_as_float(w[2 * i + 2]), __uint_as_float(w[2 * i + 3])), f.y);
          }
          if (!kPlain && capped) {
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float lo, hi;
              unpack(y[i], lo, hi);
              most = fmaxf(most, fmaxf(fabsf(lo), fabsf(hi)));
            }
            if (__all_sync(0xFFFFFFFFu, most <= 0.25f)) {
              const float c1 = -1.0f / 3.0f * cap, c2 = 2.0f / 15.0f * cap, c3 = -17.0f / 315.0f * cap;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const uint64_t z = mul2(y[i], y[i]);
                const uint64_t t = fma2(z, fma2(z, fma2(z, pack(c3, c3), pack(c2, c2)), pack(c1, c1)), pack(cap, cap));
                y[i] = mul2(y[i], t);
              }
            } else {
              cap_chunk<kFp8>(s_at + c, cap, a.factor, &sh.k_scale[all_done % 4][c]);
              tensor_load(w, s_at + c);
              tensor_loaded(w);
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = pack(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            }
          }
          if (!kPlain && biased) {
            if (__all_sync(0xFFFFFFFFu, away >= 31.0f)) {  // the chunk is not past the row's position
              const float base = -slope * away;
#pragma unroll
              for (int i = 0; i < 16; ++i)
                y[i] = add2(y[i], fma2(pack(slope, slope), pack(2.0f * i, 2.0f * i + 1.0f), pack(base, base)));
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float lo, hi;
                unpack(y[i], lo, hi);
                y[i] = pack(fmaf(-slope, fabsf(away - 2.0f * i), lo), fmaf(-slope, fabsf(away - (2.0f * i + 1.0f)), hi));
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float lo, hi;
            unpack(y[i], lo, hi);
            w[2 * i] = __float_as_uint(lo);
            w[2 * i + 1] = __float_as_uint(hi);
          }
          away -= 32.0f;
          if (!whole) {
            // columns of this chunk as bits
            uint32_t seen = bits_from(c_lo - c) & ~bits_from(c_hi - c);
            if (absent >> (c / 16) & 1) seen &= 0xFFFF0000u;
            if (absent >> (c / 16 + 1) & 1) seen &= 0xFFFFu;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(seen >> i & 1)) w[i] = __float_as_uint(-INFINITY);
          }
#pragma unroll
          for (int i = 0; i < 32; i += 2)
            tops[i / 2 % 4] = fmaxf(tops[i / 2 % 4], fmaxf(__uint_as_float(w[i]), __uint_as_float(w[i + 1])));
          tensor_store32(s_at + c, w);
        }
        tensor_stored();
      }
      uint32_t w[kKeys / 32][32];
#pragma unroll
      for (int c = 0; c < kKeys / 32; ++c) tensor_load(w[c], s_at + c * 32);
#pragma unroll
      for (int c = 0; c < kKeys / 32; ++c) tensor_loaded(w[c]);
      const float unit = direct && !kFp8 ? a.factor : 1.0f;  // of what w holds, in scores
      if (kFp8 && direct) {
#pragma unroll
        for (int c = 0; c < kKeys / 32; ++c)
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(&sh.k_scale[all_done % 4][c * 32 + i]);
            float y[4];
            unpack(mul2(pack(__uint_as_float(w[c][i]), __uint_as_float(w[c][i + 1])), k.x), y[0], y[1]);
            unpack(mul2(pack(__uint_as_float(w[c][i + 2]), __uint_as_float(w[c][i + 3])), k.y), y[2], y[3]);
            tops[i / 4 % 2] = fmaxf(tops[i / 4 % 2], fmaxf(y[0], y[1]));
            tops[2 + i / 4 % 2] = fmaxf(tops[2 + i / 4 % 2], fmaxf(y[2], y[3]));
#pragma unroll
            for (int e = 0; e < 4; ++e) w[c][i + e] = __float_as_uint(y[e]);
          }
      } else if (direct) {
#pragma unroll
        for (int i = 0; i < 32; i += 2)
#pragma unroll
          for (int c = 0; c < kKeys / 32; ++c) tops[c] = fmaxf(tops[c], fmaxf(__uint_as_float(w[c][i]), __uint_as_float(w[c][i + 1])));
#pragma unroll
        for (int i = 0; i < 4; ++i) tops[i] *= a.factor;
      }
      float best = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      if (!(best > top + kSlack)) best = top;
      const bool moves = best > top;
      if (__any_sync(0xFFFFFFFFu, moves && top > -INFINITY)) {
        // the product before has to be done with O
        if (!warp_wait(&sh.o_done[x], (s_done - 1) & 1, watch)) return;
        fence_after();
        const float keep = moves ? exp2_approx(top - best) : 1.0f;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          tensor_load(o, o_at + c);
          tensor_loaded(o);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
          tensor_store32(o_at + c, o);
        }
        sum *= keep;
      }
      top = best;
      const float zero = top == -INFINITY ? 0.0f : top;
      const uint64_t units = pack(unit, unit), zeros = pack(-zero, -zero);
      uint64_t sums[2] = {pack(sum, 0.0f), pack(0.0f, 0.0f)};
#pragma unroll
      for (int c = 0; c < kKeys / 32; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          float y[4];
          uint64_t x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            unpack(fma2(pack(__uint_as_float(w[c][i + 2 * e]), __uint_as_float(w[c][i + 2 * e + 1])), units, zeros), y[2 * e], y[2 * e + 1]);
            x[e] = pack(exp2_approx(y[2 * e]), exp2_approx(y[2 * e + 1]));
            sums[e] = add2(sums[e], x[e]);
          }
          if (kFp8) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&sh.v_scale[stage][c * 32 + i]);
            x[0] = mul2(x[0], v.x);
            x[1] = mul2(x[1], v.y);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            unpack(x[e], y[2 * e], y[2 * e + 1]);
            p[i / 2 + e] = pack_bf16(y[2 * e], y[2 * e + 1]);
          }
        }
        tensor_store16(s_at + c * 16, p);
      }
      {
        float s0, s1, s2, s3;
        unpack(sums[0], s0, s1);
        unpack(sums[1], s2, s3);
        sum = (s0 + s1) + (s2 + s3);
      }
      tensor_stored();
      fence_before();
      warp_arrive(&sh.p_full[x], lane);
      if (tile + 1 == tile1) {
        // The products have read the last of this unit's queries: those of the next one can
        // come while this one is finished, if it has rows for this warpgroup. (To look further
        // with this unit held would stop the walk.)
        ++n;
        ended = !take(sh, watch, n);
        fetched = !ended && sh.unit[n % kUnits].rows > x * 128;
        if (fetched) row_next = take_row<D, kFp8>(sh, batch, a, sh.unit[n % kUnits], x, thread, h_next);
      }
    }
    if (fetched) hand_over(sh, x, lane);
    tiles_before += tile1 - tile0;

    // --- the unit's rows are done, here at least
    if (!warp_wait(&sh.o_done[x], (s_done - 1) & 1, watch)) return;
    fence_after();
    const int c_first = unit.c_first, c_last = unit.c_last;
    const int self = static_cast<int>(blockIdx.x);
    const bool shared_unit = c_first != c_last;
    const int r_part = x * 128 + thread;
    Part<D>& part = parts[self == c_first ? 2 * self + 1 : 2 * self];
    const bool some = top > -INFINITY || sum != sum;
    const float inv = some ? 1.0f / sum : 0.0f;
    uint16_t* out = a.out + static_cast<uint64_t>(max(row.token, 0)) * a.out_stride + static_cast<uint64_t>(h) * D;
#pragma unroll
    for (int c = 0; c < D; c += 32) {
      uint32_t w[32];
      __syncwarp();
      tensor_load(w, o_at + c);
      tensor_loaded(w);
      if (row.token < 0) continue;
      if (shared_unit) {
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          part.o[(c + i) / 4][r_part] = make_float4(__uint_as_float(w[i]), __uint_as_float(w[i + 1]), __uint_as_float(w[i + 2]), __uint_as_float(w[i + 3]));
      } else {
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          uint32_t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            y[e] = some ? pack_bf16(__uint_as_float(w[i + 2 * e]) * inv, __uint_as_float(w[i + 2 * e + 1]) * inv) : 0u;
          *reinterpret_cast<uint4*>(out + c + i) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
    }
    if (sh.bad_count[mine % kUnits] != 0 && row.token >= 0 && some)
      add_bad<D, kFp8>(sh, mine, row.lo, row.hi, out, shared_unit ? reinterpret_cast<float*>(&part.o[0][r_part]) : nullptr);
    if (shared_unit) {
      if (row.token >= 0) {
        part.top[r_part] = top;
        part.sum[r_part] = sum;
      }
      if (!group_sync(sh, watch, x, phase, lane)) return;
      if (thread == 0) {
        sh.last[x] = count_done(&counters[2 * c_first + x]) == static_cast<uint32_t>(c_last - c_first);
        if (sh.last[x]) counters[2 * c_first + x] = 0;
      }
      if (!group_sync(sh, watch, x, phase, lane)) return;
      if (sh.last[x]) {
        const int n = c_last - c_first + 1;
        auto part_of = [&](int i) -> const Part<D>& { return parts[2 * (c_first + i) + (i == 0)]; };
        if (row.token >= 0) {
          float most = -INFINITY, l = 0.0f;
#pragma unroll 4
          for (int i = 0; i < n; ++i) most = fmaxf(most, __ldcg(&part_of(i).top[r_part]));
          const float z = most == -INFINITY ? 0.0f : most;
#pragma unroll 4
          for (int i = 0; i < n; ++i) l += __ldcg(&part_of(i).sum[r_part]) * exp2_approx(__ldcg(&part_of(i).top[r_part]) - z);
          const bool any = most > -INFINITY || l != l;
          const float i1 = any ? 1.0f / l : 0.0f;
          if (a.lse != nullptr) a.lse[static_cast<uint64_t>(row.token) * a.q_heads + h] = any ? most * kLn2 + logf(l) : -INFINITY;
#pragma unroll 1
          for (int c = 0; c < D / 4; c += 16) {
            float4 y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = make_float4(0, 0, 0, 0);
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
              const Part<D>& from = part_of(i);
              const float f = exp2_approx(__ldcg(&from.top[r_part]) - z);
              float4 v[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] = __ldcg(&from.o[c + e][r_part]);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                y[e].x += v[e].x * f;
                y[e].y += v[e].y * f;
                y[e].z += v[e].z * f;
                y[e].w += v[e].w * f;
              }
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2)
              *reinterpret_cast<uint4*>(out + (c + e) * 4) =
                  any ? make_uint4(pack_bf16(y[e].x * i1, y[e].y * i1), pack_bf16(y[e].z * i1, y[e].w * i1),
                                   pack_bf16(y[e + 1].x * i1, y[e + 1].y * i1), pack_bf16(y[e + 1].z * i1, y[e + 1].w * i1))
                      : make_uint4(0, 0, 0, 0);
          }
        }
        __syncwarp();
      }
      if (!group_sync(sh, watch, x, phase, lane)) return;  // sh.last has been read
    } else if (row.token >= 0 && a.lse != nullptr) {
      a.lse[static_cast<uint64_t>(row.token) * a.q_heads + h] = some ? top * kLn2 + logf(sum) : -INFINITY;
    }
    __syncwarp();
    fence_before();  // before the next unit's products write O
    leave(sh, mine, lane);
    more = fetched;
    skipped = 0;
    if (!fetched && !ended) {
      more = find(skipped);
      if (more) {
        row_next = take_row<D, kFp8>(sh, batch, a, sh.unit[n % kUnits], x, thread, h_next);
        hand_over(sh, x, lane);
      }
    }
  }
}

template <bool kFp8>
constexpr int threads_of() { return kFp8 ? 512 : 384; }

// kPlain: scores are scale q.k, with scale > 0, alone.
template <int D, bool kFp8, bool kPlain>
__global__ void __launch_bounds__(threads_of<kFp8>(), 1)
many_rows_kernel(const CacheView cache, const BatchView batch, const AttentionArgs a, const Plan* plan, uint32_t* counters,
                 int* flag, Part<D>* parts, int tries, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  extern __shared__ uint8_t raw[];
  Shared<D, kFp8>& sh = *reinterpret_cast<Shared<D, kFp8>*>(raw + ((1024 - (shared_address(raw) & 1023)) & 1023));
  const Watch watch{&sh.failed, tries};
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      barrier_init(&sh.q_full[i], 4);
      barrier_init(&sh.s_full[i], 2);
      barrier_init(&sh.p_full[i], 4);
      barrier_init(&sh.o_done[i], 1);
      barrier_init(&sh.group[i], 4);
    }
    for (int i = 0; i < kStages; ++i) {
      barrier_init(&sh.k_full[i], kFp8 ? kPieces / 2 : 1);
      barrier_init(&sh.k_empty[i], 1);
      barrier_init(&sh.v_full[i], kFp8 ? kPieces / 2 : 1);
      barrier_init(&sh.v_empty[i], 1);
      barrier_init(&sh.v_fixed[i], 2);
    }
    for (int i = 0; i < kRaw; ++i) {
      barrier_init(&sh.raw_full[i], 1);
      barrier_init(&sh.raw_empty[i], 1);
    }
    for (int i = 0; i < kUnits; ++i) {
      barrier_init(&sh.unit_full[i], 1);
      barrier_init(&sh.unit_empty[i], kFp8 ? 9 + kRaw : 11);  // the warps that take units
    }
    barrier_init(&sh.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.failed = 0;
    sh.cache = cache;
    sh.batch = batch;
  }
  constexpr int kIssuer = kFp8 ? 8 + kRaw : 8;
  if (warp == kIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sh.tensor)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  wait_for_previous();

  // The warpgroups of the rows hold a tile's scores in registers. The shares add up to what the
  // block is launched with: 256 x 216 + 128 x 72 = 384 x 168, and 256 x (200 + 56) = 512 x 128
  // (FP8 prompt of 8,191 tokens: 706 us; 192 + 64 718, 184 + 72 748, 176 + 80 756).
  if (warp < 8) {
    if (kFp8) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
  } else {
    if (kFp8) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  }
  if (warp < 8) {
    soften<D, kFp8, kPlain>(sh, watch, cache, batch, a, counters, parts, warp / 4, threadIdx.x % 128, lane);
  } else if (warp == kIssuer) {
    issue_products<D, kFp8>(sh, watch, lane);
    __syncwarp();
    if (elected()) commit(&sh.drained);  // by the lane that issued the products: none outlives the tensor memory
    __syncwarp();
    barrier_settle(&sh.drained, 0);
  } else {
    if constexpr (kFp8) {
      if (warp < 8 + kRaw) convert_tiles<D>(sh, watch, cache, batch, a, warp - 8, lane);
      else copy_codes<D>(sh, watch, cache, batch, a, plan, &k_map, &v_map, lane);
    } else {
      if (warp == 9) copy_tiles<D>(sh, watch, cache, batch, a, plan, &k_map, &v_map, lane);
      else fix_tiles<D>(sh, watch, threadIdx.x - 10 * 32, lane);
    }
  }
  __syncwarp();
  asm volatile("cp.async.wait_all;" ::: "memory");
  let_next_start();
  fence_before();
  __syncthreads();
  fence_after();
  if (threadIdx.x == 0 && sh.failed) *flag = 1;
  if (warp == kIssuer)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tensor) : "memory");
}

std::atomic<int> tries_of_a_wait{kMostTries};

constexpr uint64_t kPlanBytes = (sizeof(Plan) + 255) / 256 * 256;

template <int D, bool kFp8, bool kPlain>
cudaError_t launch_kernel(const CacheView& cache, const CUtensorMap* maps, const BatchView& batch, const AttentionArgs& args,
                   char* workspace, uint32_t* counters, int* flag, cudaStream_t stream) {
  auto kernel = many_rows_kernel<D, kFp8, kPlain>;
  constexpr int kShared = static_cast<int>(sizeof(Shared<D, kFp8>)) + 1024;
  int device = 0;
  cudaGetDevice(&device);
  // SMs of each device whose kernel has been given its shared memory
  static std::atomic<int> sms_of[64];
  int sms = device < 64 ? sms_of[device].load(std::memory_order_relaxed) : 0;
  if (sms == 0) {
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (err != cudaSuccess) {
      cudaGetLastError();
      return err;
    }
    if (device < 64) sms_of[device].store(sms, std::memory_order_relaxed);
  }
  const int grid = std::min(sms, kMaxGrid);
  Plan* plan = reinterpret_cast<Plan*>(workspace);
  const cudaError_t err = launch_early(plan_kernel, 1, kPlanThreads, 0, stream, batch, args, cache.kv_heads, grid,
                                       unit_cost<kFp8, kPlain>(), plan);
  if (err != cudaSuccess) return err;
  return launch_early(kernel, grid, threads_of<kFp8>(), kShared, stream, cache, batch, args, static_cast<const Plan*>(plan), counters,
                      flag, reinterpret_cast<Part<D>*>(workspace + kPlanBytes), tries_of_a_wait.load(std::memory_order_relaxed), maps[0], maps[1]);
}

template <int D, bool kFp8>
cudaError_t launch(const CacheView& cache, const CUtensorMap* maps, const BatchView& batch, const AttentionArgs& args,
                   char* workspace, uint32_t* counters, int* flag, cudaStream_t stream) {
  const bool plain = args.softcap <= 0.0f && args.slopes == nullptr && args.scale > 0.0f;
  return plain ? launch_kernel<D, kFp8, true>(cache, maps, batch, args, workspace, counters, flag, stream)
               : launch_kernel<D, kFp8, false>(cache, maps, batch, args, workspace, counters, flag, stream);
}

}  // namespace

void set_wait_tries(int tries) { tries_of_a_wait.store(tries < 0 ? kMostTries : tries, std::memory_order_relaxed); }

uint64_t many_rows_workspace_bytes(int head_dim) {
  return kPlanBytes + 2 * kMaxGrid * (head_dim == 128 ? sizeof(Part<128>) : sizeof(Part<64>));
}

cudaError_t launch_many_rows(const CacheView& cache, const CUtensorMap* maps, bool fp8, int head_dim, const BatchView& batch,
                             const AttentionArgs& args, char* workspace, uint32_t* counters, int* flag, cudaStream_t stream) {
  auto f = head_dim == 128 ? (fp8 ? launch<128, true> : launch<128, false>) : (fp8 ? launch<64, true> : launch<64, false>);
  return f(cache, maps, batch, args, workspace, counters, flag, stream);
}

}  // namespace esopt
