// es_project and es_project_experts: products of matrices with rows that choose them.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "es_attention.cuh"
#include "es_checks.h"
#include "es_project_internal.h"
#include "es_tensor.cuh"

namespace esopt {
namespace {

constexpr int kFeatures = 128;  // of a tile: lanes of the tensor memory
constexpr int kDepth = 64;      // of a stage: 128 bytes of bf16
constexpr int kMaxGrid = 192;
constexpr int kCounters = 1024;
constexpr int kBand = 8;        // column tiles whose feature tiles are neighbours
constexpr int kBlock = 16;      // rows whose adapters are looked at together

static_assert(kCounters * sizeof(uint32_t) == ES_PROJECT_GAVE_UP, "the flag is behind the counters");
constexpr uint64_t kHead = ES_PROJECT_GAVE_UP + 256;

// What a block of 16 rows has: one adapter for all of them, none, or several.
constexpr int kNone = -1, kMixed = -2;

// The adapters' part of a product: h = scale (A x) as the sum of two bf16 numbers, [rows][2][padded rank].
struct ExpandView {
  const uint16_t* h;  // NULL: no adapters
  const uint16_t* b;
  const int32_t* of_row;    // adapter of each row, or -1
  const int32_t* of_block;  // of each 16 rows
  const float* extra;       // [rows][out] B h of the rows of mixed blocks, or NULL: where they are written
  uint64_t b_stride;
  int rank, padded;
};

__device__ __forceinline__ float bf16_value(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// --- A x --------------------------------------------------------------------------------

struct ShrinkArgs {
  const uint16_t* x;
  const int32_t* start;
  const int32_t* adapter;
  const uint16_t* a;
  const float* scale;
  const float* w_scale;  // of the shared matrix's codes, or NULL
  uint16_t* h;
  int32_t* of_row;
  int32_t* of_block;
  uint64_t x_stride, a_stride;
  int requests, rows, count, rank, padded, in;
};

constexpr int kShrinkWarps = 8;

// 1 / scale where the matrix's codes are multiplied by their scale in the end and the adapters'
// part must not be; 1 where that is infinite: then the codes count as zeros.
__device__ __forceinline__ float undo_of(const float* w_scale) {
  const float u = w_scale != nullptr ? 1.0f / *w_scale : 1.0f;
  return isinf(u) ? 1.0f : u;
}

// h of 16 rows with the (blockIdx.y)-th adapter among them, and which adapters rows and blocks
// have. The warps share the depth; the two products of a lane's 16 bytes of x and A take its
// elements in the order in which they lie, the same in both, so each is one load.
template <int kSteps>  // of 8 ranks
__global__ void __launch_bounds__(kShrinkWarps * 32)
shrink_kernel(const ShrinkArgs a) {
  __shared__ float parts[kShrinkWarps][16][kSteps * 8 + 1];
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int row0 = blockIdx.x * kBlock;
  const int end = a.start != nullptr ? min(max(a.start[a.requests], 0), a.rows) : a.rows;
  // the adapter of row `lane`
  const int row = row0 + lane % kBlock;
  int mine = kNone;
  if (row < end) {
    int r = row;
    if (a.start != nullptr) {
      int lo = 0, hi = a.requests;  // the last request that starts at or before the row
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.start[mid] <= row) lo = mid;
        else hi = mid;
      }
      r = lo;
    }
    mine = a.adapter[r];
    if (static_cast<unsigned>(mine) >= static_cast<unsigned>(a.count)) mine = kNone;
  }
  const uint32_t there = __ballot_sync(0xFFFFFFFFu, row < end) & 0xFFFFu;
  const uint32_t same = __match_any_sync(0xFFFFFFFFu, mine) & there;
  if (blockIdx.y == 0 && warp == 0) {
    if (lane < kBlock && row < end) a.of_row[row] = mine;
    if (lane == 0 && there != 0) a.of_block[blockIdx.x] = same == there ? mine : kMixed;
  }
  const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, lane < kBlock && mine >= 0 && (same & ((1u << lane) - 1)) == 0);
  if (static_cast<int>(blockIdx.y) >= __popc(firsts)) return;
  uint32_t left = firsts;
  for (int i = blockIdx.y; i > 0; --i) left &= left - 1;
  const int lead = __ffs(left) - 1;
  const int m = __shfl_sync(0xFFFFFFFFu, mine, lead);
  const uint32_t rows = __shfl_sync(0xFFFFFFFFu, same, lead);

  const int g = lane / 4, t = lane % 4;
  const bool low = rows >> g & 1, high = rows >> (g + 8) & 1;
  const uint16_t* x0 = a.x + static_cast<uint64_t>(row0 + g) * a.x_stride;
  const uint16_t* x1 = x0 + 8 * a.x_stride;
  const uint16_t* from = a.a + m * a.a_stride;
  float sum[kSteps][4] = {};
  const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll 4
  for (int k0 = warp * 32; k0 < a.in; k0 += kShrinkWarps * 32) {
    const int k = k0 + t * 8;
    const bool inside = k < a.in;
    const uint4 p = low && inside ? *reinterpret_cast<const uint4*>(x0 + k) : zero;
    const uint4 q = high && inside ? *reinterpret_cast<const uint4*>(x1 + k) : zero;
    uint4 w[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      w[s] = inside && s * 8 + g < a.rank ? *reinterpret_cast<const uint4*>(from + static_cast<uint64_t>(s * 8 + g) * a.in + k) : zero;
    const uint32_t first[4] = {p.x, q.x, p.y, q.y}, second[4] = {p.z, q.z, p.w, q.w};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      mma_bf16(sum[s], first, w[s].x, w[s].y);
      mma_bf16(sum[s], second, w[s].z, w[s].w);
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    parts[warp][g][s * 8 + 2 * t] = sum[s][0];
    parts[warp][g][s * 8 + 2 * t + 1] = sum[s][1];
    parts[warp][g + 8][s * 8 + 2 * t] = sum[s][2];
    parts[warp][g + 8][s * 8 + 2 * t + 1] = sum[s][3];
  }
  __syncthreads();
  const float factor = (a.scale != nullptr ? a.scale[m] : 1.0f) * undo_of(a.w_scale);
  for (int i = threadIdx.x; i < 16 * a.padded; i += kShrinkWarps * 32) {
    const int n = i / a.padded, r = i % a.padded;
    if (!(rows >> n & 1)) continue;
    float h = 0.0f;
    if (r < a.rank) {
      for (int w = 0; w < kShrinkWarps; ++w) h += parts[w][n][r];
      h *= factor;
    }
    const uint32_t hi = pack_bf16(h, 0.0f) & 0xFFFFu;
    uint16_t* to = a.h + static_cast<uint64_t>(row0 + n) * 2 * a.padded + r;
    to[0] = static_cast<uint16_t>(hi);
    // an infinite or NaN h has no second part
    const float rest = h - bf16_value(hi);
    to[a.padded] = static_cast<uint16_t>(pack_bf16(isfinite(rest) ? rest : 0.0f, 0.0f));
  }
}

// --- B h of rows beside others' -------------------------------------------------------------

constexpr int kExpandWarps = 4;
constexpr int kExpandRows = 4;  // of a warp

// extra = B h for the rows of mixed blocks: a warp has kExpandRows rows and 128 features, a lane 4 of them,
// with B's elements kept from row to row where the adapter stays.
template <int kChunk>  // ranks at a time
__global__ void __launch_bounds__(kExpandWarps * 32)
expand_kernel(const ExpandView e, const int32_t* start, float* extra, int requests, int rows, int out) {
  let_next_start();
  wait_for_previous();
  const int end = start != nullptr ? min(max(start[requests], 0), rows) : rows;
  const int lane = threadIdx.x % 32, f = (blockIdx.x * kExpandWarps + threadIdx.x / 32) * kFeatures + lane * 4;
  const int row0 = blockIdx.y * kExpandRows;
  if (row0 >= end || f >= out || e.of_block[row0 / kBlock] != kMixed) return;
  float y[kExpandRows][4] = {};
  int m[kExpandRows];
#pragma unroll
  for (int i = 0; i < kExpandRows; ++i) m[i] = row0 + i < end ? e.of_row[row0 + i] : kNone;
  for (int r0 = 0; r0 < e.rank; r0 += kChunk) {
    uint4 b[4][kChunk / 8];
#pragma unroll
    for (int i = 0; i < kExpandRows; ++i) {
      if (m[i] < 0) continue;
      if (i == 0 || m[i] != m[i - 1]) {
        const uint16_t* from = e.b + m[i] * e.b_stride + static_cast<uint64_t>(f) * e.rank + r0;
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int c = 0; c < kChunk / 8; ++c) b[n][c] = *reinterpret_cast<const uint4*>(from + n * e.rank + c * 8);
      }
      const uint16_t* h = e.h + static_cast<uint64_t>(row0 + i) * 2 * e.padded + r0;
#pragma unroll
      for (int c = 0; c < kChunk / 8; ++c) {
        const uint4 p = *reinterpret_cast<const uint4*>(h + c * 8), q = *reinterpret_cast<const uint4*>(h + e.padded + c * 8);
        const uint32_t pw[4] = {p.x, p.y, p.z, p.w}, qw[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const float lo = bf16_value(pw[d]) + bf16_value(qw[d]), hi = bf16_high(pw[d]) + bf16_high(qw[d]);
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const uint32_t w = d == 0 ? b[n][c].x : d == 1 ? b[n][c].y : d == 2 ? b[n][c].z : b[n][c].w;
            y[i][n] = fmaf(hi, bf16_high(w), fmaf(lo, bf16_value(w), y[i][n]));
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kExpandRows; ++i)
    if (m[i] >= 0)
      *reinterpret_cast<float4*>(extra + static_cast<uint64_t>(row0 + i) * out + f) = make_float4(y[i][0], y[i][1], y[i][2], y[i][3]);
}

// --- the products -----------------------------------------------------------------------

template <int kRows, bool kFp8>
struct Shape {
  static constexpr int kBox = kRows == 64 ? 16 : 64;  // rows of a copy
  static constexpr uint32_t kW = kFeatures * kDepth * 2, kX = kRows * kDepth * 2, kRaw = kFp8 ? kFeatures * kDepth : 0;
  static constexpr int kStages = kFp8 ? (kRows == 64 ? 6 : 3) : (kRows == 64 ? 8 : 4);
  static constexpr int kThreads = kFp8 ? 512 : 256;
};

constexpr int kStaged = 16;  // columns that pass through shared memory together

template <int kRows, bool kFp8>
struct Shared {
  using S = Shape<kRows, kFp8>;
  uint8_t w[S::kStages][S::kW];
  uint8_t x[S::kStages][S::kX];
  uint8_t raw[kFp8 ? S::kStages : 1][kFp8 ? S::kRaw : 16];
  float staged[2][kStaged][kFeatures + 4];
  uint64_t full[S::kStages], ready[S::kStages], empty[S::kStages], sum_full[2], sum_empty[2], group, drained;
  int before[ES_MAX_EXPERTS + 1];  // column tiles of the segments before each
  int sums[32];
  uint32_t tensor;
  int failed;
  uint32_t order;
  int4 named[2][kRows / 8];  // rows of the fours of each copying warp
};

// What all roles need of a call's tiles. A tile is kFeatures features (gated: 64 and the 64 that
// they are multiplied with) and up to kRows rows of a segment; a whole tile's depth is `depth`
// stages. Tiles go to blocks in turn, or, where that leaves blocks idle, all tiles' stages
// lie end to end and each block takes `per` of them.
struct Plan {
  int columns, features, depth;  // tiles, tiles, stages
  int tiles;
  int per;  // 0: whole tiles
};

struct Item {
  int row0, rows, group, f0;
  int k0, k1;  // stages
  int tile, first, last;  // blocks that share the tile
};

template <class Sh>
struct Walk {
  const RowView& rows;
  const Sh& sh;
  Plan plan;
  int at, end;  // tiles or stages
  int kRowsOf;
  bool gated;

  __device__ __forceinline__ Walk(const RowView& r, const Sh& s, const Plan& p, int tile_rows, bool g)
      : rows(r), sh(s), plan(p), kRowsOf(tile_rows), gated(g) {
    at = p.per > 0 ? static_cast<int>(min(static_cast<int64_t>(blockIdx.x) * p.per, static_cast<int64_t>(p.tiles) * p.depth))
                   : blockIdx.x;
    end = p.per > 0 ? static_cast<int>(min(static_cast<int64_t>(blockIdx.x + 1) * p.per, static_cast<int64_t>(p.tiles) * p.depth))
                    : p.tiles;
  }

  __device__ __forceinline__ bool next(Item& item) {
    if (at >= end) return false;
    if (plan.per > 0) {
      item.tile = at / plan.depth;
      item.k0 = at - item.tile * plan.depth;
      item.k1 = min(plan.depth, item.k0 + end - at);
      at += item.k1 - item.k0;
      item.first = item.tile * plan.depth / plan.per;
      item.last = (item.tile * plan.depth + plan.depth - 1) / plan.per;
    } else {
      item.tile = at;
      item.k0 = 0;
      item.k1 = plan.depth;
      item.first = item.last = blockIdx.x;
      at += gridDim.x;
    }
    const int band = item.tile / (kBand * plan.features);
    const int rest = item.tile - band * kBand * plan.features;
    const int wide = min(kBand, plan.columns - band * kBand);
    const int f = rest / wide;
    const int column = band * kBand + rest - f * wide;
    item.f0 = f * (gated ? kFeatures / 2 : kFeatures);
    int s = 0;
    if (!rows.joined) {
      int hi = rows.segments;  // before[s] <= column < before[s + 1]
      while (hi - s > 1) {
        const int mid = (s + hi) / 2;
        if (sh.before[mid] <= column) s = mid;
        else hi = mid;
      }
    }
    int begin, stop;
    segment_of(rows, s, begin, stop, item.group);
    item.row0 = begin + (column - (rows.joined ? 0 : sh.before[s])) * kRowsOf;
    item.rows = min(kRowsOf, stop - item.row0);
    return true;
  }
};

// Runs of a tile's blocks of 16 rows that have one adapter.
struct Runs {
  int id, count;
  __device__ __forceinline__ Runs(const ExpandView& e, int row0, int rows, int lane) {
    count = (rows + kBlock - 1) / kBlock;
    id = lane < count ? e.of_block[row0 / kBlock + lane] : kMixed;
  }
  // The run at block i or behind it: blocks [i, j) with adapter m.
  __device__ __forceinline__ bool next(int& i, int& j, int& m) const {
    while (i < count) {
      m = __shfl_sync(0xFFFFFFFFu, id, i);
      const uint32_t alike = __ballot_sync(0xFFFFFFFFu, id == m) >> i;
      j = min(count, i + (alike == 0xFFFFFFFFu ? 32 : __ffs(~alike) - 1));
      if (m >= 0) return true;
      i = j;
    }
    return false;
  }
};

// Stages of one run: both parts of h in one where 64 columns hold them, else each in its own.
struct Extra {
  int column;    // of h
  int b_column;  // of B
  int steps;     // products of 16
  int twice;     // columns from the first part to the second, 0: one part
};
__device__ __forceinline__ int extras_of(int padded) { return 2 * padded <= kDepth ? 1 : 2 * ((padded + kDepth - 1) / kDepth); }
__device__ __forceinline__ Extra extra_of(int padded, int i) {
  if (2 * padded <= kDepth) return Extra{0, 0, padded / 16, padded};
  const int chunk = i / 2, part = i % 2;
  return Extra{part * padded + chunk * kDepth, chunk * kDepth, min(4, padded / 16 - chunk * 4), 0};
}

template <int kRows, bool kFp8, bool kGated>
__global__ void __launch_bounds__(Shape<kRows, kFp8>::kThreads, 1)
product_kernel(const MatrixView w, const RowView rows, const ExpandView expand, uint32_t* counters, int* flag, float* parts, int tries, bool early,
               const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
               const __grid_constant__ CUtensorMap h_map, const __grid_constant__ CUtensorMap b_map) {
  using S = Shape<kRows, kFp8>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t dynamic[];
  Shared<kRows, kFp8>& sh = *reinterpret_cast<Shared<kRows, kFp8>*>(dynamic + ((1024 - (shared_address(dynamic) & 1023)) & 1023));
  const Watch watch{&sh.failed, tries};
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  constexpr int kConverters = kFp8 ? 8 : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      barrier_init(&sh.full[i], 1);
      barrier_init(&sh.ready[i], kFp8 ? kConverters : 1);
      barrier_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(&sh.sum_full[i], 1);
      barrier_init(&sh.sum_empty[i], 4);
    }
    barrier_init(&sh.group, 4);
    barrier_init(&sh.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.failed = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sh.tensor)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  // Behind the kernels of the adapters' part, which wait for all that came before them and then let
  // the next start, only what they make has to be waited for.
  if (!early) wait_for_previous();

  const int outs = kGated ? w.out / 2 : w.out;
  Plan plan;
  plan.features = (outs + (kGated ? kFeatures / 2 : kFeatures) - 1) / (kGated ? kFeatures / 2 : kFeatures);
  plan.depth = (w.in + kDepth - 1) / kDepth;
  if (rows.joined) {
    int begin, end, group;
    segment_of(rows, 0, begin, end, group);
    plan.columns = (end - begin + kRows - 1) / kRows;
  } else {
    // column tiles of each segment, summed over the segments before it
    int base = 0;
    for (int s0 = 0; s0 < rows.segments; s0 += blockDim.x) {
      const int s = s0 + threadIdx.x;
      int begin = 0, end = 0, group = 0;
      if (s < rows.segments) segment_of(rows, s, begin, end, group);
      const int n = (end - begin + kRows - 1) / kRows;
      int sum = n;
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, sum, m);
        if (lane >= m) sum += y;
      }
      if (lane == 31) sh.sums[warp] = sum;
      __syncthreads();
      int ahead = base;
      for (int i = 0; i < static_cast<int>(blockDim.x) / 32; ++i) {
        if (i < warp) ahead += sh.sums[i];
        base += sh.sums[i];
      }
      if (s < rows.segments) sh.before[s] = ahead + sum - n;
      __syncthreads();
    }
    plan.columns = base;
  }
  plan.tiles = plan.columns * plan.features;
  plan.per = 0;
  const int grid = gridDim.x, waves = (plan.tiles + grid - 1) / grid;
  if (plan.tiles <= kCounters && plan.tiles * 10 < waves * grid * 9)
    plan.per = max(4, static_cast<int>((static_cast<int64_t>(plan.tiles) * plan.depth + grid - 1) / grid));

  if (warp == 0) {
    // --- copies
    Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
    Item item;
    uint32_t done = 0;
    bool fine = true;
    while (fine && walk.next(item)) {
      const int padded = (item.rows + 15) & ~15;
      const int boxes = (padded + S::kBox - 1) / S::kBox;
      for (int k = item.k0; k < item.k1; ++k, ++done) {
        const uint32_t stage = done % kStages;
        if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
        const uint32_t x_to = shared_address(sh.x[stage]);
        if (elected()) {
          barrier_expect(&sh.full[stage], (kFp8 ? S::kRaw : S::kW) + (rows.index != nullptr ? padded : boxes * S::kBox) * kDepth * 2);
          const uint32_t w_to = kFp8 ? shared_address(sh.raw[stage]) : shared_address(sh.w[stage]);
          load_box(&w_map, w_to, &sh.full[stage], k * kDepth, item.f0, item.group);
          load_box(&w_map, w_to + (kFp8 ? S::kRaw : S::kW) / 2, &sh.full[stage], k * kDepth, item.f0 + (kGated ? outs : 64), item.group);
          if (rows.index == nullptr)
            for (int i = 0; i < boxes; ++i)
              load_box(&x_map, x_to + i * (S::kBox * kDepth * 2), &sh.full[stage], k * kDepth, item.row0 + i * S::kBox);
        }
        __syncwarp();
      }
      if (!fine || expand.h == nullptr || item.k1 < plan.depth) continue;
      if (early) wait_for_previous();
      const Runs runs(expand, item.row0, item.rows, lane);
      for (int i = 0, j, m; fine && runs.next(i, j, m); i = j) {
        const int run_boxes = ((j - i) * kBlock + S::kBox - 1) / S::kBox;
        for (int e = 0; e < extras_of(expand.padded); ++e, ++done) {
          const Extra extra = extra_of(expand.padded, e);
          const uint32_t stage = done % kStages;
          if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
          if (elected()) {
            barrier_expect(&sh.full[stage], S::kW + run_boxes * S::kBox * kDepth * 2);
            const uint32_t w_to = shared_address(sh.w[stage]), x_to = shared_address(sh.x[stage]);
            load_box(&b_map, w_to, &sh.full[stage], extra.b_column, item.f0, m);
            load_box(&b_map, w_to + S::kW / 2, &sh.full[stage], extra.b_column, item.f0 + 64, m);
            for (int b = 0; b < run_boxes; ++b)
              load_box(&h_map, x_to + b * (S::kBox * kDepth * 2), &sh.full[stage], extra.column, item.row0 + i * kBlock + b * S::kBox);
          }
          __syncwarp();
        }
      }
    }
    // no copy outlives the block
    for (uint32_t i = done > kStages ? done - kStages : 0; i < done; ++i) barrier_settle(&sh.full[i % kStages], i / kStages & 1);
  } else if (warp == 1) {
    // --- products
    Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
    Item item;
    uint32_t done = 0, items = 0;
    const uint64_t plain = operand(0, 16);
    bool fine = true;
    while (fine && walk.next(item)) {
      const uint32_t half = items & 1;
      const uint32_t sum = sh.tensor + half * 256;
      if (!(fine = warp_wait(&sh.sum_empty[half], (items / 2 & 1) ^ 1, watch))) break;
      fence_after();
      const uint32_t kind = product_of(0, false) | static_cast<uint32_t>((item.rows + 15) / 16 * 2) << 17;
      for (int k = item.k0; k < item.k1; ++k, ++done) {
        const uint32_t stage = done % kStages;
        if (!(fine = warp_wait(&sh.full[stage], done / kStages & 1, watch))) break;
        if (kFp8 && !(fine = warp_wait(&sh.ready[stage], done / kStages & 1, watch))) break;
        fence_after();
        const uint64_t a = plain + (shared_address(sh.w[stage]) >> 4), b = plain + (shared_address(sh.x[stage]) >> 4);
        if (elected()) {
#pragma unroll
          for (int i = 0; i < 4; ++i) multiply(sum, a + i * 2, b + i * 2, kind, k > item.k0 || i > 0);
          commit(&sh.empty[stage]);
        }
        __syncwarp();
      }
      if (fine && expand.h != nullptr && item.k1 == plan.depth) {
        if (early) wait_for_previous();
        const Runs runs(expand, item.row0, item.rows, lane);
        for (int i = 0, j, m; fine && runs.next(i, j, m); i = j) {
          const uint32_t run_kind = product_of(0, false) | static_cast<uint32_t>((j - i) * 2) << 17;
          for (int e = 0; e < extras_of(expand.padded); ++e, ++done) {
            const Extra extra = extra_of(expand.padded, e);
            const uint32_t stage = done % kStages;
            if (!(fine = warp_wait(&sh.full[stage], done / kStages & 1, watch))) break;
            if (kFp8 && !(fine = warp_wait(&sh.ready[stage], done / kStages & 1, watch))) break;
            fence_after();
            const uint64_t a = plain + (shared_address(sh.w[stage]) >> 4), b = plain + (shared_address(sh.x[stage]) >> 4);
            if (elected()) {
              for (int s = 0; s < extra.steps; ++s) {
                multiply(sum + i * kBlock, a + s * 2, b + s * 2, run_kind, true);
                if (extra.twice > 0) multiply(sum + i * kBlock, a + s * 2, b + extra.twice / 8 + s * 2, run_kind, true);
              }
              commit(&sh.empty[stage]);
            }
            __syncwarp();
          }
        }
      }
      if (!fine) break;
      if (elected()) commit(&sh.sum_full[half]);
      __syncwarp();
      ++items;
    }
    __syncwarp();
    if (elected()) commit(&sh.drained);  // by the lane that issued the products: none outlives the tensor memory
    __syncwarp();
    barrier_settle(&sh.drained, 0);
  } else if (warp < 4) {
    // --- copies of rows that are named one by one, four at a time, half of them by each of two warps
    if (rows.index != nullptr) {
      Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
      Item item;
      uint32_t done = 0;
      bool fine = true;
      int4* named = sh.named[warp - 2];
      while (fine && walk.next(item)) {
        const int fours = (item.rows + 15) / 16 * 4;
        const int begin = warp == 2 ? 0 : fours / 2, end = warp == 2 ? fours / 2 : fours;
        __syncwarp();
        if (lane < end - begin) {
          int v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int r = (begin + lane) * 4 + q;
            v[q] = r < item.rows ? rows.index[item.row0 + r] : 0;
            if (static_cast<unsigned>(v[q]) >= static_cast<unsigned>(rows.x_rows)) v[q] = 0;
          }
          named[lane] = make_int4(v[0], v[1], v[2], v[3]);
        }
        __syncwarp();
        for (int k = item.k0; k < item.k1; ++k, ++done) {
          const uint32_t stage = done % kStages;
          if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
          if (elected()) {
            const uint32_t x_to = shared_address(sh.x[stage]);
#pragma unroll 4
            for (int i = begin; i < end; ++i)
              gather_rows(&x_map, x_to + i * (4 * kDepth * 2), &sh.full[stage], k * kDepth, named[i - begin]);
          }
          __syncwarp();
        }
      }
      for (uint32_t i = done > kStages ? done - kStages : 0; i < done; ++i) barrier_settle(&sh.full[i % kStages], i / kStages & 1);
    }
  } else if (warp < 8) {
    // --- results: a thread reads a feature's lane, and writes four features of a row
    Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
    Item item;
    uint32_t items = 0, chunks = 0;
    const int mine = warp - 4, feature = threadIdx.x - 128;
    uint32_t syncs = 0;
    // the four warps; false as barrier_wait
    auto group_sync = [&] {
      warp_arrive(&sh.group, lane);
      return warp_wait(&sh.group, syncs++ & 1, watch);
    };
    bool fine = true;
    if (early) wait_for_previous();
    for (; fine && walk.next(item); ++items) {
      const uint32_t half = items & 1;
      if (!(fine = warp_wait(&sh.sum_full[half], items / 2 & 1, watch))) break;
      fence_after();
      const uint32_t sum = sh.tensor + half * 256 + (static_cast<uint32_t>(mine) << 21);
      const bool alone = item.first == item.last;
      if (!alone) {
        const int slot = 2 * blockIdx.x + (item.k0 == 0 ? 1 : 0);
        float* to = parts + static_cast<uint64_t>(slot) * kRows * kFeatures + feature;
        for (int c = 0; c < item.rows; c += kStaged) {
          uint32_t r[kStaged];
          tensor_load(r, sum + c);
          tensor_loaded(r);
#pragma unroll
          for (int i = 0; i < kStaged; ++i)
            if (c + i < item.rows) to[(c + i) * kFeatures] = __uint_as_float(r[i]);
        }
        fence_before();
        if (!(fine = group_sync())) break;
        if (feature == 0) sh.order = count_done(&counters[item.tile]);
        if (!(fine = group_sync())) break;
        const bool last = sh.order == static_cast<uint32_t>(item.last - item.first);
        if (lane == 0) barrier_arrive(&sh.sum_empty[half]);
        if (!(fine = group_sync())) break;  // before the next item's count
        if (!last) continue;
        if (feature == 0) counters[item.tile] = 0;
      }
      float scale = kFp8 ? *(w.scale + item.group) : 1.0f;
      if (kFp8 && expand.h != nullptr && isinf(1.0f / scale)) scale = 1.0f;
      for (int c = 0; c < item.rows; c += kStaged, ++chunks) {
        float v[kStaged];
        if (alone) {
          uint32_t r[kStaged];
          tensor_load(r, sum + c);
          tensor_loaded(r);
#pragma unroll
          for (int i = 0; i < kStaged; ++i) v[i] = __uint_as_float(r[i]);
          if (c + kStaged >= item.rows) {
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(&sh.sum_empty[half]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kStaged; ++i) v[i] = 0.0f;
          for (int b = item.first; b <= item.last; ++b) {
            const int slot = 2 * b + (b == item.first ? 1 : 0);
            const float* part = parts + static_cast<uint64_t>(slot) * kRows * kFeatures + feature;
#pragma unroll
            for (int i = 0; i < kStaged; ++i)
              if (c + i < item.rows) v[i] += __ldcg(part + (c + i) * kFeatures);
          }
        }
        auto& staged = sh.staged[chunks & 1];
#pragma unroll
        for (int i = 0; i < kStaged; ++i) staged[i][feature] = v[i];
        if (!(fine = group_sync())) break;
#pragma unroll
        for (int i = 0; i < kStaged / 4; ++i) {
          const int column = mine * (kStaged / 4) + i;
          const int row = item.row0 + c + column;
          if (c + column >= item.rows) continue;
          if (kGated) {
            const int f = item.f0 + lane * 2;
            const float2 gate = *reinterpret_cast<const float2*>(&staged[column][lane * 2]);
            const float2 up = *reinterpret_cast<const float2*>(&staged[column][64 + lane * 2]);
            const float g0 = gate.x * scale, g1 = gate.y * scale;
            uint32_t y = pack_bf16(g0 / (1.0f + expf(-g0)) * (up.x * scale), g1 / (1.0f + expf(-g1)) * (up.y * scale));
            if (rows.index != nullptr && static_cast<unsigned>(rows.index[row]) >= static_cast<unsigned>(rows.x_rows)) y = 0;
            if (f < outs) *reinterpret_cast<uint32_t*>(rows.y + row * rows.y_stride + f) = y;
          } else {
            const int f = item.f0 + lane * 4;
            if (f >= outs) continue;
            const float4 z = *reinterpret_cast<const float4*>(&staged[column][lane * 4]);
            float y[4] = {z.x, z.y, z.z, z.w};
            if (expand.h != nullptr && expand.of_block[row / kBlock] == kMixed) {
              const int m = expand.of_row[row];
              if (m >= 0 && expand.extra != nullptr) {
                const float4 v = *reinterpret_cast<const float4*>(expand.extra + static_cast<uint64_t>(row) * outs + f);
                y[0] += v.x;
                y[1] += v.y;
                y[2] += v.z;
                y[3] += v.w;
              } else if (m >= 0) {
                const uint16_t* h = expand.h + static_cast<uint64_t>(row) * 2 * expand.padded;
                const uint16_t* b = expand.b + m * expand.b_stride + static_cast<uint64_t>(f) * expand.rank;
                for (int r = 0; r < expand.rank; r += 8) {
                  const uint4 p = *reinterpret_cast<const uint4*>(h + r), q = *reinterpret_cast<const uint4*>(h + expand.padded + r);
                  const uint32_t pw[4] = {p.x, p.y, p.z, p.w}, qw[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                  for (int n = 0; n < 4; ++n) {
                    const uint4 o = *reinterpret_cast<const uint4*>(b + n * expand.rank + r);
                    const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                      y[n] = fmaf(bf16_value(pw[d]) + bf16_value(qw[d]), bf16_value(ow[d]), y[n]);
                      y[n] = fmaf(bf16_high(pw[d]) + bf16_high(qw[d]), bf16_high(ow[d]), y[n]);
                    }
                  }
                }
              }
            }
            uint2 out = make_uint2(pack_bf16(y[0] * scale, y[1] * scale), pack_bf16(y[2] * scale, y[3] * scale));
            if (rows.index != nullptr && static_cast<unsigned>(rows.index[row]) >= static_cast<unsigned>(rows.x_rows))
              out = make_uint2(0, 0);
            *reinterpret_cast<uint2*>(rows.y + row * rows.y_stride + f) = out;
          }
        }
      }
    }
  } else if (kFp8 && warp >= 8) {
    // --- codes to bf16
    Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
    Item item;
    uint32_t done = 0;
    const bool dead = expand.h != nullptr && isinf(1.0f / *w.scale);
    bool fine = true;
    while (fine && walk.next(item)) {
      int extra = 0;
      if (expand.h != nullptr && item.k1 == plan.depth) {
        if (early) wait_for_previous();
        const Runs runs(expand, item.row0, item.rows, lane);
        for (int i = 0, j, m; runs.next(i, j, m); i = j) extra += extras_of(expand.padded);
      }
      for (int k = item.k0; k < item.k1 + extra; ++k, ++done) {
        const uint32_t stage = done % kStages;
        if (!(fine = warp_wait(&sh.full[stage], done / kStages & 1, watch))) break;
        if (k < item.k1) {
          // 16 codes a lane: row `at`, 64 bytes of codes, 128 of bf16 with the pieces of 16 bytes swizzled
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int n = (i * 8 + warp - 8) * 32 + lane;
            const int at = n / 4, piece = n % 4;
            const uint4 c = *reinterpret_cast<const uint4*>(&sh.raw[stage][at * kDepth + piece * 16]);
            const uint32_t code[4] = {c.x, c.y, c.z, c.w};
            uint32_t v[8];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              v[2 * d] = dead ? 0 : bf16_of_e4m3(code[d] & 0xFFFFu);
              v[2 * d + 1] = dead ? 0 : bf16_of_e4m3(code[d] >> 16);
            }
            uint8_t* to = &sh.w[stage][at * 128];
            *reinterpret_cast<uint4*>(to + ((piece * 2) ^ (at & 7)) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<uint4*>(to + ((piece * 2 + 1) ^ (at & 7)) * 16) = make_uint4(v[4], v[5], v[6], v[7]);
          }
          fence_async();
        }
        warp_arrive(&sh.ready[stage], lane);
      }
    }
  }
  __syncwarp();
  let_next_start();
  fence_before();
  __syncthreads();
  fence_after();
  if (threadIdx.x == 0 && sh.failed) *flag = 1;
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tensor) : "memory");
}

// --- launches ---------------------------------------------------------------------------

std::atomic<int> tries_of_a_wait{kMostTries};

// [rows][width] bf16 rows, `pitch` elements apart, in boxes of `box` rows by 64 elements.
es_status_t map_rows(CUtensorMap* map, const void* base, uint64_t width, uint64_t rows, uint64_t pitch, int box, const char* call) {
  EncodeTiled encode = nullptr;
  const es_status_t st = encode_tiled(&encode);
  if (st != ES_OK) return st;
  const cuuint64_t dims[2] = {width, rows};
  const cuuint64_t strides[1] = {pitch * 2};
  const cuuint32_t boxes[2] = {kDepth, static_cast<cuuint32_t>(box)}, steps[2] = {1, 1};
  const CUresult made = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, boxes, steps,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (made != CUDA_SUCCESS) return fail(ES_ERR_CUDA, "%s: cuTensorMapEncodeTiled returned %d", call, static_cast<int>(made));
  return ES_OK;
}

uint64_t parts_bytes(int tile_rows) { return uint64_t{2} * kMaxGrid * tile_rows * kFeatures * sizeof(float); }

template <int kRows, bool kFp8, bool kGated>
es_status_t launch(const MatrixView& w, const CUtensorMap& w_map, const RowView& rows, const ExpandView& expand, const CUtensorMap* b_map,
                   char* workspace, cudaStream_t stream, const char* call) {
  using S = Shape<kRows, kFp8>;
  auto kernel = product_kernel<kRows, kFp8, kGated>;
  constexpr int kBytes = static_cast<int>(sizeof(Shared<kRows, kFp8>)) + 1024;
  static_assert(kBytes <= 232448, "shared memory of a block");
  int device = 0;
  cudaGetDevice(&device);
  // SMs of each device whose kernel has been given its shared memory
  static std::atomic<int> sms_of[64];
  int sms = device < 64 ? sms_of[device].load(std::memory_order_relaxed) : 0;
  if (sms == 0) {
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (err != cudaSuccess) {
      cudaGetLastError();
      return cuda_fail(err, call);
    }
    if (device < 64) sms_of[device].store(sms, std::memory_order_relaxed);
  }
  CUtensorMap x_map, h_map;
  es_status_t st;
  // without rows of x every slot is absent: what is read in their place does not matter
  if (rows.x_rows > 0)
    st = map_rows(&x_map, rows.x, w.in, rows.x_rows, rows.x_stride, rows.index != nullptr ? 1 : S::kBox, call);
  else
    st = map_rows(&x_map, w.data, w.in, 1, w.in, 1, call);
  if (st != ES_OK) return st;
  h_map = x_map;
  if (expand.h != nullptr &&
      (st = map_rows(&h_map, expand.h, 2 * expand.padded, rows.rows, 2 * expand.padded, S::kBox, call)) != ES_OK)
    return st;
  const cudaError_t err =
      launch_early(kernel, std::min(sms, kMaxGrid), S::kThreads, kBytes, stream, w, rows, expand,
                   reinterpret_cast<uint32_t*>(workspace), reinterpret_cast<int*>(workspace + ES_PROJECT_GAVE_UP),
                   reinterpret_cast<float*>(workspace + kHead), tries_of_a_wait.load(std::memory_order_relaxed), expand.h != nullptr, w_map, x_map, h_map,
                   expand.h != nullptr ? *b_map : x_map);
  return err != cudaSuccess ? cuda_fail(err, call) : ES_OK;
}

template <int kRows>
es_status_t launch_rows(const MatrixView& w, const CUtensorMap& w_map, bool fp8, bool gated, const RowView& rows, const ExpandView& expand,
                        const CUtensorMap* b_map, char* workspace, cudaStream_t stream, const char* call) {
  auto f = fp8 ? (gated ? launch<kRows, true, true> : launch<kRows, true, false>)
               : (gated ? launch<kRows, false, true> : launch<kRows, false, false>);
  return f(w, w_map, rows, expand, b_map, workspace, stream, call);
}

constexpr int kFew = 64, kMany = 256;  // rows of a tile
constexpr int kMostExtra = 1024;       // rows up to which B h has room in the workspace

uint64_t padded_rank(int rank) { return static_cast<uint64_t>(rank + 15) / 16 * 16; }
uint64_t rounded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// A launch of a grid of two axes that may begin early.
template <class... P, class... A>
cudaError_t launch_grid(void (*kernel)(P...), dim3 grid, int block, cudaStream_t stream, const A&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = grid;
  config.blockDim = dim3(static_cast<unsigned>(block));
  config.stream = stream;
  config.attrs = &attr;
  config.numAttrs = 1;
  const cudaError_t err = cudaLaunchKernelEx(&config, kernel, P(args)...);
  const cudaError_t last = cudaGetLastError();
  return err != cudaSuccess ? err : last;
}

}  // namespace

void set_project_wait_tries(int tries) { tries_of_a_wait.store(tries < 0 ? kMostTries : tries, std::memory_order_relaxed); }

es_status_t map_matrices(CUtensorMap* map, const void* data, uint64_t in, uint64_t out, uint64_t groups, uint64_t row_stride,
                         uint64_t group_stride, bool fp8, const char* call) {
  EncodeTiled encode = nullptr;
  const es_status_t st = encode_tiled(&encode);
  if (st != ES_OK) return st;
  const cuuint64_t size = fp8 ? 1 : 2;
  const cuuint64_t dims[3] = {in, out, groups};
  const cuuint64_t strides[2] = {row_stride * size, group_stride * size};
  const cuuint32_t box[3] = {kDepth, kFeatures / 2, 1}, steps[3] = {1, 1, 1};
  const CUresult made = encode(map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(data),
                               dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               fp8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (made != CUDA_SUCCESS) return fail(ES_ERR_CUDA, "%s: cuTensorMapEncodeTiled returned %d", call, static_cast<int>(made));
  return ES_OK;
}

// Behind the head: parts of tiles that blocks share; h; the adapters of rows and blocks; B h of up to
// kMostExtra rows.
uint64_t project_workspace_bytes(int rank, int rows, int out) {
  const uint64_t n = rows;
  uint64_t bytes = kHead + parts_bytes(rows > kFew ? kMany : kFew);
  if (rank > 0) bytes += rounded(n * 4 * padded_rank(rank)) + 2 * rounded(n * 4) + rounded(std::min(rows, kMostExtra) * uint64_t{4} * out);
  return bytes;
}

es_status_t launch_project(const MatrixView& w, const CUtensorMap& w_map, bool fp8, const AdapterView* adapters, const CUtensorMap* b_map,
                           const int32_t* adapter, const RowView& rows, void* workspace, cudaStream_t stream, const char* call) {
  ExpandView expand{};
  char* at = static_cast<char*>(workspace);
  if (adapters != nullptr) {
    const uint64_t n = rows.rows;
    const int padded = static_cast<int>(padded_rank(adapters->rank));
    char* behind = at + kHead + parts_bytes(rows.rows > kFew ? kMany : kFew);
    uint16_t* h = reinterpret_cast<uint16_t*>(behind);
    int32_t* of_row = reinterpret_cast<int32_t*>(behind + rounded(n * 4 * padded));
    int32_t* of_block = reinterpret_cast<int32_t*>(behind + rounded(n * 4 * padded) + rounded(n * 4));
    const ShrinkArgs a{rows.x, rows.start, adapter, adapters->a, adapters->scale, w.scale, h, of_row, of_block, rows.x_stride,
                       adapters->a_stride, rows.segments, rows.rows, adapters->count, adapters->rank, padded, w.in};
    const int steps = (adapters->rank + 7) / 8;
    auto shrink = steps <= 1 ? shrink_kernel<1> : steps <= 2 ? shrink_kernel<2> : steps <= 4 ? shrink_kernel<4>
                : steps <= 8 ? shrink_kernel<8> : shrink_kernel<16>;
    const int most = std::min(std::min(rows.segments, rows.rows), kBlock);  // adapters that 16 rows can have
    cudaError_t err = launch_grid(shrink, dim3((rows.rows + kBlock - 1) / kBlock, most), kShrinkWarps * 32, stream, a);
    if (err != cudaSuccess) return cuda_fail(err, call);
    expand = ExpandView{h, adapters->b, of_row, of_block, nullptr, adapters->b_stride, adapters->rank, padded};
    if (most > 1 && rows.rows <= kMostExtra) {
      float* extra = reinterpret_cast<float*>(behind + rounded(n * 4 * padded) + 2 * rounded(n * 4));
      auto kernel = adapters->rank % 16 == 0 ? expand_kernel<16> : expand_kernel<8>;
      err = launch_grid(kernel, dim3((w.out + kExpandWarps * kFeatures - 1) / (kExpandWarps * kFeatures), (rows.rows + kExpandRows - 1) / kExpandRows),
                        kExpandWarps * 32, stream, expand, rows.start, extra, rows.segments, rows.rows, w.out);
      if (err != cudaSuccess) return cuda_fail(err, call);
      expand.extra = extra;
    }
  }
  auto f = rows.rows > kFew ? launch_rows<kMany> : launch_rows<kFew>;
  return f(w, w_map, fp8, false, rows, expand, b_map, at, stream, call);
}

es_status_t launch_experts(const MatrixView& w, const CUtensorMap& w_map, bool fp8, bool gated, const RowView& rows, void* workspace,
                           cudaStream_t stream, const char* call) {
  auto f = rows.rows > kFew && rows.rows / w.groups > 32 ? launch_rows<kMany> : launch_rows<kFew>;
  return f(w, w_map, fp8, gated, rows, ExpandView{}, nullptr, static_cast<char*>(workspace), stream, call);
}

}  // namespace esopt
