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
constexpr int kBand = 8;        // column tiles whose feature tiles are neighbours
constexpr int kBlock = 16;      // rows whose adapters are looked at together
constexpr int kMostShares = 8;  // blocks of a cluster

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

constexpr int kShrinkRows = 32;
template <int kSteps>
constexpr int kShrinkWarps = kSteps <= 2 ? 16 : kSteps <= 8 ? 8 : 4;
template <int kSteps>
constexpr int kShrinkBytes = kShrinkWarps<kSteps> * kShrinkRows * (kSteps * 8 + 1) * 4;

// 1 / scale where the matrix's codes are multiplied by their scale in the end and the adapters'
// part must not be; 1 where that is infinite: then the codes count as zeros.
__device__ __forceinline__ float undo_of(const float* w_scale) {
  const float u = w_scale != nullptr ? 1.0f / *w_scale : 1.0f;
  return isinf(u) ? 1.0f : u;
}

// The adapter of row row0 + lane for each lane of a warp, kNone for rows from `end` on.
__device__ __forceinline__ int adapter_of_lane(const ShrinkArgs& a, int row0, int end, int lane) {
  const int row = row0 + lane;
  int r = row;
  if (a.start != nullptr && row0 < end) {
    // The last request that starts at or before row0, 32 starts at a time.
    int lo = 0, span = a.requests;  // among [lo, lo + span)
    while (span > 1) {
      const int step = (span + 31) / 32;
      const int at = lo + lane * step;
      const uint32_t before = __ballot_sync(0xFFFFFFFFu, lane * step < span && a.start[at] <= row0);
      const int chosen = before != 0 ? 31 - __clz(before) : 0;
      lo += chosen * step;
      span = min(step, span - chosen * step);
    }
    // From there on: the requests that start within the 32 rows.
    r = lo;
    for (int at = lo + 1; at < a.requests; at += 32) {
      const int begins = at + lane < a.requests ? a.start[at + lane] : INT32_MAX;
      for (int i = 0; i < 32; ++i) {
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, begins <= row0 + i));
        if (lane == i) r += n;
      }
      if (__shfl_sync(0xFFFFFFFFu, begins, 31) > row0 + 31) break;
    }
  }
  if (row >= end) return kNone;
  const int m = a.adapter[r];
  return static_cast<unsigned>(m) < static_cast<unsigned>(a.count) ? m : kNone;
}

// h of 32 rows with the (blockIdx.y)-th adapter among them, and which adapters rows and blocks
// have. The warps share the depth; the two products of a lane's 16 bytes of x and A take its
// elements in the order in which they lie, the same in both, so each is one load.
template <int kSteps>  // of 8 ranks
__global__ void __launch_bounds__(kShrinkWarps<kSteps> * 32)
shrink_kernel(const ShrinkArgs a) {
  constexpr int kWarps = kShrinkWarps<kSteps>, kPitch = kSteps * 8 + 1;
  extern __shared__ float parts[];  // [warp][row][kPitch]
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int row0 = blockIdx.x * kShrinkRows;
  const int end = a.start != nullptr ? min(max(a.start[a.requests], 0), a.rows) : a.rows;
  const int mine = adapter_of_lane(a, row0, end, lane);
  const uint32_t there = __ballot_sync(0xFFFFFFFFu, row0 + lane < end);
  const uint32_t same = __match_any_sync(0xFFFFFFFFu, mine) & there;
  if (blockIdx.y == 0 && warp == 0) {
    if (row0 + lane < end) a.of_row[row0 + lane] = mine;
    const uint32_t block = 0xFFFFu << (lane & 16);
    if (lane % kBlock == 0 && (there & block) != 0)
      a.of_block[(row0 + lane) / kBlock] = (same & block) == (there & block) ? mine : kMixed;
  }
  const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, mine >= 0 && (same & ((1u << lane) - 1)) == 0);
  if (static_cast<int>(blockIdx.y) >= __popc(firsts)) return;
  uint32_t left = firsts;
  for (int i = blockIdx.y; i > 0; --i) left &= left - 1;
  const int lead = __ffs(left) - 1;
  const int m = __shfl_sync(0xFFFFFFFFu, mine, lead);
  const uint32_t rows = __shfl_sync(0xFFFFFFFFu, same, lead);
  const float factor = (a.scale != nullptr ? a.scale[m] : 1.0f) * undo_of(a.w_scale);

  const int g = lane / 4, t = lane % 4;
  const uint16_t* x0 = a.x + static_cast<uint64_t>(row0 + g) * a.x_stride;
  const uint16_t* from = a.a + m * a.a_stride;
  float sum[2][kSteps][4] = {};
  const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll(kSteps <= 4 ? 4 : 1)
  for (int k0 = warp * 32; k0 < a.in; k0 += kWarps * 32) {
    const int k = k0 + t * 8;
    const bool inside = k < a.in;
    uint4 w[kSteps], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = inside && (rows >> (g + 8 * i) & 1) ? *reinterpret_cast<const uint4*>(x0 + 8 * i * a.x_stride + k) : zero;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      w[s] = inside && s * 8 + g < a.rank ? *reinterpret_cast<const uint4*>(from + static_cast<uint64_t>(s * 8 + g) * a.in + k) : zero;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (!(rows >> (16 * half) & 0xFFFFu)) continue;
      const uint4 p = v[2 * half], q = v[2 * half + 1];
      const uint32_t first[4] = {p.x, q.x, p.y, q.y}, second[4] = {p.z, q.z, p.w, q.w};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        mma_bf16(sum[half][s], first, w[s].x, w[s].y);
        mma_bf16(sum[half][s], second, w[s].z, w[s].w);
      }
    }
  }
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        parts[(warp * kShrinkRows + half * 16 + g + i / 2 * 8) * kPitch + s * 8 + 2 * t + i % 2] = sum[half][s][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kShrinkRows * a.padded; i += kWarps * 32) {
    const int n = i / a.padded, r = i % a.padded;
    if (!(rows >> n & 1)) continue;
    float h = 0.0f;
    if (r < a.rank) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) h += parts[(w * kShrinkRows + n) * kPitch + r];
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

// --- rows that are named one by one ---------------------------------------------------------

// Copies the rows of x that slots name (zeros for those that do not exist) so that they lie in order. A
// warp has a slot.
__global__ void __launch_bounds__(256)
gather_kernel(const RowView rows, uint16_t* to, int in) {
  wait_for_previous();
  let_next_start();
  const int lane = threadIdx.x % 32;
  const int end = min(max(rows.start[rows.segments], 0), rows.rows);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 8 + threadIdx.x / 32; i < end; i += static_cast<int64_t>(gridDim.x) * 8) {
    const int from = rows.index[i];
    const bool there = static_cast<unsigned>(from) < static_cast<unsigned>(rows.x_rows);
    const uint4* x = reinterpret_cast<const uint4*>(rows.x + (there ? from : 0) * rows.x_stride);
    uint4* y = reinterpret_cast<uint4*>(to + i * in);
#pragma unroll 4
    for (int k = lane; k < in / 8; k += 32) y[k] = there ? x[k] : make_uint4(0, 0, 0, 0);
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

constexpr int kPitch = kFeatures + 4;  // of a column of sums
constexpr int kStaged = 16;  // columns that pass through shared memory together

template <int kRows, bool kFp8>
struct Shared {
  using S = Shape<kRows, kFp8>;
  uint8_t w[S::kStages][S::kW];
  uint8_t x[S::kStages][S::kX];
  uint8_t raw[kFp8 ? S::kStages : 1][kFp8 ? S::kRaw : 16];
  float staged[2][kStaged][kPitch];
  uint64_t full[S::kStages], ready[S::kStages], empty[S::kStages], sum_full[2], sum_empty[2], group, drained;
  uint64_t join_full, join_done, turn;
  int before[ES_MAX_EXPERTS + 1];  // column tiles of the segments before each
  int sums[32];
  uint32_t tensor;
  int failed;
  int4 names[2][kRows / 8];  // rows of the fours of each copying warp
};

// What all roles need of a call's tiles. A tile is kFeatures features (gated: 64 and the 64 that
// they are multiplied with) and up to kRows rows of a segment; its depth is `depth` stages. Tiles go to
// clusters in turn, and the blocks of a cluster have a share of the depth each.
struct Plan {
  int columns, features, depth;  // tiles, tiles, stages
  int tiles;
  int shares, rank;  // blocks of a cluster, and this one's place
};

struct Item {
  int row0, rows, group, f0;
  int k0, k1;  // stages
};

template <class Sh>
struct Walk {
  const RowView& rows;
  const Sh& sh;
  Plan plan;
  int at;
  int kRowsOf;
  bool gated;

  __device__ __forceinline__ Walk(const RowView& r, const Sh& s, const Plan& p, int tile_rows, bool g)
      : rows(r), sh(s), plan(p), at(blockIdx.x / p.shares), kRowsOf(tile_rows), gated(g) {}

  __device__ __forceinline__ bool next(Item& item) {
    if (at >= plan.tiles) return false;
    const int tile = at;
    at += gridDim.x / plan.shares;
    item.k0 = plan.depth * plan.rank / plan.shares;
    item.k1 = plan.depth * (plan.rank + 1) / plan.shares;
    const int band = tile / (kBand * plan.features);
    const int rest = tile - band * kBand * plan.features;
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
product_kernel(const MatrixView w, const RowView rows, const ExpandView expand, int* flag, int tries, bool early, int shares,
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
    barrier_init(&sh.join_full, 4 * shares);
    barrier_init(&sh.join_done, 4 * shares);
    barrier_init(&sh.turn, 4);
    barrier_init(&sh.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.failed = 0;
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sh.tensor)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  if (shares > 1) cluster_sync();  // no block arrives at another's barriers before they are made
  else __syncthreads();
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
  plan.shares = shares;
  plan.rank = blockIdx.x % shares;
  const bool named = rows.index != nullptr && !rows.copied;  // rows of x are asked for one by one

  if (warp == 0) {
    // --- copies
    Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
    Item item;
    uint32_t done = 0, items = 0;
    bool fine = true;
    for (; fine && walk.next(item); ++items) {
      // the stages hold what the cluster's blocks have of the tile before
      if (shares > 1 && items > 0 && !(fine = warp_wait(&sh.turn, (items - 1) & 1, watch))) break;
      const int padded = (item.rows + 15) & ~15;
      const int boxes = (padded + S::kBox - 1) / S::kBox;
      for (int k = item.k0; k < item.k1; ++k, ++done) {
        const uint32_t stage = done % kStages;
        if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
        const uint32_t x_to = shared_address(sh.x[stage]);
        if (elected()) {
          barrier_expect(&sh.full[stage], (kFp8 ? S::kRaw : S::kW) + (named ? padded : boxes * S::kBox) * kDepth * 2);
          const uint32_t w_to = kFp8 ? shared_address(sh.raw[stage]) : shared_address(sh.w[stage]);
          load_box(&w_map, w_to, &sh.full[stage], k * kDepth, item.f0, item.group);
          load_box(&w_map, w_to + (kFp8 ? S::kRaw : S::kW) / 2, &sh.full[stage], k * kDepth, item.f0 + (kGated ? outs : 64), item.group);
          if (!named)
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
    if (named) {
      Walk<Shared<kRows, kFp8>> walk(rows, sh, plan, kRows, kGated);
      Item item;
      uint32_t done = 0;
      bool fine = true;
      int4* names = sh.names[warp - 2];
      for (uint32_t items = 0; fine && walk.next(item); ++items) {
        if (shares > 1 && items > 0 && !(fine = warp_wait(&sh.turn, (items - 1) & 1, watch))) break;
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
          names[lane] = make_int4(v[0], v[1], v[2], v[3]);
        }
        __syncwarp();
        for (int k = item.k0; k < item.k1; ++k, ++done) {
          const uint32_t stage = done % kStages;
          if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
          if (elected()) {
            const uint32_t x_to = shared_address(sh.x[stage]);
#pragma unroll 4
            for (int i = begin; i < end; ++i)
              gather_rows(&x_map, x_to + i * (4 * kDepth * 2), &sh.full[stage], k * kDepth, names[i - begin]);
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
      float scale = kFp8 ? *(w.scale + item.group) : 1.0f;
      if (kFp8 && expand.h != nullptr && isinf(1.0f / scale)) scale = 1.0f;
      // Sums of the lane's features of a column to y: gated two features and the two that they are
      // multiplied with, else four.
      auto finish = [&](int column, float4 z) {
        const int row = item.row0 + column;
        const bool absent = rows.index != nullptr && static_cast<unsigned>(rows.index[row]) >= static_cast<unsigned>(rows.x_rows);
        if (kGated) {
          const int f = item.f0 + lane * 2;
          if (f >= outs) return;
          const float g0 = z.x * scale, g1 = z.y * scale;
          const uint32_t y = pack_bf16(g0 / (1.0f + expf(-g0)) * (z.z * scale), g1 / (1.0f + expf(-g1)) * (z.w * scale));
          *reinterpret_cast<uint32_t*>(rows.y + row * rows.y_stride + f) = absent ? 0 : y;
          return;
        }
        const int f = item.f0 + lane * 4;
        if (f >= outs) return;
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
        const uint2 out = make_uint2(pack_bf16(y[0] * scale, y[1] * scale), pack_bf16(y[2] * scale, y[3] * scale));
        *reinterpret_cast<uint2*>(rows.y + row * rows.y_stride + f) = absent ? make_uint2(0, 0) : out;
      };
      if (shares > 1) {
        // The blocks' sums of their depth meet in shared memory, where the stages were: each adds up a share of
        // the columns, in the order of the blocks.
        float* whole = reinterpret_cast<float*>(sh.w);
        for (int c = 0; c < item.rows; c += kStaged) {
          uint32_t r[kStaged];
          tensor_load(r, sum + c);
          tensor_loaded(r);
#pragma unroll
          for (int i = 0; i < kStaged; ++i) whole[(c + i) * kPitch + feature] = __uint_as_float(r[i]);
        }
        fence_before();
        __syncwarp();
        if (lane == 0) barrier_arrive(&sh.sum_empty[half]);
        if (lane < shares) barrier_arrive_at(address_in(shared_address(&sh.join_full), lane));
        if (!(fine = cluster_wait(&sh.join_full, items & 1, watch))) break;
        const int width = (item.rows + shares - 1) / shares;
        const int end = min(item.rows, (plan.rank + 1) * width);
        const uint32_t base = shared_address(whole) + (kGated ? lane * 8 : lane * 16);
#pragma unroll 2
        for (int c = plan.rank * width + mine; c < end; c += 4) {
          float4 v[kMostShares];
#pragma unroll
          for (int q = 0; q < kMostShares; ++q)
            if (q < shares) {
              const uint32_t from = address_in(base + c * (kPitch * 4), q);
              v[q] = kGated ? load_pairs(from, from + kFeatures * 2) : load_from(from);
            }
          float4 z = v[0];
#pragma unroll
          for (int q = 1; q < kMostShares; ++q)
            if (q < shares) {
              z.x += v[q].x;
              z.y += v[q].y;
              z.z += v[q].z;
              z.w += v[q].w;
            }
          finish(c, z);
        }
        __syncwarp();
        if (lane < shares) barrier_arrive_at(address_in(shared_address(&sh.join_done), lane));
        if (!(fine = cluster_wait(&sh.join_done, items & 1, watch))) break;
        fence_async();  // the stages are written by copies next
        warp_arrive(&sh.turn, lane);
        continue;
      }
      for (int c = 0; c < item.rows; c += kStaged, ++chunks) {
        uint32_t r[kStaged];
        tensor_load(r, sum + c);
        tensor_loaded(r);
        if (c + kStaged >= item.rows) {
          fence_before();
          __syncwarp();
          if (lane == 0) barrier_arrive(&sh.sum_empty[half]);
        }
        auto& staged = sh.staged[chunks & 1];
#pragma unroll
        for (int i = 0; i < kStaged; ++i) staged[i][feature] = __uint_as_float(r[i]);
        if (!(fine = group_sync())) break;
#pragma unroll
        for (int i = 0; i < kStaged / 4; ++i) {
          const int column = mine * (kStaged / 4) + i;
          if (c + column >= item.rows) continue;
          if (kGated) {
            const float2 gate = *reinterpret_cast<const float2*>(&staged[column][lane * 2]);
            const float2 up = *reinterpret_cast<const float2*>(&staged[column][64 + lane * 2]);
            finish(c + column, make_float4(gate.x, gate.y, up.x, up.y));
          } else {
            finish(c + column, *reinterpret_cast<const float4*>(&staged[column][lane * 4]));
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
  if (shares > 1) cluster_sync();  // no block leaves while others read its sums or arrive at its barriers
  else __syncthreads();
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

template <int kRows, bool kFp8, bool kGated>
es_status_t launch(const MatrixView& w, const CUtensorMap& w_map, const RowView& rows, const ExpandView& expand, const CUtensorMap* b_map,
                   int columns, int join, bool early, char* workspace, cudaStream_t stream, const char* call) {
  using S = Shape<kRows, kFp8>;
  auto kernel = product_kernel<kRows, kFp8, kGated>;
  constexpr int kBytes = static_cast<int>(sizeof(Shared<kRows, kFp8>)) + 1024;
  static_assert(kBytes <= 232448, "shared memory of a block");
  int device = 0;
  cudaGetDevice(&device);
  // Clusters of 1 to kMostShares blocks that each device holds at once, of a kernel that has been given its
  // shared memory.
  static std::atomic<int> held[64][kMostShares + 1];
  int clusters[kMostShares + 1];
  if (device < 64 && held[device][1].load(std::memory_order_acquire) != 0) {
    for (int i = 1; i <= kMostShares; ++i) clusters[i] = held[device][i].load(std::memory_order_relaxed);
  } else {
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&clusters[1], cudaDevAttrMultiProcessorCount, device);
    for (int i = 2; i <= kMostShares && err == cudaSuccess; ++i) {
      cudaLaunchConfig_t config{};
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = static_cast<unsigned>(i);
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      config.gridDim = dim3(static_cast<unsigned>(i));
      config.blockDim = dim3(S::kThreads);
      config.dynamicSmemBytes = kBytes;
      config.attrs = &attr;
      config.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&clusters[i], kernel, &config) != cudaSuccess) {
        cudaGetLastError();
        clusters[i] = 0;
      }
    }
    if (err != cudaSuccess) {
      cudaGetLastError();
      return cuda_fail(err, call);
    }
    if (device < 64) {
      for (int i = kMostShares; i > 1; --i) held[device][i].store(clusters[i], std::memory_order_relaxed);
      held[device][1].store(clusters[1], std::memory_order_release);
    }
  }
  // The number of blocks that share a tile's depth: the one whose rounds of tiles take the fewest stages. To
  // join costs as much as some.
  const int outs = kGated ? w.out / 2 : w.out, wide = kGated ? kFeatures / 2 : kFeatures;
  const int64_t tiles = static_cast<int64_t>(columns) * ((outs + wide - 1) / wide);
  const int depth = (w.in + kDepth - 1) / kDepth;
  int shares = 1;
  int64_t best = INT64_MAX;
  for (int i = 1; i <= kMostShares && i <= depth; ++i) {
    if (clusters[i] < 1) continue;
    const int64_t cost = (tiles + clusters[i] - 1) / clusters[i] * ((depth + i - 1) / i + (i > 1 ? join : 0));
    if (cost < best) {
      best = cost;
      shares = i;
    }
  }
  const int grid = static_cast<int>(std::min<int64_t>(tiles, clusters[shares])) * shares;
  CUtensorMap x_map, h_map;
  es_status_t st;
  // without rows of x every slot is absent: what is read in their place does not matter
  if (rows.x_rows > 0)
    st = map_rows(&x_map, rows.x, w.in, rows.copied ? rows.rows : rows.x_rows, rows.x_stride, rows.index != nullptr && !rows.copied ? 1 : S::kBox, call);
  else
    st = map_rows(&x_map, w.data, w.in, 1, w.in, 1, call);
  if (st != ES_OK) return st;
  h_map = x_map;
  if (expand.h != nullptr &&
      (st = map_rows(&h_map, expand.h, 2 * expand.padded, rows.rows, 2 * expand.padded, S::kBox, call)) != ES_OK)
    return st;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(shares);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3(static_cast<unsigned>(grid));
  config.blockDim = dim3(S::kThreads);
  config.dynamicSmemBytes = kBytes;
  config.stream = stream;
  config.attrs = attr;
  config.numAttrs = shares > 1 ? 2 : 1;
  cudaError_t err = cudaLaunchKernelEx(&config, kernel, w, rows, expand, reinterpret_cast<int*>(workspace + ES_PROJECT_GAVE_UP),
                                       tries_of_a_wait.load(std::memory_order_relaxed), early, shares, w_map, x_map, h_map,
                                       expand.h != nullptr ? *b_map : x_map);
  const cudaError_t last = cudaGetLastError();
  if (err == cudaSuccess) err = last;
  return err != cudaSuccess ? cuda_fail(err, call) : ES_OK;
}

template <int kRows>
es_status_t launch_rows(const MatrixView& w, const CUtensorMap& w_map, bool fp8, bool gated, const RowView& rows, const ExpandView& expand,
                        const CUtensorMap* b_map, int columns, int join, bool early, char* workspace, cudaStream_t stream, const char* call) {
  auto f = fp8 ? (gated ? launch<kRows, true, true> : launch<kRows, true, false>)
               : (gated ? launch<kRows, false, true> : launch<kRows, false, false>);
  return f(w, w_map, rows, expand, b_map, columns, join, early, workspace, stream, call);
}

constexpr int kFew = 64, kMany = 256;  // rows of a tile
constexpr int kMostExtra = 1024;       // rows up to which B h has room in the workspace

uint64_t padded_rank(int rank) { return static_cast<uint64_t>(rank + 15) / 16 * 16; }
uint64_t rounded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// A launch of a grid of two axes that may begin early.
template <class... P, class... A>
cudaError_t launch_grid(void (*kernel)(P...), dim3 grid, int block, size_t shared, cudaStream_t stream, const A&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = grid;
  config.blockDim = dim3(static_cast<unsigned>(block));
  config.dynamicSmemBytes = shared;
  config.stream = stream;
  config.attrs = &attr;
  config.numAttrs = 1;
  const cudaError_t err = cudaLaunchKernelEx(&config, kernel, P(args)...);
  const cudaError_t last = cudaGetLastError();
  return err != cudaSuccess ? err : last;
}

template <int kSteps>
cudaError_t launch_shrink(const ShrinkArgs& a, cudaStream_t stream) {
  constexpr int kBytes = kShrinkBytes<kSteps>;
  if (kBytes > 48 * 1024) {
    const cudaError_t err = cudaFuncSetAttribute(shrink_kernel<kSteps>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (err != cudaSuccess) {
      cudaGetLastError();
      return err;
    }
  }
  const int most = std::min(std::min(a.requests, a.rows), kShrinkRows);  // adapters that the rows of a block can have
  return launch_grid(shrink_kernel<kSteps>, dim3((a.rows + kShrinkRows - 1) / kShrinkRows, most), kShrinkWarps<kSteps> * 32, kBytes, stream, a);
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

// Behind the head: with adapters h, the adapters of rows and blocks, and B h of up to kMostExtra rows;
// without, rows that are copied in order.
uint64_t project_workspace_bytes(int rank, int rows, int in, int out) {
  const uint64_t n = rows;
  if (rank == 0) return kHead + (rows > kFew ? rounded(n * in * 2) : 0);
  return kHead + rounded(n * 4 * padded_rank(rank)) + 2 * rounded(n * 4) + rounded(std::min(rows, kMostExtra) * uint64_t{4} * out);
}

// Stages that a join of up to `rows` columns takes the time of.
int join_of(int rows) { return 4 + rows / 32; }

es_status_t launch_project(const MatrixView& w, const CUtensorMap& w_map, bool fp8, const AdapterView* adapters, const CUtensorMap* b_map,
                           const int32_t* adapter, const RowView& rows, void* workspace, cudaStream_t stream, const char* call) {
  ExpandView expand{};
  char* at = static_cast<char*>(workspace);
  if (adapters != nullptr) {
    const uint64_t n = rows.rows;
    const int padded = static_cast<int>(padded_rank(adapters->rank));
    char* behind = at + kHead;
    uint16_t* h = reinterpret_cast<uint16_t*>(behind);
    int32_t* of_row = reinterpret_cast<int32_t*>(behind + rounded(n * 4 * padded));
    int32_t* of_block = reinterpret_cast<int32_t*>(behind + rounded(n * 4 * padded) + rounded(n * 4));
    const ShrinkArgs a{rows.x, rows.start, adapter, adapters->a, adapters->scale, w.scale, h, of_row, of_block, rows.x_stride,
                       adapters->a_stride, rows.segments, rows.rows, adapters->count, adapters->rank, padded, w.in};
    const int steps = (adapters->rank + 7) / 8;
    cudaError_t err = steps <= 1   ? launch_shrink<1>(a, stream)
                      : steps <= 2 ? launch_shrink<2>(a, stream)
                      : steps <= 4 ? launch_shrink<4>(a, stream)
                      : steps <= 8 ? launch_shrink<8>(a, stream)
                                   : launch_shrink<16>(a, stream);
    if (err != cudaSuccess) return cuda_fail(err, call);
    expand = ExpandView{h, adapters->b, of_row, of_block, nullptr, adapters->b_stride, adapters->rank, padded};
    if (std::min(rows.segments, rows.rows) > 1 && rows.rows <= kMostExtra) {
      float* extra = reinterpret_cast<float*>(behind + rounded(n * 4 * padded) + 2 * rounded(n * 4));
      auto kernel = adapters->rank % 16 == 0 ? expand_kernel<16> : expand_kernel<8>;
      err = launch_grid(kernel, dim3((w.out + kExpandWarps * kFeatures - 1) / (kExpandWarps * kFeatures), (rows.rows + kExpandRows - 1) / kExpandRows),
                        kExpandWarps * 32, 0, stream, expand, rows.start, extra, rows.segments, rows.rows, w.out);
      if (err != cudaSuccess) return cuda_fail(err, call);
      expand.extra = extra;
    }
  }
  const int tile = rows.rows > kFew ? kMany : kFew;
  auto f = tile == kMany ? launch_rows<kMany> : launch_rows<kFew>;
  return f(w, w_map, fp8, false, rows, expand, b_map, (rows.rows + tile - 1) / tile, join_of(std::min(rows.rows, tile)), adapters != nullptr,
           at, stream, call);
}

es_status_t launch_experts(const MatrixView& w, const CUtensorMap& w_map, bool fp8, bool gated, const RowView& rows, void* workspace,
                           cudaStream_t stream, const char* call) {
  char* at = static_cast<char*>(workspace);
  const int tile = rows.rows > kFew && rows.rows / w.groups > 32 ? kMany : kFew;
  RowView r = rows;
  bool early = false;
  if (tile == kMany && rows.index != nullptr && rows.x_rows > 0) {
    uint16_t* copy = reinterpret_cast<uint16_t*>(at + kHead);
    const cudaError_t err = launch_early(gather_kernel, std::min((rows.rows + 7) / 8, 152 * 8), 256, 0, stream, rows, copy, w.in);
    if (err != cudaSuccess) return cuda_fail(err, call);
    r.x = copy;
    r.x_stride = w.in;
    r.copied = true;
  }
  // column tiles as they are where rows are spread evenly
  const int segments = std::min(rows.rows, w.groups);
  const int each = (rows.rows + segments - 1) / segments;
  auto f = tile == kMany ? launch_rows<kMany> : launch_rows<kFew>;
  return f(w, w_map, fp8, gated, r, ExpandView{}, nullptr, segments * ((each + tile - 1) / tile), join_of(std::min(each, tile)), early, at,
           stream, call);
}

}  // namespace esopt
