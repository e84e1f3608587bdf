// es_project and es_project_experts: products of matrices with rows that choose them.
//
//   y_i = c_g W_g x_{r(i)} + B_m (s_m A_m x_i)
//
// with g the matrix and m the adapter of row i, both by segments of rows; gated: silu of the first half of the
// features times the second.
//
// What bounds them: the bytes of W where an expert or a step has few rows (2 n operations a byte of bf16, so up
// to some 290 rows), the tensor cores above. So one kernel takes both: features are the lanes of the tensor
// memory, 128 a block, and rows its columns, from 16 to 256 in steps of 16, so that a ragged segment costs what
// its rows cost and weights are read once where a segment has up to 256 rows.
//   warp 0         copies W and x by TMA, 64 elements of a row a stage (FP8: 128 codes)
//   warp 1         issues the products
//   warps 2, 3     copy rows of x that are named one by one (gather4)
//   warps 4 - 7    read the sums, and write them
//   warps 8 - 15   FP8: turn codes into bf16, which holds them exactly
// Tiles of 256 rows belong to pairs of blocks (cta_group::2), each of which copies half of x: what an SM can
// ask of L2 at once bounds a block alone (650 cycles for the 512 of a stage's products; 528 by pairs). Two
// tiles' sums have room in the tensor memory, so writing one runs beside the products of the next.
//
// Blocks are persistent and take tiles in turn, in bands of kBand column tiles, so that those that run
// together share W and x in L2. Where the tiles are fewer than the blocks, up to eight share a tile's depth, in a
// cluster: each sends the others their columns of its sums, by bulk copies between shared memories into the stages,
// which are empty then, and sums what it is sent in the order of the blocks. So results do not depend on timing.
//
// Adapters. A kernel of its own makes h = s A x, for 32 rows and one adapter a block, and keeps it as the sum of two bf16
// numbers (2^-16 of it, where a result's rounding is 2^-9; and as it is, in fp32, where that kernel makes B h too). Where 16
// rows have one adapter, B h is further products into the same sums. Where members meet within 16 rows, products would
// multiply one's B by the others' zeros, and infinities or NaN of a member that has diverged would reach all of them; there
// B h is made in fp32, row by row, by that kernel where it has room in the workspace (kMostExtra), else where results are
// written. The product's kernel starts beside it, and waits where the adapters' part is needed.
//
// Measured (GB300, us a pass): project_prompts 13,741 rows of 30 members, 5,120 to 17,408 features, rank 32, 1,395 in ten
// passes (1,772 TFLOP/s, 91 % of the card's bf16 matrix rate in a burst), 1,544 to 1,590 in long loops (1,440 MHz at 1,373 W, the power
// limit); FP8 2,316. 4,096 rows without adapters 368 to 393 (FP8 687; the library's bf16 product 391). experts_prompt
// 32,764 rows of 29 experts gathered and gated 550 in ten passes, 43 of them the gather, 597 to 605 in long loops (1,530 MHz at
// 1,372 W); FP8 874. experts_step 762 MB of experts for 576 rows 114 to 116 (6,680 to 6,550 GB/s, 98 to 97 %). project_step 192 members' rows
// through 73 MB 36 (22 without the adapters).
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstddef>

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
constexpr int kMostShares = 8;  // of a tile's depth

constexpr uint64_t kHead = ES_PROJECT_GAVE_UP + 256;

// What a block of 16 rows has: one adapter for all of them, none, or several.
constexpr int kNone = -1, kMixed = -2;

// What a column of a tile is, beside the adapter that is still to be added to it: nothing is, its row
// of x does not exist, it is not there.
constexpr int kPlain = -1, kAbsent = -2, kOut = -3;

// The adapters' part of a product: h = scale (A x) as the sum of two bf16 numbers, [rows][2][padded rank].
struct ExpandView {
  const uint16_t* h;  // NULL: no adapters
  const uint16_t* b;
  const int32_t* of_row;    // adapter of each row, or -1
  const int32_t* of_block;  // of each 16 rows
  const float* extra;       // [rows][out] B h of the rows of mixed blocks, or NULL: it is made where they are written
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
  const uint16_t* b;
  float* extra;  // [rows][out] B h of the rows of mixed blocks, or NULL
  uint64_t x_stride, a_stride, b_stride;
  int requests, rows, count, rank, padded, in, out;
};

constexpr int kShrinkRows = 32;
constexpr int kShrinkWarps = 4;

// 1 / scale where the matrix's codes are multiplied by their scale in the end and the adapters'
// part, made by products into the same sums, must not be; 1 where that is infinite: then the codes count as zeros.
__device__ __forceinline__ float undo_of(const float* w_scale) {
  const float u = w_scale != nullptr ? 1.0f / *w_scale : 1.0f;
  return isinf(u) ? 1.0f : u;
}

// Whether the scale is so far from 1 that the adapters' part in its units could be infinite, or lose its second
// part, where it is an ordinary number itself (1 / 1.2e-38 times an h of 5 is infinite): then every block with adapters counts as
// mixed, and B h is added behind the scale. Real scales, max|w| / 448, are near 2^-12.
__device__ __forceinline__ bool apart_of(const float* w_scale) {
  if (w_scale == nullptr || isinf(1.0f / *w_scale)) return false;
  const float size = fabsf(*w_scale);
  return !(size >= 0x1p-32f && size <= 0x1p32f);
}

// The adapter of row row0 + lane for each lane of a warp, kNone for rows from `end` on.
__device__ __forceinline__ int adapter_of_lane(const ShrinkArgs& a, int row0, int end, int lane) {
  const int row = row0 + lane;
  int r = row;
  if (a.start != nullptr && a.requests <= 128) {
    // all starts at once: row0 + i is in the request before the first that starts behind it
    int begins[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) begins[j] = j * 32 + lane < a.requests ? a.start[j * 32 + lane] : INT32_MAX;
    r = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j * 32 >= a.requests) break;
      for (int i = 0; i < 32; ++i) {
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, begins[j] <= row0 + i));
        if (lane == i) r += n;
      }
    }
    r = max(r, 0);
  } else if (a.start != nullptr && row0 < end) {
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

// Eight ranks of B for four features, and their part of B h.
struct Factors {
  uint4 b[4];
  __device__ __forceinline__ void take(const uint16_t* from, int rank) {
#pragma unroll
    for (int n = 0; n < 4; ++n) b[n] = *reinterpret_cast<const uint4*>(from + n * rank);
  }
  __device__ __forceinline__ void add(float (&y)[4], const float* h) const {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const float low = h[d * 2], high = h[d * 2 + 1];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const uint32_t w = d == 0 ? b[n].x : d == 1 ? b[n].y : d == 2 ? b[n].z : b[n].w;
        y[n] = fmaf(high, bf16_high(w), fmaf(low, bf16_value(w), y[n]));
      }
    }
  }
};

// h of 32 rows with each adapter among them (shared out along blockIdx.y), and which adapters rows and
// blocks have. The warps of the cluster's gridDim.z blocks share the depth; the two products of a lane's 16 bytes of
// x and A take its elements in the order in which they lie, the same in both, so each is one load.
template <int kSteps>  // of 8 ranks
__global__ void __launch_bounds__(kShrinkWarps * 32)
shrink_kernel(const ShrinkArgs a) {
  constexpr int kWarps = kShrinkWarps, kPitch = kSteps * 8 + 1;
  extern __shared__ float parts[];  // [warp][row][kPitch]
  wait_for_previous();
  let_next_start();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int row0 = blockIdx.x * kShrinkRows;
  const int end = a.start != nullptr ? min(max(a.start[a.requests], 0), a.rows) : a.rows;
  const int mine = adapter_of_lane(a, row0, end, lane);
  const uint32_t there = __ballot_sync(0xFFFFFFFFu, row0 + lane < end);
  const uint32_t same = __match_any_sync(0xFFFFFFFFu, mine) & there;
  const bool apart = apart_of(a.w_scale);
  if (blockIdx.y == 0 && blockIdx.z == 0 && warp == 0) {
    if (row0 + lane < a.rows) a.of_row[row0 + lane] = mine;
    const uint32_t block = 0xFFFFu << (lane & 16);
    if (lane % kBlock == 0 && row0 + lane < a.rows)
      a.of_block[(row0 + lane) / kBlock] = (same & block) == (there & block) && !(apart && mine >= 0) ? mine : kMixed;
  }
  // rows of blocks of 16 that have one adapter alone get B h by products
  const uint32_t low = 0xFFFFu, high = 0xFFFF0000u;
  const uint32_t alone_low = __match_any_sync(0xFFFFFFFFu, mine) & there & low, alone_high = __match_any_sync(0xFFFFFFFFu, mine) & there & high;
  const bool mixed_low = __shfl_sync(0xFFFFFFFFu, alone_low, 0) != (there & low);
  const bool mixed_high = __shfl_sync(0xFFFFFFFFu, alone_high, 16) != (there & high);
  const uint32_t mixed = (mixed_low || apart ? low : 0u) | (mixed_high || apart ? high : 0u);
  const uint32_t firsts = __ballot_sync(0xFFFFFFFFu, mine >= 0 && (same & ((1u << lane) - 1)) == 0);
  const int g = lane / 4, t = lane % 4;
  const uint16_t* x0 = a.x + static_cast<uint64_t>(row0 + g) * a.x_stride;
  int turn = 0;
  for (uint32_t left = firsts; left != 0; left &= left - 1, ++turn) {
    if (turn % gridDim.y != blockIdx.y) continue;
    const int lead = __ffs(left) - 1;
    const int m = __shfl_sync(0xFFFFFFFFu, mine, lead);
    const uint32_t rows = __shfl_sync(0xFFFFFFFFu, same, lead);
    const float factor = a.scale != nullptr ? a.scale[m] : 1.0f, undo = undo_of(a.w_scale);
    const uint16_t* from = a.a + m * a.a_stride;
    const uint32_t expanded = a.extra != nullptr ? rows & mixed : 0;
    if (expanded != 0)  // B to L2 meanwhile
      for (int f = ((blockIdx.z * kWarps + warp) * 32 + lane) * 4; f < a.out; f += gridDim.z * kWarps * kFeatures)
        for (int i = 0; i < a.rank * 8; i += 128)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(a.b + m * a.b_stride + static_cast<uint64_t>(f) * a.rank) + i));
    float sum[2][kSteps][4] = {};
    // 64 elements of a row at a time, the next ones asked for before these are multiplied
    struct Taken {
      uint4 v[2][4], w[2][kSteps];
    };
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto take = [&](Taken& to, int k0) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int k = k0 + n * 32 + t * 8;
        const bool inside = k < a.in;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          to.v[n][i] = inside && (rows >> (g + 8 * i) & 1) ? *reinterpret_cast<const uint4*>(x0 + 8 * i * a.x_stride + k) : zero;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
          to.w[n][s] = inside && s * 8 + g < a.rank ? *reinterpret_cast<const uint4*>(from + static_cast<uint64_t>(s * 8 + g) * a.in + k) : zero;
      }
    };
    auto add = [&](const Taken& of) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(rows >> (16 * half) & 0xFFFFu)) continue;
          const uint4 p = of.v[n][2 * half], q = of.v[n][2 * half + 1];
          const uint32_t first[4] = {p.x, q.x, p.y, q.y}, second[4] = {p.z, q.z, p.w, q.w};
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            mma_bf16(sum[half][s], first, of.w[n][s].x, of.w[n][s].y);
            mma_bf16(sum[half][s], second, of.w[n][s].z, of.w[n][s].w);
          }
        }
    };
    const int stride = gridDim.z * kWarps * 64;
    int k0 = (blockIdx.z * kWarps + warp) * 64;
    if constexpr (kSteps <= 4) {
      Taken one, two;
      take(one, k0);
      for (; k0 < a.in; k0 += 2 * stride) {
        take(two, k0 + stride);
        add(one);
        take(one, k0 + 2 * stride);
        add(two);
      }
    } else {
      for (; k0 < a.in; k0 += stride) {
        Taken one;
        take(one, k0);
        add(one);
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
    const int shares = gridDim.z;
    if (shares > 1) {
      // the block's sums to where its first warp's are, each by the thread that has read them
      for (int i = threadIdx.x; i < kShrinkRows * a.rank; i += kWarps * 32) {
        float* at = parts + i / a.rank * kPitch + i % a.rank;
        float h = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) h += at[w * kShrinkRows * kPitch];
        *at = h;
      }
      cluster_sync();
    }
    float* whole = parts + kWarps * kShrinkRows * kPitch;  // [row][padded]
    if (blockIdx.z == 0 || expanded != 0) {
      for (int i = threadIdx.x; i < kShrinkRows * a.padded; i += kWarps * 32) {
        const int n = i / a.padded, r = i % a.padded;
        if (!(rows >> n & 1)) continue;
        float h = 0.0f;
        if (r < a.rank) {
          const float* at = parts + n * kPitch + r;
          if (shares > 1) {
#pragma unroll 8
            for (int z = 0; z < shares; ++z) h += load_float(address_in(shared_address(at), z));
          } else {
#pragma unroll
            for (int w = 0; w < kWarps; ++w) h += at[w * kShrinkRows * kPitch];
          }
          h *= mixed >> n & 1 ? factor : factor * undo;
        }
        whole[i] = h;
        if (blockIdx.z != 0) continue;
        const uint32_t hi = pack_bf16(h, 0.0f) & 0xFFFFu;
        uint16_t* to = a.h + static_cast<uint64_t>(row0 + n) * 2 * a.padded + r;
        to[0] = static_cast<uint16_t>(hi);
        // an infinite or NaN h has no second part
        const float rest = h - bf16_value(hi);
        to[a.padded] = static_cast<uint16_t>(pack_bf16(isfinite(rest) ? rest : 0.0f, 0.0f));
      }
    }
    if (expanded != 0) {
      __syncthreads();
      // The cluster's warps share the features, 128 at a time, a lane 4 of them; for ranks above 16 also the rows, by eights.
      if constexpr (kSteps <= 2) {
        for (int f = ((blockIdx.z * kWarps + warp) * 32 + lane) * 4; f < a.out; f += shares * kWarps * kFeatures) {
          const uint16_t* factors = a.b + m * a.b_stride + static_cast<uint64_t>(f) * a.rank;
          Factors b[kSteps];
#pragma unroll
          for (int r = 0; r < kSteps; ++r) b[r].take(factors + r * 8, a.rank);
          for (uint32_t left = expanded; left != 0; left &= left - 1) {
            const int row = __ffs(left) - 1;
            float y[4] = {};
#pragma unroll
            for (int r = 0; r < kSteps; ++r) b[r].add(y, whole + row * a.padded + r * 8);
            *reinterpret_cast<float4*>(a.extra + static_cast<uint64_t>(row0 + row) * a.out + f) = make_float4(y[0], y[1], y[2], y[3]);
          }
        }
      } else {
        constexpr int kRows = 8, kAtOnce = 4;  // kAtOnce: eights of ranks whose B is under way together
        const int groups = (__popc(expanded) + kRows - 1) / kRows, tiles = (a.out + kFeatures - 1) / kFeatures;
        for (int u = blockIdx.z * kWarps + warp; u < tiles * groups; u += shares * kWarps) {
          const int f = u / groups * kFeatures + lane * 4;
          if (f >= a.out) continue;
          uint32_t left = expanded;
          for (int i = u % groups * kRows; i > 0; --i) left &= left - 1;
          int row[kRows];
          float y[kRows][4] = {};
#pragma unroll
          for (int i = 0; i < kRows; ++i) {
            row[i] = left != 0 ? __ffs(left) - 1 : -1;
            left &= left - 1;
          }
          const uint16_t* factors = a.b + m * a.b_stride + static_cast<uint64_t>(f) * a.rank;
          for (int r0 = 0; r0 < a.rank; r0 += 8 * kAtOnce) {
            Factors b[kAtOnce];
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r)
              if (r0 + r * 8 < a.rank) b[r].take(factors + r0 + r * 8, a.rank);
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r)
              if (r0 + r * 8 < a.rank)
#pragma unroll
                for (int i = 0; i < kRows; ++i)
                  if (row[i] >= 0) b[r].add(y[i], whole + row[i] * a.padded + r0 + r * 8);
          }
#pragma unroll
          for (int i = 0; i < kRows; ++i)
            if (row[i] >= 0)
              *reinterpret_cast<float4*>(a.extra + static_cast<uint64_t>(row0 + row[i]) * a.out + f) =
                  make_float4(y[i][0], y[i][1], y[i][2], y[i][3]);
        }
      }
    }
    // the sums have been read before they are written again, and before a block leaves
    if (shares > 1) cluster_sync();
    else __syncthreads();
  }
}

// --- rows that are named one by one ---------------------------------------------------------

// Copies the rows of x that slots name (zeros for those that do not exist) so that they lie in order, for tiles of
// many rows: there the copies one by one, four rows an instruction and 65 cycles each, took 1,581 us for a prompt whose
// product takes 480 so. A warp has a slot. 40 us for 8,191 rows of 5,120 bytes, read once and written four times (210 MB), 77 % of the
// copy bandwidth.
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

// --- the products -----------------------------------------------------------------------

// Tiles of up to 16 or 64 rows belong to a block each, those of up to 256 to a pair of blocks: 128 features and half
// of the rows' x are in each one's shared memory.
template <int kRows, bool kFp8>
struct Shape {
  static constexpr bool kPair = kRows == 256;
  static constexpr int kBlocks = kPair ? 2 : 1;
  static constexpr int kBox = kPair ? 64 : 16;  // rows of a copy of h
  // Converted codes of four stages, in the tensor memory behind two tiles' sums, or for pairs in shared memory.
  static constexpr int kSlots = 4;
  static constexpr bool kInTensor = kFp8 && !kPair;
  static constexpr int kSums = kInTensor ? 64 : 256;  // columns from one tile's sums to the next one's
  // Elements of a row in a stage, and how many times 64 of them. What an SM has under way is bound by requests,
  // so codes come 128 bytes at a time where the stages have room (a step's experts 56 us by 64 bytes).
  static constexpr int kDeep = kFp8 && !kPair ? 128 : 64, kHalves = kDeep / kDepth;
  static constexpr uint32_t kW = kFeatures * kDepth * 2, kX = kRows / kBlocks * kDepth * 2, kRaw = kFp8 ? kFeatures * kDeep : 0;
  static constexpr int kStages = kFp8 ? (kPair ? 5 : kRows == 64 ? 6 : 9) : (kPair ? 6 : kRows == 64 ? 8 : 10);
  static constexpr int kThreads = kFp8 ? 512 : 256;
  // FP8: 96 registers, so that some are left for the adapters' kernel beside it. (The kernels that are not gated spill 208 to
  // 220 bytes for it, around `expanded`.)
  static constexpr int kBound = kFp8 ? 640 : 256;
  // blocks or pairs that share a tile: what they send and receive has room in the stages
  static constexpr int kMostShares = kPair ? 3 : 8;
  static constexpr int kTeam = kInTensor ? 4 : 2;  // of the eight warps that convert codes, those on one part of a stage
};

constexpr int kPitch = kFeatures + 4;  // of a column of sums
constexpr int kStaged = 16;  // columns that pass through shared memory together

template <int kRows, bool kFp8>
struct Shared {
  using S = Shape<kRows, kFp8>;
  uint8_t w[S::kInTensor ? 1 : kFp8 ? S::kSlots : S::kStages][S::kInTensor ? 1024 : S::kW];
  uint8_t x[S::kStages][S::kX * S::kHalves];
  uint8_t raw[kFp8 ? S::kStages : 1][kFp8 ? S::kRaw : 16];
  float staged[2][kStaged][kPitch];
  uint64_t full[S::kStages], empty[S::kStages], ready[S::kSlots], free[S::kSlots], sum_full[2], sum_empty[2], drained;
  uint64_t open, joined, taken, turn;  // of blocks that share a tile
  int sums[32];
  uint32_t tensor;
  int failed;
  int notes[2][kRows];         // of a tile's columns
  int4 names[2][S::kPair ? 1 : kRows / 8];  // rows of the fours of each copying warp
  // Behind it: for each segment, the column tiles of those before it; then the first row of each, and the last one's end.
  __device__ __forceinline__ int* before() { return reinterpret_cast<int*>(this + 1); }
};
constexpr int segment_bytes(int segments) { return (2 * segments + 1) * 4; }

// 16 E4M3 codes as bf16 numbers, exactly. A code's bits, in their place, are those of a bf16 number 2^120 times
// smaller, denormals among them, so shifts and a product (with `unit`, two times 2^120) convert two. Only NaN
// differs: bits of `nan` 0x80808080 say that there is one.
__device__ __forceinline__ void bf16_of_codes(uint4 code, uint32_t unit, uint4 (&v)[2], uint32_t& nan) {
  const uint32_t in[4] = {code.x, code.y, code.z, code.w};
  uint32_t out[8];
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    nan |= (in[d] & 0x7F7F7F7Fu) + 0x01010101u;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const uint32_t w = __byte_perm(in[d], 0, p == 0 ? 0x4140 : 0x4342);  // each code in the lower byte of its half
      const uint32_t bits = (w * 256 & 0x80008000u) | (w * 16 & 0x07F007F0u);
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(out[2 * d + p]) : "r"(bits), "r"(unit), "r"(0x80008000u));
    }
  }
  v[0] = make_uint4(out[0], out[1], out[2], out[3]);
  v[1] = make_uint4(out[4], out[5], out[6], out[7]);
}

// x / (1 + exp(-x)), off by 2^-21 of it. With root = exp(-|x| / 2), in (0, 1], the denominator is within 1 .. 2 where the
// fast division is exact to 2^-22; for negative x it is x root (root / (1 + root^2)), in which nothing overflows and
// nothing underflows before the result does. (x by the fast division through 1 + exp(-x), of up to 2^127, lost all from -87.4 on,
// where silu still is 1e-36; the fast exponential 2^-18 at -80. experts_prompt 590 so, 600 this way, 680 by a true division.)
__device__ __forceinline__ float silu(float x) {
  const float root = expf(-0.5f * fabsf(x)), part = __fdividef(1.0f, fmaf(root, root, 1.0f)), f = x < 0.0f ? root : 1.0f;
  return (x * f) * (part * f);
}

// What all roles need of a call's tiles. A tile is kFeatures features a block (gated: 64 and the 64 that
// they are multiplied with) and up to kRows rows of a segment; its depth is `depth` stages. Tiles go to
// clusters in turn, and the blocks, or pairs, of a cluster have a share of the depth each.
struct Plan {
  int columns, features, depth;  // tiles, tiles, stages
  int tiles;
  int shares, share, place;  // of the depth, this block's, and its place in a pair
};

struct Item {
  int row0, rows, group, f0;
  int k0, k1;  // stages
};

template <int kRows, bool kFp8, bool kGated>
struct Walk {
  using S = Shape<kRows, kFp8>;
  const RowView& rows;
  const int* before;
  const int* begin;
  const Plan& plan;
  int at;

  __device__ __forceinline__ Walk(const RowView& r, Shared<kRows, kFp8>& s, const Plan& p)
      : rows(r), before(s.before()), begin(before + (r.joined ? 1 : r.segments)), plan(p), at(blockIdx.x / (p.shares * S::kBlocks)) {}

  __device__ __forceinline__ bool next(Item& item) {
    if (at >= plan.tiles) return false;
    const int tile = at;
    at += gridDim.x / (plan.shares * S::kBlocks);
    item.k0 = plan.depth * plan.share / plan.shares;
    item.k1 = plan.depth * (plan.share + 1) / plan.shares;
    const int band = tile / (kBand * plan.features);
    const int rest = tile - band * kBand * plan.features;
    const int wide = min(kBand, plan.columns - band * kBand);
    const int f = rest / wide;
    const int column = band * kBand + rest - f * wide;
    item.f0 = (f * S::kBlocks + plan.place) * (kGated ? kFeatures / 2 : kFeatures);
    int s = 0;
    if (!rows.joined) {
      int hi = rows.segments;  // the last with before[s] <= column
      while (hi - s > 1) {
        const int mid = (s + hi) / 2;
        if (before[mid] <= column) s = mid;
        else hi = mid;
      }
    }
    item.group = s;
    item.row0 = begin[s] + (column - before[s]) * kRows;
    item.rows = min(kRows, begin[s + 1] - item.row0);
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

// B h of four features of a row with adapter m.
__device__ __noinline__ float4 expanded(const ExpandView& e, uint64_t row, int m, int f) {
  const uint16_t* h = e.h + row * 2 * e.padded;
  const uint16_t* b = e.b + m * e.b_stride + static_cast<uint64_t>(f) * e.rank;
  float y[4] = {};
  for (int r = 0; r < e.rank; r += 8) {
    const uint4 p = *reinterpret_cast<const uint4*>(h + r), q = *reinterpret_cast<const uint4*>(h + e.padded + r);
    const uint32_t pw[4] = {p.x, p.y, p.z, p.w}, qw[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint4 o = *reinterpret_cast<const uint4*>(b + n * e.rank + r);
      const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        y[n] = fmaf(bf16_value(pw[d]) + bf16_value(qw[d]), bf16_value(ow[d]), y[n]);
        y[n] = fmaf(bf16_high(pw[d]) + bf16_high(qw[d]), bf16_high(ow[d]), y[n]);
      }
    }
  }
  return make_float4(y[0], y[1], y[2], y[3]);
}

template <int kRows, bool kFp8, bool kGated>
__global__ void __launch_bounds__(Shape<kRows, kFp8>::kBound, 1)
product_kernel(const MatrixView w, const RowView rows, const ExpandView expand, int* flag, int tries, bool early, int shares, int box,
               const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map,
               const __grid_constant__ CUtensorMap h_map, const __grid_constant__ CUtensorMap b_map) {
  using S = Shape<kRows, kFp8>;
  constexpr int kStages = S::kStages;
  constexpr bool kPair = S::kPair;
  extern __shared__ uint8_t dynamic[];
  Shared<kRows, kFp8>& sh = *reinterpret_cast<Shared<kRows, kFp8>*>(dynamic + ((1024 - (shared_address(dynamic) & 1023)) & 1023));
  const Watch watch{&sh.failed, tries};
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      barrier_init(&sh.full[i], 1);
      barrier_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < S::kSlots; ++i) {
      barrier_init(&sh.ready[i], S::kTeam * S::kBlocks);
      barrier_init(&sh.free[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(&sh.sum_full[i], 1);
      barrier_init(&sh.sum_empty[i], 4 * S::kBlocks);
    }
    if (shares > 1) {
      barrier_init(&sh.open, shares - 1);
      barrier_init(&sh.joined, 1);
      barrier_init(&sh.taken, shares - 1);
    }
    barrier_init(&sh.turn, 4);
    barrier_init(&sh.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.failed = 0;
  }
  if (warp == 0 && elected()) {
    fetch_map(&w_map);
    fetch_map(&x_map);
  }
  if (warp == 1) {
    if (kPair) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sh.tensor)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&sh.tensor)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  fence_before();
  if (kPair || shares > 1) cluster_sync();  // no block arrives at another's barriers before they are made
  else __syncthreads();
  fence_after();
  // Behind the kernel of the adapters' part, which waits for all that came before it and then lets
  // the next start, only what it makes has to be waited for.
  if (!early) wait_for_previous();

  const int outs = kGated ? w.out / 2 : w.out;
  constexpr int kWide = (kGated ? kFeatures / 2 : kFeatures) * S::kBlocks;
  Plan plan;
  plan.features = (outs + kWide - 1) / kWide;
  plan.depth = (w.in + S::kDeep - 1) / S::kDeep;
  // where each segment begins, and how many column tiles those before it have
  {
    const int segments = rows.joined ? 1 : rows.segments;
    int base = 0;
    for (int s0 = 0; s0 < segments; s0 += blockDim.x) {
      const int s = s0 + threadIdx.x;
      int begin = 0, end = 0;
      if (s < segments) segment_of(rows, s, begin, end);
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
#pragma unroll
      for (int i = 0; i < S::kThreads / 32; ++i) {
        if (i < warp) ahead += sh.sums[i];
        base += sh.sums[i];
      }
      if (s < segments) {
        sh.before()[s] = ahead + sum - n;
        sh.before()[segments + s] = begin;
        if (s + 1 == segments) sh.before()[segments + s + 1] = end;
      }
      __syncthreads();
    }
    // Starts that decrease could name rows many times over: no more column tiles than starts in order have.
    plan.columns = min(base, rows.rows / kRows + segments);
  }
  plan.tiles = plan.columns * plan.features;
  const int seat = blockIdx.x % (shares * S::kBlocks);  // in the cluster
  plan.shares = shares;
  plan.share = seat / S::kBlocks;
  plan.place = seat % S::kBlocks;
  const uint32_t first = seat - plan.place;  // of the pair
  const bool named = rows.index != nullptr && !rows.copied;  // rows of x are asked for one by one

  if (warp == 0) {
    // --- copies
    Walk<kRows, kFp8, kGated> walk(rows, sh, plan);
    Item item;
    uint32_t done = 0, items = 0;
    bool fine = true;
    // A pair's copies of bf16 are counted together, at the first block's barrier; codes are converted by each block.
    constexpr bool kTogether = kPair && !kFp8;
    auto expect = [&](uint32_t stage, uint32_t bytes) {
      if (!kTogether) barrier_expect(&sh.full[stage], bytes);
      else if (plan.place == 0) barrier_expect(&sh.full[stage], 2 * bytes);
    };
    auto copy3 = [&](const CUtensorMap* map, uint32_t to, uint32_t stage, int x, int y, int z) {
      if constexpr (kTogether) load_box_pair(map, to, address_in(shared_address(&sh.full[stage]), first), x, y, z);
      else load_box(map, to, &sh.full[stage], x, y, z);
    };
    auto copy2 = [&](const CUtensorMap* map, uint32_t to, uint32_t stage, int x, int y) {
      if constexpr (kTogether) load_box_pair(map, to, address_in(shared_address(&sh.full[stage]), first), x, y);
      else load_box(map, to, &sh.full[stage], x, y);
    };
    Item upcoming;
    bool more = walk.next(upcoming);
    for (; fine && more; ++items) {
      item = upcoming;
      // the stages hold what the cluster's blocks have of the tile before, and what others are still to take
      if (shares > 1 && items > 0 && !(fine = warp_wait(&sh.turn, (items - 1) & 1, watch) && warp_wait(&sh.taken, (items - 1) & 1, watch)))
        break;
      const int padded = ((item.rows + 15) & ~15) / S::kBlocks, row0 = item.row0 + plan.place * padded;  // here
      const int boxes = (padded + box - 1) / box;
      for (int k = item.k0; k < item.k1; ++k, ++done) {
        const uint32_t stage = done % kStages;
        if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
        const uint32_t x_to = shared_address(sh.x[stage]);
        if (elected()) {
          expect(stage, (kFp8 ? S::kRaw : S::kW) + (named ? padded : boxes * box) * S::kDeep * 2);
          const uint32_t w_to = kFp8 ? shared_address(sh.raw[stage]) : shared_address(sh.w[stage]);
          copy3(&w_map, w_to, stage, k * S::kDeep, item.f0, item.group);
          if (kGated) copy3(&w_map, w_to + (kFp8 ? S::kRaw : S::kW) / 2, stage, k * S::kDeep, item.f0 + outs, item.group);
          if (!named)
#pragma unroll
            for (int j = 0; j < S::kHalves; ++j)
              for (int i = 0; i < boxes; ++i)
                copy2(&x_map, x_to + j * S::kX + i * (box * kDepth * 2), stage, k * S::kDeep + j * kDepth, row0 + i * box);
        }
        __syncwarp();
        if (k == item.k0) more = walk.next(upcoming);
      }
      if (!fine || expand.h == nullptr || item.k1 < plan.depth) continue;
      if (early) wait_for_previous();
      const Runs runs(expand, item.row0, item.rows, lane);
      for (int i = 0, j, m; fine && runs.next(i, j, m); i = j) {
        const int run_rows = (j - i) * kBlock / S::kBlocks, run_row0 = item.row0 + i * kBlock + plan.place * run_rows;
        const int run_boxes = (run_rows + S::kBox - 1) / S::kBox;
        for (int e = 0; e < extras_of(expand.padded); ++e, ++done) {
          const Extra extra = extra_of(expand.padded, e);
          const uint32_t stage = done % kStages;
          if (!(fine = warp_wait(&sh.empty[stage], (done / kStages & 1) ^ 1, watch))) break;
          // in shared memory, the products of the slot's stage before; by that stage's barrier, since this warp may be several
          // turns of the slots ahead
          const uint32_t before = done - S::kSlots;
          if (kFp8 && kPair && done >= S::kSlots && !(fine = warp_wait(&sh.empty[before % kStages], before / kStages & 1, watch))) break;
          if (elected()) {
            expect(stage, S::kW + run_boxes * S::kBox * kDepth * 2);
            const uint32_t w_to = shared_address(S::kInTensor ? sh.raw[stage] : sh.w[kFp8 ? done % S::kSlots : stage]), x_to = shared_address(sh.x[stage]);
            copy3(&b_map, w_to, stage, extra.b_column, item.f0, m);
            for (int b = 0; b < run_boxes; ++b)
              copy2(&h_map, x_to + b * (S::kBox * kDepth * 2), stage, extra.column, run_row0 + b * S::kBox);
          }
          __syncwarp();
        }
      }
    }
    // No copy outlives the block: the stage has been filled, or, where the first block of a pair is told of that,
    // its products are done. After a wait that was given up a pair's copies may be counted nowhere (see the end).
    if (fine || !kTogether)
      for (uint32_t i = done > kStages ? done - kStages : 0; i < done; ++i)
        barrier_settle(kTogether && plan.place != 0 ? &sh.empty[i % kStages] : &sh.full[i % kStages], i / kStages & 1);
  } else if (warp == 1) {
    // --- products, issued by the first block of a pair
    Walk<kRows, kFp8, kGated> walk(rows, sh, plan);
    Item item;
    uint32_t done = 0, items = 0;
    const uint64_t plain = operand(0, 16);
    const uint32_t shape = product_of(0, false) + (kPair ? 128u >> 4 << 24 : 0u);
    const bool issues = plan.place == 0;
    bool fine = true;
    auto multiply_here = [&](uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
      if constexpr (kPair) multiply_pair(d, a, b, kind, add);
      else multiply(d, a, b, kind, add);
    };
    auto commit_here = [&](uint64_t* barrier) {
      if constexpr (kPair) commit_pair(barrier, 3u << first);
      else commit(barrier);
    };
    // Both blocks of a pair write converted codes, so there arrivals release and this wait acquires at the cluster's scope
    // (4,096 rows of 5,120 to 17,408 features 687 us either way, by 30 members 861 and 841; by one lane's wait 931, by a fence of the lane
    // that issues the products 1,118).
    auto stage_full = [&] {
      return kFp8 ? warp_wait<kPair>(&sh.ready[done % S::kSlots], done / S::kSlots & 1, watch)
                  : warp_wait(&sh.full[done % kStages], done / kStages & 1, watch);
    };
    auto stage_done = [&] {
      if (kFp8) commit_here(&sh.free[done % S::kSlots]);
      commit_here(&sh.empty[done % kStages]);
    };
    // of shared memory; adapters' B is where a stage's codes were
    auto w_of = [&] {
      return plain + (shared_address(S::kInTensor ? sh.raw[done % kStages] : sh.w[kFp8 ? done % S::kSlots : done % kStages]) >> 4);
    };
    auto x_of = [&] { return plain + (shared_address(sh.x[done % kStages]) >> 4); };
    while (fine && issues && walk.next(item)) {
      const uint32_t half = items & 1;
      const uint32_t sum = sh.tensor + half * S::kSums;
      if (!(fine = warp_wait(&sh.sum_empty[half], (items / 2 & 1) ^ 1, watch))) break;
      fence_after();
      const uint32_t kind = shape | static_cast<uint32_t>((item.rows + 15) / 16 * 2) << 17;
      for (int k = item.k0; k < item.k1; ++k, ++done) {
        if (!(fine = stage_full())) break;
        fence_after();
        const uint64_t a = w_of(), b = x_of();
        const uint32_t slot = sh.tensor + 128 + done % S::kSlots * 64;
        if (elected()) {
#pragma unroll
          for (int j = 0; j < S::kHalves; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool add = k > item.k0 || j > 0 || i > 0;
              if constexpr (S::kInTensor) multiply_from_tensor(sum, slot + j * 32 + i * 8, b + j * (S::kX >> 4) + i * 2, kind, add);
              else multiply_here(sum, a + i * 2, b + i * 2, kind, add);
            }
          stage_done();
        }
        __syncwarp();
      }
      if (fine && expand.h != nullptr && item.k1 == plan.depth) {
        if (early) wait_for_previous();
        const Runs runs(expand, item.row0, item.rows, lane);
        for (int i = 0, j, m; fine && runs.next(i, j, m); i = j) {
          const uint32_t run_kind = shape | static_cast<uint32_t>((j - i) * 2) << 17;
          for (int e = 0; e < extras_of(expand.padded); ++e, ++done) {
            const Extra extra = extra_of(expand.padded, e);
            if (!(fine = stage_full())) break;
            fence_after();
            const uint64_t a = w_of(), b = x_of();
            if (elected()) {
              for (int s = 0; s < extra.steps; ++s) {
                multiply_here(sum + i * kBlock, a + s * 2, b + s * 2, run_kind, true);
                if (extra.twice > 0) multiply_here(sum + i * kBlock, a + s * 2, b + extra.twice / 8 + s * 2, run_kind, true);
              }
              stage_done();
            }
            __syncwarp();
          }
        }
      }
      if (!fine) break;
      if (elected()) commit_here(&sh.sum_full[half]);
      __syncwarp();
      ++items;
    }
    __syncwarp();
    if (issues) {
      if (elected()) {  // the lane that issued the products: none outlives the tensor memory
        if constexpr (kPair) commit_pair(&sh.drained, 1u << first);
        else commit(&sh.drained);
      }
      __syncwarp();
      barrier_settle(&sh.drained, 0);
    }
  } else if (warp < 4) {
    // --- copies of rows that are named one by one, four at a time, half of them by each of two warps
    if (named) {
      Walk<kRows, kFp8, kGated> walk(rows, sh, plan);
      Item item;
      uint32_t done = 0;
      bool fine = true;
      int4* names = sh.names[warp - 2];
      for (uint32_t items = 0; fine && walk.next(item); ++items) {
        if (shares > 1 && items > 0 && !(fine = warp_wait(&sh.turn, (items - 1) & 1, watch) && warp_wait(&sh.taken, (items - 1) & 1, watch)))
          break;
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
#pragma unroll
              for (int j = 0; j < S::kHalves; ++j)
                gather_rows(&x_map, x_to + j * S::kX + i * (4 * kDepth * 2), &sh.full[stage], k * S::kDeep + j * kDepth, names[i - begin]);
          }
          __syncwarp();
        }
      }
      for (uint32_t i = done > kStages ? done - kStages : 0; i < done; ++i) barrier_settle(&sh.full[i % kStages], i / kStages & 1);
    }
  } else if (warp < 8) {
    // --- results: a thread reads a feature's lane, and writes four features of a row
    Walk<kRows, kFp8, kGated> walk(rows, sh, plan);
    Item item;
    uint32_t items = 0, chunks = 0;
    const int mine = warp - 4, feature = threadIdx.x - 128;
    // The four warps meet, as often in each whatever a wait has come to (through a barrier in shared memory a tile of
    // 256 rows took 27,000 cycles to write); and agree whether all of their waits were fine.
    auto meet = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    auto agree = [](bool fine) {
      uint32_t all;
      asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 q, %1, 0;\n bar.red.and.pred p, 1, 128, q;\n selp.b32 %0, 1, 0, p;\n}"
                   : "=r"(all)
                   : "r"(static_cast<uint32_t>(fine))
                   : "memory");
      return all != 0;
    };
    bool fine = true;
    if (early) wait_for_previous();
    for (; fine && walk.next(item); ++items) {
      const uint32_t half = items & 1;
      // what the columns are, looked up while their sums are made
      int* notes = sh.notes[half];
      for (int c = feature; c < item.rows; c += 128) {
        const int row = item.row0 + c;
        int note = kPlain;
        if (rows.index != nullptr && static_cast<unsigned>(rows.index[row]) >= static_cast<unsigned>(rows.x_rows)) note = kAbsent;
        if (expand.h != nullptr && expand.of_block[row / kBlock] == kMixed) note = max(expand.of_row[row], kPlain);
        notes[c] = note;
      }
      if (!(fine = agree(warp_wait(&sh.sum_full[half], items / 2 & 1, watch)))) break;
      fence_after();
      const uint32_t sum = sh.tensor + half * S::kSums + (static_cast<uint32_t>(mine) << 21);
      auto sum_read = [&] {
        if (lane != 0) return;
        if (kPair) barrier_signal_at(address_in(shared_address(&sh.sum_empty[half]), first));
        else barrier_arrive(&sh.sum_empty[half]);
      };
      float scale = kFp8 ? *(w.scale + item.group) : 1.0f;
      if (kFp8 && expand.h != nullptr && isinf(1.0f / scale)) scale = 1.0f;
      // What is added to the lane's features of four columns; those from `stop` on are left out.
      auto prepare = [&](int column, int stop, int (&note)[4], float4 (&more)[4]) {
        const int f = item.f0 + lane * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = column + i;
          note[i] = c < stop ? notes[c] : kOut;
          more[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (!kGated && expand.extra != nullptr && note[i] >= 0 && f < outs)
            more[i] = __ldcg(reinterpret_cast<const float4*>(expand.extra + static_cast<uint64_t>(item.row0 + c) * outs + f));
        }
      };
      // Sums of the lane's features of these columns to y: gated two features and the two that they are
      // multiplied with, else four.
      auto finish = [&](int column, const float4 (&z)[4], const int (&note)[4], float4 (&more)[4]) {
        const int f = item.f0 + (kGated ? lane * 2 : lane * 4);
        if (f >= outs) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (note[i] == kOut) continue;
          const uint64_t row = item.row0 + column + i;
          uint16_t* to = rows.y + row * rows.y_stride + f;
          if (kGated) {
            const uint32_t y = pack_bf16(silu(z[i].x * scale) * (z[i].z * scale), silu(z[i].y * scale) * (z[i].w * scale));
            *reinterpret_cast<uint32_t*>(to) = note[i] == kAbsent ? 0 : y;
          } else {
            if (expand.h != nullptr && expand.extra == nullptr && note[i] >= 0) more[i] = expanded(expand, row, note[i], f);
            const uint2 y = make_uint2(pack_bf16(fmaf(z[i].x, scale, more[i].x), fmaf(z[i].y, scale, more[i].y)),
                                       pack_bf16(fmaf(z[i].z, scale, more[i].z), fmaf(z[i].w, scale, more[i].w)));
            *reinterpret_cast<uint2*>(to) = note[i] == kAbsent ? make_uint2(0, 0) : y;
          }
        }
      };
      // Columns [lo, hi) are this block's to finish. Where others share the tile's depth, each sends it what it has of
      // these, and is sent what this one has of theirs, through the memory of the stages, which are empty now.
      int lo = 0, hi = item.rows;
      float* send = reinterpret_cast<float*>(&sh);  // of other blocks' columns, in their order
      const float* received = send;                  // of these, from each other block in turn
      // of two chunks of columns, each asked for two chunks ahead
      int note_a[4], note_b[4];
      float4 more_a[4], more_b[4];
      auto prepare_both = [&] {
        prepare(lo + mine * 4, hi, note_a, more_a);
        prepare(lo + kStaged + mine * 4, hi, note_b, more_b);
      };
      if (shares == 1) prepare_both();
      if (shares > 1) {
        const int width = ((item.rows + shares - 1) / shares + kStaged - 1) / kStaged * kStaged;
        auto from_of = [&](int q) { return min(q * width, item.rows); };
        lo = from_of(plan.share);
        hi = from_of(plan.share + 1);
        received = send + (item.rows - (hi - lo)) * kPitch;
        prepare_both();
        if (feature == 0) barrier_expect(&sh.joined, (shares - 1) * (hi - lo) * kPitch * 4);
        if (mine == 0 && lane < shares && lane != plan.share)
          barrier_signal_at(address_in(shared_address(&sh.open), lane * S::kBlocks + plan.place));
        for (int c = 0; c < item.rows; c += kStaged) {
          if (c >= lo && c < hi) continue;
          uint32_t r[kStaged];
          tensor_load(r, sum + c);
          tensor_loaded(r);
#pragma unroll
          for (int i = 0; i < kStaged; ++i)
            if (c + i < item.rows) send[(c < lo ? c + i : c + i - (hi - lo)) * kPitch + feature] = __uint_as_float(r[i]);
        }
        if (lo == hi) {
          fence_before();
          __syncwarp();
          sum_read();
        }
        fence_async();
        meet();
        if (mine == 0) {
          fine = warp_wait(&sh.open, items & 1, watch);
          if (fine && lane < shares && lane != plan.share) {
            const int q = lane, begin = from_of(q), wide = from_of(q + 1) - begin;
            const int place = (item.rows - wide) + (plan.share < q ? plan.share : plan.share - 1) * wide;  // there
            const uint32_t there = q * S::kBlocks + plan.place;
            if (wide > 0)
              copy_to_block(address_in(shared_address(send + place * kPitch), there),
                            shared_address(send + (q < plan.share ? begin : begin - (hi - lo)) * kPitch), wide * kPitch * 4,
                            address_in(shared_address(&sh.joined), there));
          }
          __syncwarp();
        }
        if (!(fine = agree(fine && warp_wait(&sh.joined, items & 1, watch)))) break;
        if (mine == 0 && lane < shares && lane != plan.share)
          barrier_signal_at(address_in(shared_address(&sh.taken), lane * S::kBlocks + plan.place));
      }
      auto write_chunk = [&](int c, int (&note)[4], float4 (&more)[4]) {
        uint32_t r[kStaged];
        tensor_load(r, sum + c);
        tensor_loaded(r);
        if (c + kStaged >= hi) {
          fence_before();
          __syncwarp();
          sum_read();
        }
        auto& staged = sh.staged[chunks & 1];
        float v[kStaged];
#pragma unroll
        for (int i = 0; i < kStaged; ++i) v[i] = __uint_as_float(r[i]);
        for (int q = 0; q < shares - 1; ++q) {
          const float* from = received + (q * (hi - lo) + c - lo) * kPitch + feature;
#pragma unroll
          for (int i = 0; i < kStaged; ++i)
            if (c + i < hi) v[i] += from[i * kPitch];
        }
#pragma unroll
        for (int i = 0; i < kStaged; ++i) staged[i][feature] = v[i];
        meet();
        float4 z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* from = staged[mine * 4 + i];
          if (kGated) {
            const float2 gate = *reinterpret_cast<const float2*>(from + lane * 2), up = *reinterpret_cast<const float2*>(from + 64 + lane * 2);
            z[i] = make_float4(gate.x, gate.y, up.x, up.y);
          } else {
            z[i] = *reinterpret_cast<const float4*>(from + lane * 4);
          }
        }
        finish(c + mine * 4, z, note, more);
        prepare(c + 2 * kStaged + mine * 4, hi, note, more);
        ++chunks;
      };
      for (int c = lo; c < hi; c += 2 * kStaged) {
        write_chunk(c, note_a, more_a);
        if (c + kStaged < hi) write_chunk(c + kStaged, note_b, more_b);
      }
      if (shares > 1) {
        fence_async();  // the stages are written by copies next
        warp_arrive(&sh.turn, lane);
      }
    }
  } else if (kFp8 && warp >= 8) {
    // --- codes to bf16: groups of warps take stages in turn, so that one's latency is beside others' work
    Walk<kRows, kFp8, kGated> walk(rows, sh, plan);
    Item item;
    uint32_t done = 0;
    const uint32_t unit = expand.h != nullptr && isinf(1.0f / *w.scale) ? 0 : 0x7B807B80u;  // 2^120, or all codes count as 0
    const uint32_t team = (warp - 8) / S::kTeam, member = (warp - 8) % S::kTeam;
    uint32_t part = team;  // the team's next one
    bool fine = true;
    while (fine && walk.next(item)) {
      const uint32_t codes = (done + item.k1 - item.k0);
      uint32_t end = codes;
      bool more = expand.h != nullptr && item.k1 == plan.depth;
      done += item.k1 - item.k0;
      for (;;) {
        if (part >= end) {
          if (!more) break;
          // the adapters' stages, which are bf16 already, once it is known how many there are
          more = false;
          if (early) wait_for_previous();
          const Runs runs(expand, item.row0, item.rows, lane);
          int extra = 0;
          for (int i = 0, j, m; runs.next(i, j, m); i = j) extra += extras_of(expand.padded);
          done += extra;
          end += extra;
          continue;
        }
        const uint32_t stage = part % kStages;
        auto slot_free = [&] { return warp_wait(&sh.free[part % S::kSlots], (part / S::kSlots & 1) ^ 1, watch); };
        // The stage's barrier cannot be a phase behind the one that is waited for: the products of kSlots stages before are
        // done, or, where the slot is waited for later, those of the slots and of the teams' turn before.
        static_assert(!kFp8 || S::kStages >= (S::kInTensor ? S::kSlots + 8 / S::kTeam : S::kSlots), "stages that a team may be ahead");
        if (!S::kInTensor || part >= codes)
          if (!(fine = slot_free())) break;
        if (!(fine = warp_wait(&sh.full[stage], part / kStages & 1, watch))) break;
        if (part < codes) {
          if constexpr (S::kInTensor) {
            // a thread has a row, which is a lane of the tensor memory; rows of 128 bytes of codes are swizzled
            const int at = (warp % 4) * 32 + lane;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint4 c[4], v[4][2];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                c[i] = *reinterpret_cast<const uint4*>(&sh.raw[stage][at * S::kDeep + (((half * 4 + i) ^ (at & 7)) * 16)]);
              uint32_t nan = 0;
#pragma unroll
              for (int i = 0; i < 4; ++i) bf16_of_codes(c[i], unit, v[i], nan);
              if (nan & 0x80808080u && unit != 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  v[i][0] = make_uint4(bf16_of_e4m3(c[i].x & 0xFFFFu), bf16_of_e4m3(c[i].x >> 16), bf16_of_e4m3(c[i].y & 0xFFFFu), bf16_of_e4m3(c[i].y >> 16));
                  v[i][1] = make_uint4(bf16_of_e4m3(c[i].z & 0xFFFFu), bf16_of_e4m3(c[i].z >> 16), bf16_of_e4m3(c[i].w & 0xFFFFu), bf16_of_e4m3(c[i].w >> 16));
                }
              uint32_t words[32];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const uint4 q = v[i / 2][i % 2];
                words[4 * i] = q.x;
                words[4 * i + 1] = q.y;
                words[4 * i + 2] = q.z;
                words[4 * i + 3] = q.w;
              }
              __syncwarp();
              if (half == 0) {
                if (!(fine = slot_free())) break;
                fence_after();
              }
              tensor_store32(sh.tensor + 128 + part % S::kSlots * 64 + half * 32 + (static_cast<uint32_t>(warp % 4) << 21), words);
            }
            if (!fine) break;
            tensor_stored();
            fence_before();
          } else {
            // 16 codes a lane and turn; eight lanes have four pieces of two rows, r and r ^ 5, which write no bank twice
            constexpr int kTurns = kFeatures * kDepth / 16 / 32 / S::kTeam;
            const int within = lane & 4 ? lane >> 3 ^ 5 : lane >> 3, piece = lane & 3;
            const int from = piece * 16;
            const uint8_t* codes_at = &sh.raw[stage][(member * 8 + within) * S::kDeep + from];
            uint8_t* to = &sh.w[part % S::kSlots][(member * 8 + within) * 128];
            const int place[2] = {((piece * 2) ^ within) * 16, ((piece * 2 + 1) ^ within) * 16};
            uint32_t nan = 0;
            constexpr int kAtOnce = 4;
#pragma unroll 1
            for (int i0 = 0; i0 < kTurns; i0 += kAtOnce) {
              uint4 c[kAtOnce];
#pragma unroll
              for (int i = 0; i < kAtOnce; ++i)
                c[i] = *reinterpret_cast<const uint4*>(codes_at + (i0 + i) * (S::kTeam * 8 * S::kDeep));
#pragma unroll
              for (int i = 0; i < kAtOnce; ++i) {
                uint4 v[2];
                bf16_of_codes(c[i], unit, v, nan);
#pragma unroll
                for (int h = 0; h < 2; ++h) *reinterpret_cast<uint4*>(to + (i0 + i) * (S::kTeam * 8 * 128) + place[h]) = v[h];
              }
            }
            if (nan & 0x80808080u && unit != 0) {
              for (int i = 0; i < kTurns; ++i) {
                const uint4 c = *reinterpret_cast<const uint4*>(codes_at + i * (S::kTeam * 8 * S::kDeep));
                const uint4 v[2] = {make_uint4(bf16_of_e4m3(c.x & 0xFFFFu), bf16_of_e4m3(c.x >> 16), bf16_of_e4m3(c.y & 0xFFFFu), bf16_of_e4m3(c.y >> 16)),
                                    make_uint4(bf16_of_e4m3(c.z & 0xFFFFu), bf16_of_e4m3(c.z >> 16), bf16_of_e4m3(c.w & 0xFFFFu), bf16_of_e4m3(c.w >> 16))};
                for (int h = 0; h < 2; ++h) *reinterpret_cast<uint4*>(to + i * (S::kTeam * 8 * 128) + place[h]) = v[h];
              }
            }
            fence_async();
          }
        }
        if (kPair) {
          __syncwarp();
          if (lane == 0) barrier_release_at(address_in(shared_address(&sh.ready[part % S::kSlots]), first));
        } else {
          warp_arrive(&sh.ready[part % S::kSlots], lane);
        }
        part += 8 / S::kTeam;
      }
    }
  }
  __syncwarp();
  // Copies between blocks that nobody waits for any more end within microseconds.
  if ((kPair || shares > 1) && sh.failed)
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  let_next_start();
  fence_before();
  if (kPair || shares > 1) cluster_sync();  // no block leaves while others read its sums or arrive at its barriers
  else __syncthreads();
  fence_after();
  if (threadIdx.x == 0 && sh.failed) *flag = 1;
  if (warp == 1) {
    if (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(sh.tensor) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tensor) : "memory");
  }
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
                   int columns, int most_rows, bool early, char* workspace, cudaStream_t stream, const char* call) {
  using S = Shape<kRows, kFp8>;
  auto kernel = product_kernel<kRows, kFp8, kGated>;
  using Sh = Shared<kRows, kFp8>;
  constexpr int kLeastBytes = static_cast<int>(sizeof(Sh)) + 1024, kBytes = kLeastBytes + segment_bytes(ES_MAX_EXPERTS);
  static_assert(kBytes <= 232448, "shared memory of a block");
  constexpr int kWidth = ((kRows + S::kMostShares - 1) / S::kMostShares + kStaged - 1) / kStaged * kStaged;
  static_assert((kRows + (S::kMostShares - 2) * kWidth) * kPitch * 4 <= offsetof(Sh, staged),
                "the stages hold what blocks that share a tile exchange");
  int device = 0;
  cudaGetDevice(&device);
  // Clusters of 1 to kMostShares shares that each device holds at once, of a kernel that has been given its
  // shared memory.
  static std::atomic<int> held[64][kMostShares + 1];
  int clusters[kMostShares + 1];
  if (device < 64 && held[device][1].load(std::memory_order_acquire) != 0) {
    for (int i = 1; i <= kMostShares; ++i) clusters[i] = held[device][i].load(std::memory_order_relaxed);
  } else {
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    for (int i = 1; i <= kMostShares && err == cudaSuccess; ++i) {
      clusters[i] = 0;
      if (i > S::kMostShares) continue;
      cudaLaunchConfig_t config{};
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = static_cast<unsigned>(i * S::kBlocks);
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      config.gridDim = dim3(static_cast<unsigned>(i * S::kBlocks));
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
  // How many blocks, or pairs, share a tile's depth: what takes least time, by the bytes of weights at the memory's rate
  // or a block's stages at its own, whichever is more, and the joins. 48 tiles of 40 stages (project_token): 16.0 us by
  // one block each, 14.1 by two, 20.4 by three (two rounds). 80 of 40 (experts_token): 16.2, 21.6 (two rounds), 18.6. 20 FP8
  // ones of 76 stages (project_step_e4m3): 61, 43, 36, 32 by four, 31 by six, 33 by eight (two rounds).
  const int outs = kGated ? w.out / 2 : w.out, wide = (kGated ? kFeatures / 2 : kFeatures) * S::kBlocks;
  const int64_t tiles = static_cast<int64_t>(columns) * ((outs + wide - 1) / wide);
  const int depth = (w.in + S::kDeep - 1) / S::kDeep;
  constexpr int kStageNs = S::kPair ? (kFp8 ? 400 : 270) : kFp8 ? 300 : 220;  // a pair's FP8 stages are the converters'
  const int64_t streamed = tiles * depth * (S::kBlocks * (kFp8 ? S::kRaw : S::kW)) / 6700;
  int shares = 1;
  int64_t best = INT64_MAX;
  for (int i = 1; i <= S::kMostShares && i <= depth; ++i) {
    if (clusters[i] < 1) continue;
    const int64_t rounds = (tiles + clusters[i] - 1) / clusters[i];
    const int64_t cost = std::max(streamed, rounds * ((depth + i - 1) / i) * kStageNs) + (i > 1 ? rounds * (1500 + 8 * most_rows) : 0);
    if (cost < best) {
      best = cost;
      shares = i;
    }
  }
  const int grid = static_cast<int>(std::min<int64_t>(tiles, clusters[shares])) * shares * S::kBlocks;
  // rows of a copy of x: all that a tile has where there is one column of tiles, else as many as most have
  const int here = (std::min(most_rows, kRows) + 15) / 16 * 16 / S::kBlocks;
  int box = kRows / S::kBlocks;
  if (rows.joined && columns == 1) box = here;
  else
    while (box >= 32 && box / 2 >= here) box /= 2;
  CUtensorMap x_map, h_map;
  es_status_t st;
  // without rows of x every slot is absent: what is read in their place does not matter
  if (rows.x_rows > 0 || rows.copied)
    st = map_rows(&x_map, rows.x, w.in, rows.copied ? rows.rows : rows.x_rows, rows.x_stride, rows.index != nullptr && !rows.copied ? 1 : box, call);
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
  attr[1].val.clusterDim.x = static_cast<unsigned>(shares * S::kBlocks);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3(static_cast<unsigned>(grid));
  config.blockDim = dim3(S::kThreads);
  config.dynamicSmemBytes = kLeastBytes + segment_bytes(rows.joined ? 1 : rows.segments);
  config.stream = stream;
  config.attrs = attr;
  config.numAttrs = shares * S::kBlocks > 1 ? 2 : 1;
  cudaError_t err = cudaLaunchKernelEx(&config, kernel, w, rows, expand, reinterpret_cast<int*>(workspace + ES_PROJECT_GAVE_UP),
                                       tries_of_a_wait.load(std::memory_order_relaxed), early, shares, box, w_map, x_map, h_map,
                                       expand.h != nullptr ? *b_map : x_map);
  const cudaError_t last = cudaGetLastError();
  if (err == cudaSuccess) err = last;
  return err != cudaSuccess ? cuda_fail(err, call) : ES_OK;
}

template <int kRows>
es_status_t launch_rows(const MatrixView& w, const CUtensorMap& w_map, bool fp8, bool gated, const RowView& rows, const ExpandView& expand,
                        const CUtensorMap* b_map, int columns, int most_rows, bool early, char* workspace, cudaStream_t stream, const char* call) {
  auto f = fp8 ? (gated ? launch<kRows, true, true> : launch<kRows, true, false>)
               : (gated ? launch<kRows, false, true> : launch<kRows, false, false>);
  return f(w, w_map, rows, expand, b_map, columns, most_rows, early, workspace, stream, call);
}

// Rows of a tile. One matrix of 5,120 by 7,168: 32 rows take 25.3 us by tiles of 16, 20.0 by tiles of 64 (whose fewer
// stages cost 16 rows nothing: 20.1, 19.9; those of 16 leave room where depth is short: 2,560 by 9,728 16.0, 16.3);
// 64 rows 21.2 by tiles of 64 and 21.8 by pairs; 96 rows 27.1 and 22.7; 192 rows 46.4 and 25.9. FP8 64 rows 23.0 and
// 25.9, 96 rows 35.0 and 27.6. Experts go by their mean, since their loads are not known here. With 0.4 to 1.6 times that each: 48 experts of
// 1,280 by 2,560 at 48 rows 59.8 and 61.4, at 64 rows 67.1 and 62.6; FP8 67.7 and 71.6, 81.8 and 74.2. Where one of 64 experts (2,560 by
// 2,560, gated) has three quarters of all rows, the rule's tiles of 64 are slower than pairs' would be: 178 and 157 at a mean of 40
// rows, 155 and 145 at 20; with a quarter 147 and 147, 135 and 145; even ones 137 and 141 at 40.
constexpr int kLeast = 16, kFew = 64, kMany = 256;
constexpr int kManyEach = 48;  // rows an expert above which tiles are of kMany
// B h of rows beside others' has room in the workspace (4 bytes a feature and row) up to here, which bounds what a workspace
// takes. Beyond it is made where results are written: nothing where prompts leave few mixed blocks (project_prompts), but slow for
// single rows: 5,120 to 17,408 features, rank 16, eight rows a member, 1,900 rows 303 us and 1,960 rows 641 (one a member 944); rank 64 708 and
// 2,169; 2,560 to 9,728, rank 40, 3,400 rows 449 and 3,460 rows 1,037.
constexpr uint64_t kMostExtra = uint64_t{128} << 20;
uint64_t extra_bytes(uint64_t rows, uint64_t out) { return rows * out * 4; }

uint64_t padded_rank(int rank) { return static_cast<uint64_t>(rank + 15) / 16 * 16; }
uint64_t rounded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// A launch of a grid of several axes that may begin early, in clusters of all of its z.
template <class... P, class... A>
cudaError_t launch_grid(void (*kernel)(P...), dim3 grid, int block, size_t shared, cudaStream_t stream, const A&... args) {
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = grid.z;
  cudaLaunchConfig_t config{};
  config.gridDim = grid;
  config.blockDim = dim3(static_cast<unsigned>(block));
  config.dynamicSmemBytes = shared;
  config.stream = stream;
  config.attrs = attr;
  config.numAttrs = grid.z > 1 ? 2 : 1;
  const cudaError_t err = cudaLaunchKernelEx(&config, kernel, P(args)...);
  const cudaError_t last = cudaGetLastError();
  return err != cudaSuccess ? err : last;
}

template <int kSteps>
cudaError_t launch_shrink(const ShrinkArgs& a, cudaStream_t stream) {
  constexpr int kBytes = (kShrinkWarps * (kSteps * 8 + 1) + (kSteps * 8 + 15) / 16 * 16) * kShrinkRows * 4;
  if (kBytes > 48 * 1024) {
    const cudaError_t err = cudaFuncSetAttribute(shrink_kernel<kSteps>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (err != cudaSuccess) {
      cudaGetLastError();
      return err;
    }
  }
  const int most = std::min(std::min(a.requests, a.rows), kShrinkRows);  // adapters that the rows of a block can have
  const int blocks = (a.rows + kShrinkRows - 1) / kShrinkRows;
  // Few blocks share their depth, so that its loads are all under way, and B's features (1,000 rows, 9,728 features, rank
  // 40: 80 us by four, 71 by eight); adapters of a block go to blocks of their own as far as there are likely so many, since
  // one without any costs a look at the requests.
  const int likely = std::min(std::min(most, 4), a.requests / blocks + 2);
  const dim3 grid = blocks <= 16   ? dim3(blocks, std::min(most, std::max(8, 48 / blocks)), 8)
                    : blocks <= 64 ? dim3(blocks, likely, 8)
                    : blocks <= 128 ? dim3(blocks, likely, 4)
                                    : dim3(blocks, 1, 2);
  return launch_grid(shrink_kernel<kSteps>, grid, kShrinkWarps * 32, kBytes, stream, a);
}

}  // namespace

void set_project_wait_tries(int tries) { tries_of_a_wait.store(tries < 0 ? kMostTries : tries, std::memory_order_relaxed); }

es_status_t map_matrices(CUtensorMap* map, const void* data, uint64_t in, uint64_t out, uint64_t groups, uint64_t row_stride,
                         uint64_t group_stride, bool fp8, int wide, int rows, const char* call) {
  EncodeTiled encode = nullptr;
  const es_status_t st = encode_tiled(&encode);
  if (st != ES_OK) return st;
  const cuuint64_t size = fp8 ? 1 : 2;
  const cuuint64_t dims[3] = {in, out, groups};
  const cuuint64_t strides[2] = {row_stride * size, group_stride * size};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(wide), static_cast<cuuint32_t>(rows), 1}, steps[3] = {1, 1, 1};
  const CUresult made = encode(map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(data),
                               dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               wide * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (made != CUDA_SUCCESS) return fail(ES_ERR_CUDA, "%s: cuTensorMapEncodeTiled returned %d", call, static_cast<int>(made));
  return ES_OK;
}

// Behind the head: with adapters h, the adapters of rows and blocks, and B h of up to kMostExtra bytes;
// without, rows that are copied in order.
uint64_t project_workspace_bytes(int rank, int rows, int in, int out) {
  const uint64_t n = rows;
  if (rank == 0) return kHead + (rows > kFew ? rounded(n * in * 2) : 0);
  return kHead + rounded(n * 4 * padded_rank(rank)) + 2 * rounded(n * 4) + rounded(std::min(extra_bytes(n, out), kMostExtra));
}

uint64_t project_workspace_head() { return kHead; }

es_status_t launch_project(const MatrixView& w, const CUtensorMap* w_maps, bool fp8, const AdapterView* adapters, const CUtensorMap* b_map,
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
    float* extra = std::min(rows.segments, rows.rows) > 1 && extra_bytes(n, w.out) <= kMostExtra
                       ? reinterpret_cast<float*>(behind + rounded(n * 4 * padded) + 2 * rounded(n * 4)) : nullptr;
    const ShrinkArgs a{rows.x, rows.start, adapter, adapters->a, adapters->scale, w.scale, h, of_row, of_block, adapters->b, extra,
                       rows.x_stride, adapters->a_stride, adapters->b_stride, rows.segments, rows.rows, adapters->count, adapters->rank,
                       padded, w.in, w.out};
    const int steps = (adapters->rank + 7) / 8;
    const cudaError_t err = steps <= 1   ? launch_shrink<1>(a, stream)
                            : steps <= 2 ? launch_shrink<2>(a, stream)
                            : steps <= 4 ? launch_shrink<4>(a, stream)
                            : steps <= 8 ? launch_shrink<8>(a, stream)
                                         : launch_shrink<16>(a, stream);
    if (err != cudaSuccess) return cuda_fail(err, call);
    expand = ExpandView{h, adapters->b, of_row, of_block, extra, adapters->b_stride, adapters->rank, padded};
  }
  const int tile = rows.rows > kFew ? kMany : rows.rows > kLeast ? kFew : kLeast;
  auto f = tile == kMany ? launch_rows<kMany> : tile == kFew ? launch_rows<kFew> : launch_rows<kLeast>;
  return f(w, w_maps[tile == kMany ? 0 : 2], fp8, false, rows, expand, b_map, (rows.rows + tile - 1) / tile, std::min(rows.rows, tile), adapters != nullptr,
           at, stream, call);
}

es_status_t launch_experts(const MatrixView& w, const CUtensorMap* w_maps, bool fp8, bool gated, const RowView& rows, void* workspace,
                           cudaStream_t stream, const char* call) {
  char* at = static_cast<char*>(workspace);
  const int tile = rows.rows > kFew && rows.rows / w.groups > kManyEach ? kMany : rows.rows > kLeast ? kFew : kLeast;
  RowView r = rows;
  bool early = false;
  if (tile == kMany && rows.index != nullptr) {
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
  auto f = tile == kMany ? launch_rows<kMany> : tile == kFew ? launch_rows<kFew> : launch_rows<kLeast>;
  return f(w, w_maps[(tile == kMany ? 0 : 2) + gated], fp8, gated, r, ExpandView{}, nullptr, segments * ((each + tile - 1) / tile), std::min(each, tile), early, at,
           stream, call);
}

}  // namespace esopt
