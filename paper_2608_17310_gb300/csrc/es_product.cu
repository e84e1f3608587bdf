// es_project and es_project_experts.
#include "es_attention.cuh"
#include "es_project_internal.h"

namespace esopt {
namespace {

// The adapters' part of a product: h = scale (A x), already rounded to bf16, and B.
struct ExpandView {
  const uint16_t* h;  // [rows][rank]
  const uint16_t* b;
  const int32_t* start;
  const int32_t* adapter;
  uint64_t b_stride;
  int count, rank, requests;
};

__device__ __forceinline__ float bf16_value(uint16_t w) { return __uint_as_float(static_cast<uint32_t>(w) << 16); }

// Adapter of a row, or -1.
__device__ int adapter_of(const ExpandView& e, int row) {
  int r = row;
  if (e.start != nullptr) {
    int lo = 0, hi = e.requests;  // the last request that starts at or before the row
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (e.start[mid] <= row) lo = mid;
      else hi = mid;
    }
    r = lo;
  }
  const int m = e.adapter[r];
  return static_cast<unsigned>(m) < static_cast<unsigned>(e.count) ? m : -1;
}

constexpr int kTile = 64, kDepth = 16;

// A block has 64 rows of one segment and 64 features, a thread 4 x 4 of them. `factor`: of each
// matrix's results.
template <bool kFp8, bool kGated>
__global__ void __launch_bounds__(256)
product_kernel(const MatrixView w, const RowView rows, const float* factor, const ExpandView expand) {
  constexpr int kParts = kGated ? 2 : 1;
  __shared__ float xs[kDepth][kTile + 4], ws[kParts][kDepth][kTile + 4];
  __shared__ int found[4];
  wait_for_previous();
  if (threadIdx.x == 0) {
    int tile = blockIdx.x;
    found[0] = 0;
    for (int s = 0; s < (rows.joined ? 1 : rows.segments); ++s) {
      int begin, end, group;
      segment_of(rows, s, begin, end, group);
      if (static_cast<unsigned>(group) >= static_cast<unsigned>(w.groups)) continue;
      const int tiles = (end - begin + kTile - 1) / kTile;
      if (tile < tiles) {
        found[0] = 1;
        found[1] = begin + tile * kTile;
        found[2] = end;
        found[3] = group;
        break;
      }
      tile -= tiles;
    }
  }
  __syncthreads();
  if (!found[0]) return;
  const int row0 = found[1], end = found[2], group = found[3];
  const int outs = kGated ? w.out / 2 : w.out, f0 = blockIdx.y * kTile;
  const int tr = threadIdx.x / 16 * 4, tf = threadIdx.x % 16 * 4;
  float sum[kParts][4][4] = {};
  // the part of the tiles that this thread copies: row `at`, depth 4 * quarter ..
  const int at = threadIdx.x / 4, quarter = threadIdx.x % 4;
  int from = row0 + at < end ? row0 + at : -1;
  if (from >= 0 && rows.index != nullptr) from = rows.index[from];
  if (static_cast<unsigned>(from) >= static_cast<unsigned>(rows.x_rows)) from = -1;
  for (int k0 = 0; k0 < w.in; k0 += kDepth) {
    const int k = k0 + quarter * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xs[quarter * 4 + i][at] = from >= 0 && k + i < w.in ? bf16_value(rows.x[from * rows.x_stride + k + i]) : 0.0f;
#pragma unroll
      for (int p = 0; p < kParts; ++p) {
        float v = 0.0f;
        if (f0 + at < outs && k + i < w.in) {
          const uint64_t e = group * w.group_stride + (f0 + at + static_cast<uint64_t>(p) * outs) * w.row_stride + k + i;
          v = kFp8 ? bf16_value(static_cast<uint16_t>(bf16_of_e4m3(static_cast<const uint8_t*>(w.data)[e])))
                   : bf16_value(static_cast<const uint16_t*>(w.data)[e]);
        }
        ws[p][quarter * 4 + i][at] = v;
      }
    }
    __syncthreads();
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
#pragma unroll
      for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[p][i][j] = fmaf(xs[d][tr + i], ws[p][d][tf + j], sum[p][i][j]);
    }
    __syncthreads();
  }
  const float scale = (kFp8 ? w.scale[group] : 1.0f) * (factor != nullptr ? factor[group] : 1.0f);
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + tr + i;
    if (row >= end) continue;
    const int m = expand.h != nullptr ? adapter_of(expand, row) : -1;
    bool absent = false;
    if (rows.index != nullptr) absent = static_cast<unsigned>(rows.index[row]) >= static_cast<unsigned>(rows.x_rows);
    for (int j = 0; j < 4; ++j) {
      const int f = f0 + tf + j;
      if (f >= outs) continue;
      float y = sum[0][i][j] * scale;
      if (kGated) y = y / (1.0f + expf(-y)) * (sum[kParts - 1][i][j] * scale);
      if (m >= 0) {
        float more = 0.0f;
        for (int r = 0; r < expand.rank; ++r)
          more = fmaf(bf16_value(expand.h[static_cast<uint64_t>(row) * expand.rank + r]),
                      bf16_value(expand.b[m * expand.b_stride + static_cast<uint64_t>(f) * expand.rank + r]), more);
        y += more;
      }
      rows.y[row * rows.y_stride + f] = absent ? 0 : static_cast<uint16_t>(pack_bf16(y, 0.0f));
    }
  }
}

template <bool kFp8, bool kGated>
cudaError_t launch(const MatrixView& w, const RowView& rows, const float* factor, const ExpandView& expand, cudaStream_t stream) {
  const int outs = kGated ? w.out / 2 : w.out;
  const int tiles = (rows.rows + kTile - 1) / kTile + (rows.joined ? 0 : rows.segments);
  product_kernel<kFp8, kGated><<<dim3(tiles, (outs + kTile - 1) / kTile), 256, 0, stream>>>(w, rows, factor, expand);
  return cudaGetLastError();
}

constexpr uint64_t kHead = ES_PROJECT_GAVE_UP + 256;

}  // namespace

uint64_t project_workspace_bytes(int rank, int rows) { return kHead + static_cast<uint64_t>(rank) * rows * 2; }

cudaError_t launch_project(const MatrixView& w, bool fp8, const AdapterView* adapters, const int32_t* adapter, const RowView& rows,
                           void* workspace, cudaStream_t stream) {
  ExpandView expand{};
  if (adapters != nullptr) {
    uint16_t* h = reinterpret_cast<uint16_t*>(static_cast<char*>(workspace) + kHead);
    const MatrixView a{adapters->a, nullptr, adapters->a_stride, static_cast<uint64_t>(w.in), adapters->count, adapters->rank, w.in};
    RowView shrink = rows;
    shrink.y = h;
    shrink.y_stride = adapters->rank;
    shrink.group = adapter;
    shrink.joined = false;
    if (rows.start == nullptr) shrink.segments = rows.rows;
    const cudaError_t err = launch<false, false>(a, shrink, adapters->scale, ExpandView{}, stream);
    if (err != cudaSuccess) return err;
    expand = ExpandView{h, adapters->b, rows.start, adapter, adapters->b_stride, adapters->count, adapters->rank, rows.segments};
  }
  return fp8 ? launch<true, false>(w, rows, nullptr, expand, stream) : launch<false, false>(w, rows, nullptr, expand, stream);
}

cudaError_t launch_experts(const MatrixView& w, bool fp8, bool gated, const RowView& rows, void*, cudaStream_t stream) {
  if (gated) return fp8 ? launch<true, true>(w, rows, nullptr, ExpandView{}, stream) : launch<false, true>(w, rows, nullptr, ExpandView{}, stream);
  return fp8 ? launch<true, false>(w, rows, nullptr, ExpandView{}, stream) : launch<false, false>(w, rows, nullptr, ExpandView{}, stream);
}

}  // namespace esopt
