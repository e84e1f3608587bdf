// Shared by the host layer and the kernels of the products whose rows choose their weights.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/es_project.h"

namespace esopt {

// The matrices of a product: `groups` of them, element (o, i) of matrix g at
// data + g * group_stride + o * row_stride + i.
struct MatrixView {
  const void* data;
  const float* scale;  // of each matrix's codes; NULL for bf16
  uint64_t group_stride, row_stride;
  int groups, out, in;
};

struct AdapterView {
  const uint16_t* a;
  const uint16_t* b;
  const float* scale;
  uint64_t a_stride, b_stride;
  int count, rank;
};

// The rows of a product, in segments that go through one matrix each, the matrix of the segment's number. start comes from device
// memory and is taken through segment_of, which bounds it.
struct RowView {
  const uint16_t* x;
  uint16_t* y;
  const int32_t* start;  // NULL: one row a segment
  const int32_t* index;  // row of x of each row; NULL: its number
  uint64_t x_stride, y_stride;
  int segments, rows, x_rows;
  bool joined;  // all segments are one, through matrix 0
  bool copied;  // x holds the rows that index names already, in order
};

#ifdef __CUDACC__
// Rows [begin, end) of segment s.
__device__ __forceinline__ void segment_of(const RowView& r, int s, int& begin, int& end) {
  if (r.joined) {
    begin = 0;
    end = r.start != nullptr ? min(max(r.start[r.segments], 0), r.rows) : r.rows;
    return;
  }
  begin = r.start != nullptr ? min(max(r.start[s], 0), r.rows) : min(s, r.rows);
  end = r.start != nullptr ? min(max(r.start[s + 1], 0), r.rows) : min(s + 1, r.rows);
  end = max(begin, end);
}
#endif

// For TMA: matrices in boxes of `rows` rows by `wide` elements, swizzled where those are 128 bytes.
es_status_t map_matrices(CUtensorMap* map, const void* data, uint64_t in, uint64_t out, uint64_t groups, uint64_t row_stride,
                         uint64_t group_stride, bool fp8, int wide, int rows, const char* call);

// w_maps, b_map: of the matrices by 64 elements, in boxes of 128 rows and of 64, then the same by 128 bytes; and
// of the adapters' B by 64 elements in boxes of 128. These record their own errors.
es_status_t launch_project(const MatrixView& w, const CUtensorMap* w_maps, bool fp8, const AdapterView* adapters, const CUtensorMap* b_map,
                           const int32_t* adapter, const RowView& rows, void* workspace, cudaStream_t stream, const char* call);
es_status_t launch_experts(const MatrixView& w, const CUtensorMap* w_maps, bool fp8, bool gated, const RowView& rows, void* workspace,
                           cudaStream_t stream, const char* call);
uint64_t project_workspace_bytes(int rank, int rows, int in, int out);  // rank 0: no adapters
uint64_t project_workspace_head();  // what calls without adapters and without named rows use of it
// For tests: tries after which the products' waits are given up in calls from now on (0: at once;
// negative: as it was).
void set_project_wait_tries(int tries);

cudaError_t launch_route(const es_route_t& args, void* workspace, cudaStream_t stream);
uint64_t route_workspace_bytes(int tokens, int experts, int top);
cudaError_t launch_combine(const es_combine_t& args, cudaStream_t stream);

}  // namespace esopt
