// Shared by the rollout operators' host layer and kernels.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/es_rollout.h"

namespace esopt {

// A cache as the kernels see it. Offsets are 64-bit: a cache may hold more than 2^32
// elements.
struct CacheView {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  uint64_t page_stride;   // elements
  uint64_t scale_stride;  // floats
  int num_pages;
  int page_shift;  // page_size = 1 << page_shift
  int kv_heads;
};

// The sequences of a call. seq_len and start come from device memory and are taken
// through the functions below, which bound them.
struct BatchView {
  const int32_t* pages;
  const int32_t* seq_len;
  const int32_t* start;
  int pages_per_row;
  int sequences;
  int tokens;
  int max_new;
  int capacity;  // tokens a row of the page table reaches, at most 2^31 - 1
};

struct AppendArgs {
  const uint16_t* qkv;
  uint16_t* q_out;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  const float* rope;
  const int32_t* positions;
  uint64_t qkv_stride, q_out_stride, rope_rows;
  int q_heads, rotary_dim, interleaved;
  float eps;
};

struct AttentionArgs {
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const float* slopes;
  const int32_t* first;
  const int32_t* last;
  uint64_t q_stride, out_stride;
  int q_heads, group;  // group: query heads per key head
  int window;
  float scale, softcap;
  float factor;  // of a dot product: to a score in units of log 2, or to x / softcap where it is capped
};

#ifdef __CUDACC__
// Programmatic dependent launch: a kernel may be resident before the one ahead of it in its
// stream has ended, and touches no memory until that one has.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Launches a kernel that calls wait_for_previous before anything else.
template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), int grid, int block, size_t shared, cudaStream_t stream,
                         const A&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3(static_cast<unsigned>(grid));
  config.blockDim = dim3(static_cast<unsigned>(block));
  config.dynamicSmemBytes = shared;
  config.stream = stream;
  config.attrs = &attr;
  config.numAttrs = 1;
  const cudaError_t err = cudaLaunchKernelEx(&config, kernel, P(args)...);
  const cudaError_t last = cudaGetLastError();
  return err != cudaSuccess ? err : last;
}

__device__ __forceinline__ int sequence_length(const BatchView& b, int s) {
  return min(max(b.seq_len[s], 0), b.capacity);
}

// Rows [begin, begin + count) of the token arrays are sequence s's new tokens, the first
// of them at position `base` (negative where the sequence is shorter than its new tokens).
__device__ __forceinline__ void new_tokens(const BatchView& b, int s, int& begin, int& count, int& base) {
  int all;
  if (b.start == nullptr) {
    begin = s;
    all = s < b.tokens ? 1 : 0;
  } else {
    begin = min(max(b.start[s], 0), b.tokens);
    all = max(min(max(b.start[s + 1], 0), b.tokens) - begin, 0);
  }
  count = min(all, b.max_new);
  base = sequence_length(b, s) - all;
}

// The page of token p of sequence s, or -1 where the table names none.
__device__ __forceinline__ int page_of(const CacheView& c, const BatchView& b, int s, int p) {
  const int page = b.pages[static_cast<int64_t>(s) * b.pages_per_row + (p >> c.page_shift)];
  return static_cast<unsigned>(page) < static_cast<unsigned>(c.num_pages) ? page : -1;
}
#endif

// One launch each. fp8: the cache's storage type.
cudaError_t launch_append(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                          const AppendArgs& args, cudaStream_t stream);
cudaError_t launch_read(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                        uint16_t* k_out, uint16_t* v_out, cudaStream_t stream);
// maps: of the keys and the values, for TMA.
cudaError_t launch_attention(const CacheView& cache, const CUtensorMap* maps, bool fp8, int head_dim, const BatchView& batch,
                             const AttentionArgs& args, void* workspace, cudaStream_t stream);
uint64_t attention_workspace_bytes(int head_dim);
// For tests: tries after which the waits of the kernel of many rows are given up in calls from now on
// (0: at once; negative: as it was).
void set_wait_tries(int tries);

}  // namespace esopt
