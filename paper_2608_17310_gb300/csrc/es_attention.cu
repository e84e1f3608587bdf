// es_attention: which kernel takes a call.
#include <algorithm>

#include "es_attention.cuh"
#include "es_rollout_internal.h"

namespace esopt {

uint64_t attention_workspace_bytes(int head_dim) {
  return kWorkspaceHead + std::max(few_rows_workspace_bytes(head_dim), many_rows_workspace_bytes(head_dim));
}

cudaError_t launch_attention(const CacheView& cache, const CUtensorMap* maps, bool fp8, int head_dim, const BatchView& batch,
                             const AttentionArgs& args, void* workspace, cudaStream_t stream) {
  uint32_t* counters = static_cast<uint32_t*>(workspace);
  char* rest = static_cast<char*>(workspace) + kWorkspaceHead;
  // Up to 16 rows a key head go to the kernel whose products are 8 or 16 rows wide. Measured at 12 and 16 rows
  // of 8 key heads of 128, here and in the kernel of many rows: one sequence of 500 tokens 12 and 19 us (FP8
  // 13 and 23), of 20,000 33 and 42 (33 and 60), 24 of up to 8,000 99 and 103 (94 and 162), 96 of up to 9,000
  // 328 and 310 (316 and 520); a single row of 777 tokens 8.4 and 21. Beyond 16 rows there is only the other.
  if (static_cast<int64_t>(batch.max_new) * args.group <= 16)
    return launch_few_rows(cache, fp8, head_dim, batch, args, rest, counters, stream);
  return launch_many_rows(cache, maps, fp8, head_dim, batch, args, rest, counters, reinterpret_cast<int*>(counters + kCounters), stream);
}

}  // namespace esopt
