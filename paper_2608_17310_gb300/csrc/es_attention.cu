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
  if (static_cast<int64_t>(batch.max_new) * args.group <= 16)
    return launch_few_rows(cache, fp8, head_dim, batch, args, rest, counters, stream);
  return launch_many_rows(cache, maps, fp8, head_dim, batch, args, rest, counters, reinterpret_cast<int*>(counters + kCounters), stream);
}

}  // namespace esopt
