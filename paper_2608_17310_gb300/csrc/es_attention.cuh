// Device code that the attention kernels share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cfloat>

#include "es_rollout_internal.h"

namespace esopt {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}

// Two E4M3 codes as two bf16 numbers, exactly.
__device__ __forceinline__ uint32_t bf16_of_e4m3(uint32_t pair) {
  uint32_t h, w;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(pair)));
  asm("{\n .reg .f16 a, b;\n .reg .f32 x, y;\n mov.b32 {a, b}, %1;\n cvt.f32.f16 x, a;\n"
      " cvt.f32.f16 y, b;\n cvt.rn.bf16x2.f32 %0, y, x;\n}"
      : "=r"(w)
      : "r"(h));
  return w;
}

// Two E4M3 codes as two f16 numbers, exactly.
__device__ __forceinline__ uint32_t f16_of_e4m3(uint32_t pair) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(pair)));
  return h;
}

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t shared_address(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// Whether a word holds a bf16 infinity or NaN.
__device__ __forceinline__ bool has_nonfinite(uint32_t w) {
  return (w & 0x7F800000u) == 0x7F800000u || (w & 0x7F80u) == 0x7F80u;
}

// What row r of a (sequence, key head) sees: token, position, and [lo, hi) of the cache.
struct Row {
  int token, pos, lo, hi;
};

__device__ __forceinline__ Row row_of(const BatchView& b, const AttentionArgs& a, int begin, int count,
                                      int base, int length, int r) {
  const int i = r / a.group;
  Row row{-1, 0, 0, 0};
  if (i >= count) return row;
  row.token = begin + i;
  row.pos = base + i;
  row.lo = a.first != nullptr ? max(a.first[row.token], 0) : 0;
  if (a.window > 0) row.lo = max(row.lo, row.pos - a.window + 1);
  row.hi = min(a.last != nullptr ? a.last[row.token] : row.pos + 1, length);
  if (row.pos < 0 || row.hi <= row.lo) row.lo = row.hi = 0;
  return row;
}

// cap tanh(x / cap). With u = x / cap and z = u^2 the series x (1 - z / 3 + 2 z^2 / 15 - 17 z^3 / 315)
// where |u| <= 1 / 4, off by 62 z^4 / 2835 = 3.4e-7 of it at most, else cap (1 - 2 / (2^(2 u log2(e)) + 1)),
// off by 1e-7 cap: no more than 4e-7 of the score. (That form alone keeps nothing of scores that are
// small beside the cap: off by 0.09 at a cap of 1e6.)
__device__ __forceinline__ float capped(float x, float cap) {
  const float u = __fdividef(x, cap), z = u * u;
  if (fabsf(u) <= 0.25f) return x * fmaf(z, fmaf(z, fmaf(z, -17.0f / 315.0f, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
  return cap * (1.0f - __fdividef(2.0f, exp2_approx(u * (2.0f * kLog2e)) + 1.0f));
}

// The score of one key, in units of log 2, from scale q.k.
__device__ __forceinline__ float score_of(const AttentionArgs& a, float x, float slope, int distance) {
  if (a.softcap > 0.0f) x = capped(x, a.softcap);
  return (x - slope * static_cast<float>(abs(distance))) * kLog2e;
}

// Counts one more block as done, after what it wrote (ordered through a barrier of its threads)
// and before what it reads of the others'.
__device__ __forceinline__ uint32_t count_done(uint32_t* counter) {
  uint32_t before;
  asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
  return before;
}

// The workspace of es_attention: counters of the blocks that have finished their part of a
// unit, zero between calls; a flag that a kernel sets when it gave up a wait; what the
// kernels keep of a call.
constexpr int kCounters = 1024;
constexpr uint64_t kWorkspaceHead = kCounters * sizeof(uint32_t) + 256;
static_assert(kCounters * sizeof(uint32_t) == ES_ATTENTION_GAVE_UP, "the flag is behind the counters");

// es_attention of at most 16 rows per (sequence, key head), and of any number.
cudaError_t launch_few_rows(const CacheView& cache, bool fp8, int head_dim, const BatchView& batch,
                            const AttentionArgs& args, char* workspace, uint32_t* counters, cudaStream_t stream);
cudaError_t launch_many_rows(const CacheView& cache, const CUtensorMap* maps, bool fp8, int head_dim, const BatchView& batch,
                             const AttentionArgs& args, char* workspace, uint32_t* counters, int* flag, cudaStream_t stream);
uint64_t few_rows_workspace_bytes(int head_dim);
uint64_t many_rows_workspace_bytes(int head_dim);

}  // namespace esopt
