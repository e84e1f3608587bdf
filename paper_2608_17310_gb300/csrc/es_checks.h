// What the rollout operators' host layers share: statuses with their text, checks of buffers, TMA maps.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "es_internal.h"
#include "es_memcheck.h"

namespace esopt {

inline es_status_t fail(es_status_t st, const char* fmt, ...) {
  char text[400];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  return record_status(st, text);
}

inline es_status_t ok() { return record_status(ES_OK, ""); }

inline es_status_t cuda_fail(cudaError_t err, const char* what) {
  return fail(ES_ERR_CUDA, "%s: %s (%s)", what, cudaGetErrorName(err), cudaGetErrorString(err));
}

// A device buffer of the call: present, aligned and device memory.
inline es_status_t check_buffer(const void* p, unsigned align, int device, const char* call, const char* name) {
  if (p == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: %s is NULL", call, name);
  if (reinterpret_cast<uintptr_t>(p) % align != 0)
    return fail(ES_ERR_ALIGNMENT, "%s: %s is not %u-byte aligned", call, name, align);
  if (!is_device_memory(p, device))
    return fail(ES_ERR_INVALID_ARG, "%s: %s is not device memory of the current device %d", call, name, device);
  return ES_OK;
}

inline es_status_t check_optional(const void* p, unsigned align, int device, const char* call, const char* name) {
  return p == nullptr ? ES_OK : check_buffer(p, align, device, call, name);
}

// A row of `width` elements, `stride` elements apart, multiples of 8.
inline es_status_t check_stride(uint64_t stride, int64_t width, const char* call, const char* name) {
  if (stride < static_cast<uint64_t>(width) || stride > (uint64_t{1} << 40))
    return fail(ES_ERR_INVALID_ARG, "%s: %s %llu is less than a row or out of range", call, name,
                static_cast<unsigned long long>(stride));
  if (stride % 8 != 0)
    return fail(ES_ERR_ALIGNMENT, "%s: %s %llu is not a multiple of 8", call, name, static_cast<unsigned long long>(stride));
  return ES_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's cuTensorMapEncodeTiled, which the library is not linked against; looked up once.
inline es_status_t encode_tiled(EncodeTiled* out) {
  static std::atomic<EncodeTiled> kept{nullptr};
  *out = kept.load(std::memory_order_acquire);
  if (*out != nullptr) return ES_OK;
  void* found = nullptr;
  cudaDriverEntryPointQueryResult result;
  const cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &found, 12000, cudaEnableDefault, &result);
  if (err != cudaSuccess || found == nullptr)
    return cuda_fail(err != cudaSuccess ? err : cudaErrorNotSupported, "cuTensorMapEncodeTiled");
  *out = reinterpret_cast<EncodeTiled>(found);
  kept.store(*out, std::memory_order_release);
  return ES_OK;
}

}  // namespace esopt
