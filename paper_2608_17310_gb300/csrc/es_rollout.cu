// C-ABI host layer of the rollout operators: cache handles, argument checks, dispatch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/es_rollout.h"
#include "es_checks.h"
#include "es_rollout_internal.h"

struct es_cache {
  int device;
  es_dtype_t dtype;
  int page_size;
  int head_dim;
  esopt::CacheView view;
  CUtensorMap maps[2];  // of k and v
};

namespace {

using esopt::check_buffer;
using esopt::check_optional;
using esopt::check_stride;
using esopt::cuda_fail;
using esopt::fail;
using esopt::ok;

// Positions and the ends of tiles of keys stay within 32 bits.
constexpr int64_t kLongest = INT32_MAX - 1023;

// Caps above this one count as it, so that neither cap log2(e) nor scale / cap leaves fp32's normal
// numbers. Scores beyond a quarter of it are all that could tell.
constexpr float kLargestCap = 1.2676506002282294e30f;  // 2^100

// The checks that every operator makes of its cache and batch; ES_OK fills `view`.
es_status_t check_batch(es_cache_t cache, const es_batch_t* b, const char* call,
                        esopt::BatchView* view) {
  if (cache == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: cache is NULL", call);
  if (b == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: batch is NULL", call);
  if (b->sequences < 1 || b->sequences > ES_MAX_SEQUENCES)
    return fail(ES_ERR_INVALID_ARG, "%s: %d sequences; 1 .. %d are allowed", call, b->sequences,
                ES_MAX_SEQUENCES);
  if (b->pages_per_row < 1)
    return fail(ES_ERR_INVALID_ARG, "%s: pages_per_row is %d", call, b->pages_per_row);
  if (b->tokens < 0) return fail(ES_ERR_INVALID_ARG, "%s: %d tokens", call, b->tokens);
  if (b->tokens > 0 && (b->max_new < 1 || b->max_new > b->tokens))
    return fail(ES_ERR_INVALID_ARG, "%s: max_new %d is not within 1 .. %d tokens", call,
                b->max_new, b->tokens);
  if (b->start == nullptr && b->tokens > b->sequences)
    return fail(ES_ERR_INVALID_ARG, "%s: %d tokens of %d sequences need `start`", call, b->tokens,
                b->sequences);
  int device = -1;
  cudaError_t err = cudaGetDevice(&device);
  if (err != cudaSuccess) return cuda_fail(err, "cudaGetDevice");
  if (device != cache->device)
    return fail(ES_ERR_WRONG_DEVICE, "%s: the cache lives on device %d but device %d is current",
                call, cache->device, device);
  es_status_t st;
  if ((st = check_buffer(b->pages, 4, device, call, "pages")) != ES_OK) return st;
  if ((st = check_buffer(b->seq_len, 4, device, call, "seq_len")) != ES_OK) return st;
  if ((st = check_optional(b->start, 4, device, call, "start")) != ES_OK) return st;
  const int64_t capacity = static_cast<int64_t>(b->pages_per_row) * cache->page_size;
  *view = esopt::BatchView{b->pages, b->seq_len, b->start, b->pages_per_row, b->sequences,
                           b->tokens, b->max_new,
                           static_cast<int>(std::min(capacity, kLongest))};
  return ES_OK;
}

es_status_t check_heads(es_cache_t cache, int q_heads, const char* call) {
  const int kv = cache->view.kv_heads;
  if (q_heads < 1 || q_heads % kv != 0 || q_heads / kv > 16)
    return fail(ES_ERR_INVALID_ARG,
                "%s: %d query heads: 1 to 16 for each of the %d key heads are allowed", call,
                q_heads, kv);
  return ES_OK;
}

// Pages as [page][head and slot][element]; pages past the last one read as zeros. bf16 is read
// in boxes of one page of a head by 64 elements (128 bytes, swizzled), FP8 in boxes of up to
// 32 whole codes' vectors as they lie.
es_status_t make_map(CUtensorMap* map, void* base, const es_cache_desc_t& d, const char* call) {
  esopt::EncodeTiled encode = nullptr;
  const es_status_t st = esopt::encode_tiled(&encode);
  if (st != ES_OK) return st;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d.head_dim), static_cast<cuuint64_t>(d.kv_heads) * d.page_size, d.num_pages};
  const bool fp8 = d.dtype == ES_FP8_E4M3;
  const cuuint64_t size = fp8 ? 1 : 2;
  const cuuint64_t strides[2] = {d.head_dim * size, d.page_stride * size};
  const cuuint32_t box[3] = {fp8 ? static_cast<cuuint32_t>(d.head_dim) : 64u,
                             static_cast<cuuint32_t>(fp8 && d.page_size > 32 ? 32 : d.page_size), 1};
  const cuuint32_t steps[3] = {1, 1, 1};
  const CUresult made = encode(
      map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
      fp8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (made != CUDA_SUCCESS) return fail(ES_ERR_CUDA, "%s: cuTensorMapEncodeTiled returned %d", call, static_cast<int>(made));
  return ES_OK;
}

}  // namespace

extern "C" {

es_status_t es_cache_create(const es_cache_desc_t* d, es_cache_t* out) {
  const char* call = "es_cache_create";
  if (out == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: out is NULL", call);
  *out = nullptr;
  if (d == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: desc is NULL", call);
  if (d->dtype != ES_BF16 && d->dtype != ES_FP8_E4M3)
    return fail(ES_ERR_INVALID_ARG, "%s: a cache is ES_BF16 or ES_FP8_E4M3, not dtype %d", call,
                static_cast<int>(d->dtype));
  const bool fp8 = d->dtype == ES_FP8_E4M3;
  int shift = 4;
  while (shift < 7 && (1 << shift) != d->page_size) ++shift;
  if ((1 << shift) != d->page_size)
    return fail(ES_ERR_INVALID_ARG, "%s: page_size %d is not 16, 32, 64 or 128", call,
                d->page_size);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(ES_ERR_INVALID_ARG, "%s: head_dim %d is not 64 or 128", call, d->head_dim);
  if (d->kv_heads < 1 || d->kv_heads > 1024)
    return fail(ES_ERR_INVALID_ARG, "%s: kv_heads %d is not within 1 .. 1024", call, d->kv_heads);
  if (d->num_pages < 1 || d->num_pages > static_cast<uint64_t>(INT32_MAX))
    return fail(ES_ERR_INVALID_ARG, "%s: num_pages is not within 1 .. 2^31 - 1", call);
  const uint64_t tokens = static_cast<uint64_t>(d->kv_heads) * d->page_size;
  if (d->page_stride < tokens * d->head_dim || d->page_stride > (uint64_t{1} << 38))
    return fail(ES_ERR_INVALID_ARG, "%s: page_stride is less than a page or out of range", call);
  if (d->page_stride % (fp8 ? 16 : 8) != 0)
    return fail(ES_ERR_ALIGNMENT, "%s: page_stride is not a multiple of 16 bytes", call);
  if (!fp8 && (d->k_scale != nullptr || d->v_scale != nullptr))
    return fail(ES_ERR_INVALID_ARG, "%s: a bf16 cache has no scales", call);
  if (fp8 && (d->scale_stride < tokens || d->scale_stride > (uint64_t{1} << 40)))
    return fail(ES_ERR_INVALID_ARG, "%s: scale_stride is less than a page or out of range", call);
  if (d->k == nullptr || d->v == nullptr || (fp8 && (d->k_scale == nullptr || d->v_scale == nullptr)))
    return fail(ES_ERR_INVALID_ARG, "%s: a buffer is NULL", call);
  if (reinterpret_cast<uintptr_t>(d->k) % 16 != 0 || reinterpret_cast<uintptr_t>(d->v) % 16 != 0)
    return fail(ES_ERR_ALIGNMENT, "%s: k or v is not 16-byte aligned", call);
  int device = -1;
  cudaError_t err = cudaGetDevice(&device);
  if (err != cudaSuccess) return cuda_fail(err, "cudaGetDevice");
  es_status_t st;
  if ((st = check_buffer(d->k, 16, device, call, "k")) != ES_OK) return st;
  if ((st = check_buffer(d->v, 16, device, call, "v")) != ES_OK) return st;
  if (fp8) {
    if ((st = check_buffer(d->k_scale, 4, device, call, "k_scale")) != ES_OK) return st;
    if ((st = check_buffer(d->v_scale, 4, device, call, "v_scale")) != ES_OK) return st;
  }
  es_cache* c = new (std::nothrow) es_cache{};
  if (c == nullptr) return fail(ES_ERR_NO_MEMORY, "%s: host allocation failed", call);
  c->device = device;
  c->dtype = d->dtype;
  c->page_size = d->page_size;
  c->head_dim = d->head_dim;
  c->view = esopt::CacheView{d->k, d->v, d->k_scale, d->v_scale, d->page_stride, d->scale_stride,
                             static_cast<int>(d->num_pages), shift, d->kv_heads};
  if ((st = make_map(&c->maps[0], d->k, *d, call)) != ES_OK || (st = make_map(&c->maps[1], d->v, *d, call)) != ES_OK) {
    delete c;
    return st;
  }
  *out = c;
  return ok();
}

es_status_t es_cache_destroy(es_cache_t cache) {
  delete cache;
  return ok();
}

es_status_t es_cache_append(es_cache_t cache, const es_batch_t* batch, const es_append_t* a,
                            void* stream) {
  const char* call = "es_cache_append";
  esopt::BatchView b;
  es_status_t st = check_batch(cache, batch, call, &b);
  if (st != ES_OK) return st;
  if (a == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: args is NULL", call);
  if ((st = check_heads(cache, a->q_heads, call)) != ES_OK) return st;
  if (!std::isfinite(a->eps)) return fail(ES_ERR_NONFINITE, "%s: eps is not finite", call);
  if (a->eps < 0.0f) return fail(ES_ERR_INVALID_ARG, "%s: eps is negative", call);
  const int d = cache->head_dim;
  if (a->rotary_dim < 0 || a->rotary_dim > d || a->rotary_dim % 16 != 0)
    return fail(ES_ERR_INVALID_ARG, "%s: rotary_dim %d is not a multiple of 16 up to %d", call,
                a->rotary_dim, d);
  if ((a->rope == nullptr) != (a->rotary_dim == 0))
    return fail(ES_ERR_INVALID_ARG, "%s: rope and rotary_dim go together", call);
  if (a->interleaved != 0 && a->interleaved != 1)
    return fail(ES_ERR_INVALID_ARG, "%s: interleaved is %d", call, a->interleaved);
  if ((st = check_stride(a->qkv_stride, int64_t{d} * (a->q_heads + 2 * cache->view.kv_heads), call, "qkv_stride")) != ES_OK)
    return st;
  if ((st = check_stride(a->q_out_stride, int64_t{d} * a->q_heads, call, "q_out_stride")) != ES_OK) return st;
  if (b.tokens == 0) return ok();
  const int dev = cache->device;
  if ((st = check_buffer(a->qkv, 16, dev, call, "qkv")) != ES_OK) return st;
  if ((st = check_buffer(a->q_out, 16, dev, call, "q_out")) != ES_OK) return st;
  if ((st = check_optional(a->q_weight, 16, dev, call, "q_weight")) != ES_OK) return st;
  if ((st = check_optional(a->k_weight, 16, dev, call, "k_weight")) != ES_OK) return st;
  if ((st = check_optional(a->rope, 16, dev, call, "rope")) != ES_OK) return st;
  if ((st = check_optional(a->positions, 4, dev, call, "positions")) != ES_OK) return st;
  const esopt::AppendArgs args{static_cast<const uint16_t*>(a->qkv), static_cast<uint16_t*>(a->q_out),
                               static_cast<const uint16_t*>(a->q_weight),
                               static_cast<const uint16_t*>(a->k_weight), a->rope, a->positions,
                               a->qkv_stride, a->q_out_stride, a->rope_rows, a->q_heads,
                               a->rotary_dim, a->interleaved, a->eps};
  const cudaError_t err = esopt::launch_append(cache->view, cache->dtype == ES_FP8_E4M3, d, b, args,
                                               static_cast<cudaStream_t>(stream));
  if (err != cudaSuccess) return cuda_fail(err, call);
  return ok();
}

es_status_t es_cache_read(es_cache_t cache, const es_batch_t* batch, void* k_out, void* v_out,
                          void* stream) {
  const char* call = "es_cache_read";
  esopt::BatchView b;
  es_status_t st = check_batch(cache, batch, call, &b);
  if (st != ES_OK) return st;
  if (b.tokens == 0 || (k_out == nullptr && v_out == nullptr)) return ok();
  if ((st = check_optional(k_out, 16, cache->device, call, "k_out")) != ES_OK) return st;
  if ((st = check_optional(v_out, 16, cache->device, call, "v_out")) != ES_OK) return st;
  const cudaError_t err = esopt::launch_read(cache->view, cache->dtype == ES_FP8_E4M3,
                                             cache->head_dim, b, static_cast<uint16_t*>(k_out),
                                             static_cast<uint16_t*>(v_out),
                                             static_cast<cudaStream_t>(stream));
  if (err != cudaSuccess) return cuda_fail(err, call);
  return ok();
}

es_status_t es_attention(es_cache_t cache, const es_batch_t* batch, const es_attention_t* a,
                         void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* call = "es_attention";
  esopt::BatchView b;
  es_status_t st = check_batch(cache, batch, call, &b);
  if (st != ES_OK) return st;
  if (a == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: args is NULL", call);
  if ((st = check_heads(cache, a->q_heads, call)) != ES_OK) return st;
  if (!std::isfinite(a->scale) || !std::isfinite(a->softcap))
    return fail(ES_ERR_NONFINITE, "%s: scale or softcap is not finite", call);
  if (a->softcap < 0.0f || (a->softcap > 0.0f && a->softcap < 1e-6f) || a->window < 0)
    return fail(ES_ERR_INVALID_ARG, "%s: softcap or window is negative, or softcap below 1e-6", call);
  const int d = cache->head_dim;
  if ((st = check_stride(a->q_stride, int64_t{d} * a->q_heads, call, "q_stride")) != ES_OK) return st;
  if ((st = check_stride(a->out_stride, int64_t{d} * a->q_heads, call, "out_stride")) != ES_OK) return st;
  const uint64_t need = es_attention_workspace(cache, a->q_heads);
  if (workspace_bytes < need)
    return fail(ES_ERR_INVALID_ARG, "%s: the workspace has %llu bytes and needs %llu", call,
                static_cast<unsigned long long>(workspace_bytes),
                static_cast<unsigned long long>(need));
  if (b.tokens == 0) return ok();
  const int dev = cache->device;
  if ((st = check_buffer(a->q, 16, dev, call, "q")) != ES_OK) return st;
  if ((st = check_buffer(a->out, 16, dev, call, "out")) != ES_OK) return st;
  if ((st = check_optional(a->lse, 4, dev, call, "lse")) != ES_OK) return st;
  if ((st = check_optional(a->slopes, 4, dev, call, "slopes")) != ES_OK) return st;
  if ((st = check_optional(a->first, 4, dev, call, "first")) != ES_OK) return st;
  if ((st = check_optional(a->last, 4, dev, call, "last")) != ES_OK) return st;
  if ((st = check_buffer(workspace, 16, dev, call, "workspace")) != ES_OK) return st;
  const float cap = std::min(a->softcap, kLargestCap);
  const esopt::AttentionArgs args{static_cast<const uint16_t*>(a->q), static_cast<uint16_t*>(a->out),
                                  a->lse, a->slopes, a->first, a->last, a->q_stride, a->out_stride,
                                  a->q_heads, a->q_heads / cache->view.kv_heads, a->window,
                                  a->scale, cap,
                                  cap > 0.0f ? a->scale / cap : a->scale * 1.4426950408889634f};
  const cudaError_t err = esopt::launch_attention(cache->view, cache->maps, cache->dtype == ES_FP8_E4M3, d, b,
                                                  args, workspace, static_cast<cudaStream_t>(stream));
  if (err != cudaSuccess) return cuda_fail(err, call);
  return ok();
}

uint64_t es_attention_workspace(es_cache_t cache, int q_heads) {
  if (cache == nullptr || q_heads < 1 || q_heads % cache->view.kv_heads != 0 ||
      q_heads / cache->view.kv_heads > 16)
    return 0;
  return esopt::attention_workspace_bytes(cache->head_dim);
}

// Not in the header: for tests of given-up waits.
void es_attention_wait_tries(int tries) { esopt::set_wait_tries(tries); }

}  // extern "C"
