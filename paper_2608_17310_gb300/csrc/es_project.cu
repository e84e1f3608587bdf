// C-ABI host layer of the products whose rows choose their weights: handles, argument checks, dispatch.
#include <cuda_runtime.h>

#include <new>

#include "../../include/es_project.h"
#include "es_checks.h"
#include "es_project_internal.h"

struct es_weights {
  int device;
  es_dtype_t dtype;
  esopt::MatrixView view;
  CUtensorMap maps[4];  // by 64 elements, in boxes of 128 rows and of 64, and by 128 bytes
};

struct es_adapters {
  int device;
  int out, in;
  esopt::AdapterView view;
  CUtensorMap map;  // of B
};

namespace {

using esopt::check_buffer;
using esopt::check_optional;
using esopt::check_stride;
using esopt::cuda_fail;
using esopt::fail;
using esopt::ok;

constexpr int kMostOut = 1 << 20, kMostIn = 1 << 17, kMostAdapters = 65536;

es_status_t check_features(int out, int in, int step, const char* call) {
  if (out < 8 || out > kMostOut || out % 8 != 0)
    return fail(ES_ERR_INVALID_ARG, "%s: out_features %d is not a multiple of 8 within 8 .. 2^20", call, out);
  if (in < step || in > kMostIn || in % step != 0)
    return fail(ES_ERR_INVALID_ARG, "%s: in_features %d is not a multiple of %d up to 2^17", call, in, step);
  return ES_OK;
}

es_status_t current_device(int* device) {
  const cudaError_t err = cudaGetDevice(device);
  return err != cudaSuccess ? cuda_fail(err, "cudaGetDevice") : ES_OK;
}

es_status_t check_device(int device, const char* call, const char* what) {
  int current = -1;
  const es_status_t st = current_device(&current);
  if (st != ES_OK) return st;
  if (current != device)
    return fail(ES_ERR_WRONG_DEVICE, "%s: the %s live on device %d but device %d is current", call, what, device, current);
  return ES_OK;
}

es_status_t check_rows(int rows, const char* call, const char* name) {
  if (rows < 0 || rows > ES_MAX_ROWS)
    return fail(ES_ERR_INVALID_ARG, "%s: %s %d is not within 0 .. %d", call, name, rows, ES_MAX_ROWS);
  return ES_OK;
}

es_status_t check_workspace(const void* workspace, uint64_t have, uint64_t need, int device, const char* call) {
  if (have < need)
    return fail(ES_ERR_INVALID_ARG, "%s: the workspace has %llu bytes and needs %llu", call,
                static_cast<unsigned long long>(have), static_cast<unsigned long long>(need));
  return check_buffer(workspace, 16, device, call, "workspace");
}

}  // namespace

extern "C" {

es_status_t es_weights_create(const es_weights_desc_t* d, es_weights_t* out) {
  const char* call = "es_weights_create";
  if (out == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: out is NULL", call);
  *out = nullptr;
  if (d == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: desc is NULL", call);
  if (d->dtype != ES_BF16 && d->dtype != ES_FP8_E4M3)
    return fail(ES_ERR_INVALID_ARG, "%s: matrices are ES_BF16 or ES_FP8_E4M3, not dtype %d", call, static_cast<int>(d->dtype));
  const bool fp8 = d->dtype == ES_FP8_E4M3;
  const unsigned step = fp8 ? 16 : 8;  // elements of 16 bytes
  es_status_t st = check_features(d->out_features, d->in_features, static_cast<int>(step), call);
  if (st != ES_OK) return st;
  if (d->groups < 1 || d->groups > ES_MAX_EXPERTS)
    return fail(ES_ERR_INVALID_ARG, "%s: %d groups; 1 .. %d are allowed", call, d->groups, ES_MAX_EXPERTS);
  if (d->row_stride < static_cast<uint64_t>(d->in_features) || d->row_stride > (uint64_t{1} << 30))
    return fail(ES_ERR_INVALID_ARG, "%s: row_stride is less than a row or out of range", call);
  if (d->groups > 1 && (d->group_stride < static_cast<uint64_t>(d->out_features) * d->row_stride ||
                        d->group_stride > (uint64_t{1} << 38)))
    return fail(ES_ERR_INVALID_ARG, "%s: group_stride is less than a matrix or out of range", call);
  if (d->row_stride % step != 0 || (d->groups > 1 && d->group_stride % step != 0))
    return fail(ES_ERR_ALIGNMENT, "%s: row_stride or group_stride is not a multiple of 16 bytes", call);
  if (fp8 != (d->scale != nullptr))
    return fail(ES_ERR_INVALID_ARG, "%s: scales go with FP8 matrices, and with no others", call);
  if (d->data == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: data is NULL", call);
  if (reinterpret_cast<uintptr_t>(d->data) % 16 != 0) return fail(ES_ERR_ALIGNMENT, "%s: data is not 16-byte aligned", call);
  int device = -1;
  if ((st = current_device(&device)) != ES_OK) return st;
  if ((st = check_buffer(d->data, 16, device, call, "data")) != ES_OK) return st;
  if ((st = check_optional(d->scale, 4, device, call, "scale")) != ES_OK) return st;
  es_weights* w = new (std::nothrow) es_weights{};
  if (w == nullptr) return fail(ES_ERR_NO_MEMORY, "%s: host allocation failed", call);
  w->device = device;
  w->dtype = d->dtype;
  const uint64_t whole = static_cast<uint64_t>(d->out_features) * d->row_stride;
  w->view = esopt::MatrixView{d->data, d->scale, d->groups > 1 ? d->group_stride : whole, d->row_stride, d->groups,
                              d->out_features, d->in_features};
  for (int i = 0; i < 4; ++i)
    if ((st = esopt::map_matrices(&w->maps[i], d->data, w->view.in, w->view.out, w->view.groups, w->view.row_stride,
                                  w->view.group_stride, fp8, fp8 && i >= 2 ? 128 : 64, 128 >> i % 2, call)) != ES_OK) {
      delete w;
      return st;
    }
  *out = w;
  return ok();
}

es_status_t es_weights_destroy(es_weights_t weights) {
  delete weights;
  return ok();
}

es_status_t es_adapters_create(const es_adapters_desc_t* d, es_adapters_t* out) {
  const char* call = "es_adapters_create";
  if (out == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: out is NULL", call);
  *out = nullptr;
  if (d == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: desc is NULL", call);
  es_status_t st = check_features(d->out_features, d->in_features, 8, call);
  if (st != ES_OK) return st;
  if (d->count < 1 || d->count > kMostAdapters)
    return fail(ES_ERR_INVALID_ARG, "%s: %d adapters; 1 .. %d are allowed", call, d->count, kMostAdapters);
  if (d->rank < 8 || d->rank > 128 || d->rank % 8 != 0)
    return fail(ES_ERR_INVALID_ARG, "%s: rank %d is not a multiple of 8 within 8 .. 128", call, d->rank);
  const uint64_t a = static_cast<uint64_t>(d->rank) * d->in_features, b = static_cast<uint64_t>(d->rank) * d->out_features;
  if (d->count > 1 && (d->a_stride < a || d->b_stride < b || d->a_stride > (uint64_t{1} << 38) || d->b_stride > (uint64_t{1} << 38)))
    return fail(ES_ERR_INVALID_ARG, "%s: a_stride or b_stride is less than a matrix or out of range", call);
  if (d->count > 1 && (d->a_stride % 8 != 0 || d->b_stride % 8 != 0))
    return fail(ES_ERR_ALIGNMENT, "%s: a_stride or b_stride is not a multiple of 8", call);
  if (d->a == nullptr || d->b == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: a or b is NULL", call);
  if (reinterpret_cast<uintptr_t>(d->a) % 16 != 0 || reinterpret_cast<uintptr_t>(d->b) % 16 != 0)
    return fail(ES_ERR_ALIGNMENT, "%s: a or b is not 16-byte aligned", call);
  int device = -1;
  if ((st = current_device(&device)) != ES_OK) return st;
  if ((st = check_buffer(d->a, 16, device, call, "a")) != ES_OK) return st;
  if ((st = check_buffer(d->b, 16, device, call, "b")) != ES_OK) return st;
  if ((st = check_optional(d->scale, 4, device, call, "scale")) != ES_OK) return st;
  es_adapters* m = new (std::nothrow) es_adapters{};
  if (m == nullptr) return fail(ES_ERR_NO_MEMORY, "%s: host allocation failed", call);
  m->device = device;
  m->out = d->out_features;
  m->in = d->in_features;
  m->view = esopt::AdapterView{static_cast<const uint16_t*>(d->a), static_cast<const uint16_t*>(d->b), d->scale,
                               d->count > 1 ? d->a_stride : a, d->count > 1 ? d->b_stride : b, d->count, d->rank};
  if ((st = esopt::map_matrices(&m->map, d->b, m->view.rank, m->out, m->view.count, m->view.rank, m->view.b_stride, false, 64, 128, call)) != ES_OK) {
    delete m;
    return st;
  }
  *out = m;
  return ok();
}

es_status_t es_adapters_destroy(es_adapters_t adapters) {
  delete adapters;
  return ok();
}

uint64_t es_project_workspace(es_weights_t weights, es_adapters_t adapters, int rows) {
  if (weights == nullptr || rows < 0 || rows > ES_MAX_ROWS) return 0;
  return esopt::project_workspace_bytes(adapters != nullptr ? adapters->view.rank : 0, rows, weights->view.in, weights->view.out);
}

es_status_t es_project(es_weights_t w, es_adapters_t m, const es_project_t* a, void* workspace, uint64_t workspace_bytes,
                       void* stream) {
  const char* call = "es_project";
  if (w == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: weights is NULL", call);
  if (a == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: args is NULL", call);
  const esopt::MatrixView& v = w->view;
  if (v.groups != 1) return fail(ES_ERR_INVALID_ARG, "%s: the weights hold %d matrices, not one", call, v.groups);
  es_status_t st;
  if ((st = check_rows(a->rows, call, "rows")) != ES_OK) return st;
  if ((st = check_stride(a->x_stride, v.in, call, "x_stride")) != ES_OK) return st;
  if ((st = check_stride(a->y_stride, v.out, call, "y_stride")) != ES_OK) return st;
  if ((m != nullptr) != (a->adapter != nullptr))
    return fail(ES_ERR_INVALID_ARG, "%s: adapters and adapter go together", call);
  if (a->start != nullptr || a->adapter != nullptr) {
    if (a->requests < 1 || a->requests > ES_MAX_SEQUENCES)
      return fail(ES_ERR_INVALID_ARG, "%s: %d requests; 1 .. %d are allowed", call, a->requests, ES_MAX_SEQUENCES);
    if (a->start == nullptr && a->rows > a->requests)
      return fail(ES_ERR_INVALID_ARG, "%s: %d rows of %d requests need `start`", call, a->rows, a->requests);
  }
  if (m != nullptr && (m->out != v.out || m->in != v.in))
    return fail(ES_ERR_INVALID_ARG, "%s: the adapters go from %d to %d features, the weights from %d to %d", call, m->in, m->out,
                v.in, v.out);
  if ((st = check_device(w->device, call, "weights")) != ES_OK) return st;
  if (m != nullptr && (st = check_device(m->device, call, "adapters")) != ES_OK) return st;
  if (a->rows == 0) return ok();
  const int dev = w->device;
  if ((st = check_buffer(a->x, 16, dev, call, "x")) != ES_OK) return st;
  if ((st = check_buffer(a->y, 16, dev, call, "y")) != ES_OK) return st;
  if ((st = check_optional(a->start, 4, dev, call, "start")) != ES_OK) return st;
  if ((st = check_optional(a->adapter, 4, dev, call, "adapter")) != ES_OK) return st;
  const uint64_t need = m != nullptr ? es_project_workspace(w, m, a->rows) : esopt::project_workspace_head();
  if ((st = check_workspace(workspace, workspace_bytes, need, dev, call)) != ES_OK) return st;
  const esopt::RowView rows{static_cast<const uint16_t*>(a->x), static_cast<uint16_t*>(a->y), a->start, nullptr,
                            a->x_stride, a->y_stride, a->requests, a->rows, a->rows, true, false};
  st = esopt::launch_project(v, w->maps, w->dtype == ES_FP8_E4M3, m != nullptr ? &m->view : nullptr, m != nullptr ? &m->map : nullptr,
                             a->adapter, rows, workspace, static_cast<cudaStream_t>(stream), call);
  return st == ES_OK ? ok() : st;
}

es_status_t es_project_experts(es_weights_t w, const es_project_experts_t* a, void* workspace, uint64_t workspace_bytes,
                               void* stream) {
  const char* call = "es_project_experts";
  if (w == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: weights is NULL", call);
  if (a == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: args is NULL", call);
  const esopt::MatrixView& v = w->view;
  if (a->gated != 0 && a->gated != 1) return fail(ES_ERR_INVALID_ARG, "%s: gated is %d", call, a->gated);
  if (a->gated && v.out % 16 != 0)
    return fail(ES_ERR_INVALID_ARG, "%s: a gated product of %d features: half of them is no multiple of 8", call, v.out);
  es_status_t st;
  if ((st = check_rows(a->slots, call, "slots")) != ES_OK) return st;
  if ((st = check_rows(a->x_rows, call, "x_rows")) != ES_OK) return st;
  if (a->rows == nullptr && a->x_rows != a->slots)
    return fail(ES_ERR_INVALID_ARG, "%s: %d slots of %d rows need `rows`", call, a->slots, a->x_rows);
  if ((st = check_stride(a->x_stride, v.in, call, "x_stride")) != ES_OK) return st;
  if ((st = check_stride(a->y_stride, a->gated ? v.out / 2 : v.out, call, "y_stride")) != ES_OK) return st;
  if ((st = check_device(w->device, call, "weights")) != ES_OK) return st;
  if (a->slots == 0) return ok();
  const int dev = w->device;
  if ((st = check_buffer(a->start, 4, dev, call, "start")) != ES_OK) return st;
  if ((st = check_optional(a->rows, 4, dev, call, "rows")) != ES_OK) return st;
  if (a->x_rows > 0 && (st = check_buffer(a->x, 16, dev, call, "x")) != ES_OK) return st;
  if ((st = check_buffer(a->y, 16, dev, call, "y")) != ES_OK) return st;
  const uint64_t need = a->rows != nullptr ? es_project_workspace(w, nullptr, a->slots) : esopt::project_workspace_head();
  if ((st = check_workspace(workspace, workspace_bytes, need, dev, call)) != ES_OK) return st;
  const esopt::RowView rows{static_cast<const uint16_t*>(a->x), static_cast<uint16_t*>(a->y), a->start, a->rows,
                            a->x_stride, a->y_stride, v.groups, a->slots, a->x_rows, false, false};
  st = esopt::launch_experts(v, w->maps, w->dtype == ES_FP8_E4M3, a->gated != 0, rows, workspace, static_cast<cudaStream_t>(stream), call);
  return st == ES_OK ? ok() : st;
}

uint64_t es_route_workspace(int tokens, int experts, int top) {
  if (tokens < 0 || experts < 1 || experts > ES_MAX_EXPERTS || top < 1 || top > 32 || top > experts ||
      static_cast<int64_t>(tokens) * top > ES_MAX_ROWS)
    return 0;
  return esopt::route_workspace_bytes(tokens, experts, top);
}

es_status_t es_route(const es_route_t* a, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* call = "es_route";
  if (a == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: args is NULL", call);
  if (a->dtype != ES_BF16 && a->dtype != ES_FP32)
    return fail(ES_ERR_INVALID_ARG, "%s: scores are ES_BF16 or ES_FP32, not dtype %d", call, static_cast<int>(a->dtype));
  if (a->experts < 1 || a->experts > ES_MAX_EXPERTS)
    return fail(ES_ERR_INVALID_ARG, "%s: %d experts; 1 .. %d are allowed", call, a->experts, ES_MAX_EXPERTS);
  if (a->top < 1 || a->top > 32 || a->top > a->experts)
    return fail(ES_ERR_INVALID_ARG, "%s: top %d is not within 1 .. 32 and the %d experts", call, a->top, a->experts);
  if (a->tokens < 0 || static_cast<int64_t>(a->tokens) * a->top > ES_MAX_ROWS)
    return fail(ES_ERR_INVALID_ARG, "%s: %d tokens of %d experts each are not within 0 .. %d slots", call, a->tokens, a->top, ES_MAX_ROWS);
  if (a->normalise != 0 && a->normalise != 1) return fail(ES_ERR_INVALID_ARG, "%s: normalise is %d", call, a->normalise);
  if (a->scores_stride < static_cast<uint64_t>(a->experts) || a->scores_stride > (uint64_t{1} << 40))
    return fail(ES_ERR_INVALID_ARG, "%s: scores_stride is less than a row or out of range", call);
  int dev = -1;
  es_status_t st = current_device(&dev);
  if (st != ES_OK) return st;
  if ((st = check_buffer(a->start, 4, dev, call, "start")) != ES_OK) return st;
  if (a->tokens > 0) {
    if ((st = check_buffer(a->scores, a->dtype == ES_BF16 ? 2 : 4, dev, call, "scores")) != ES_OK) return st;
    if ((st = check_buffer(a->chosen, 4, dev, call, "chosen")) != ES_OK) return st;
    if ((st = check_buffer(a->weights, 4, dev, call, "weights")) != ES_OK) return st;
    if ((st = check_buffer(a->rows, 4, dev, call, "rows")) != ES_OK) return st;
    if ((st = check_buffer(a->places, 4, dev, call, "places")) != ES_OK) return st;
  }
  if ((st = check_workspace(workspace, workspace_bytes, es_route_workspace(a->tokens, a->experts, a->top), dev, call)) != ES_OK) return st;
  const cudaError_t err = esopt::launch_route(*a, workspace, static_cast<cudaStream_t>(stream));
  if (err != cudaSuccess) return cuda_fail(err, call);
  return ok();
}

es_status_t es_combine(const es_combine_t* a, void* stream) {
  const char* call = "es_combine";
  if (a == nullptr) return fail(ES_ERR_INVALID_ARG, "%s: args is NULL", call);
  if (a->features < 8 || a->features > kMostOut || a->features % 8 != 0)
    return fail(ES_ERR_INVALID_ARG, "%s: features %d is not a multiple of 8 within 8 .. 2^20", call, a->features);
  if (a->top < 1 || a->top > 32) return fail(ES_ERR_INVALID_ARG, "%s: top %d is not within 1 .. 32", call, a->top);
  es_status_t st;
  if ((st = check_rows(a->slots, call, "slots")) != ES_OK) return st;
  if ((st = check_rows(a->tokens, call, "tokens")) != ES_OK) return st;
  if ((st = check_stride(a->y_stride, a->features, call, "y_stride")) != ES_OK) return st;
  if (a->add != nullptr && (st = check_stride(a->add_stride, a->features, call, "add_stride")) != ES_OK) return st;
  if ((st = check_stride(a->out_stride, a->features, call, "out_stride")) != ES_OK) return st;
  int dev = -1;
  if ((st = current_device(&dev)) != ES_OK) return st;
  if (a->tokens == 0) return ok();
  if (a->slots > 0 && (st = check_buffer(a->y, 16, dev, call, "y")) != ES_OK) return st;
  if ((st = check_buffer(a->places, 4, dev, call, "places")) != ES_OK) return st;
  if ((st = check_buffer(a->weights, 4, dev, call, "weights")) != ES_OK) return st;
  if ((st = check_optional(a->add, 16, dev, call, "add")) != ES_OK) return st;
  if ((st = check_buffer(a->out, 16, dev, call, "out")) != ES_OK) return st;
  const cudaError_t err = esopt::launch_combine(*a, static_cast<cudaStream_t>(stream));
  if (err != cudaSuccess) return cuda_fail(err, call);
  return ok();
}

// Not in the header: for tests of given-up waits.
void es_project_wait_tries(int tries) { esopt::set_project_wait_tries(tries); }

}  // extern "C"
