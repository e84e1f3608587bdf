/*
 * es_project.h -- C ABI of the rollouts' products whose rows choose their weights:
 * what a program needs, beside the attention layer (es_rollout.h), to roll many
 * members of a population out in one batch, and models with experts.
 *
 *   es_project          y = W x, one matrix for all rows, plus a low-rank adapter
 *                       per request beside it: members that differ by adapters
 *                       (whose tensors an ES plan perturbs) share one pass over W
 *   es_route            each token's experts, and the rows of each expert
 *   es_project_experts  products grouped by expert, with ragged row counts
 *   es_combine          the weighted sum of each token's rows
 *
 * ES evaluates members forward only, so the operators have no backward pass.
 * The conventions of es_rollout.h hold: device memory belongs to the caller, calls
 * are asynchronous on `stream`, run on the current device, return an es_status_t
 * with es_last_error() for the detail, neither allocate nor synchronise (so they can
 * be captured in a CUDA graph; the device arrays are read when the graph runs), and
 * give bit-identical results from call to call. Buffers have to be device (or
 * managed) memory of the current device, 16-byte aligned except where said.
 *
 * What device arrays hold (starts, adapters, rows, places) cannot be checked on the
 * host. The kernels take every value: nothing is read or written outside the
 * buffers that the arguments describe.
 */
#ifndef ES_PROJECT_H_
#define ES_PROJECT_H_

#include <stdint.h>

#include "es_rollout.h"
#include "esopt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest number of matrices in one es_weights_t, and of experts in es_route. */
#define ES_MAX_EXPERTS 1024

/* Largest number of rows (tokens, slots) of one call. */
#define ES_MAX_ROWS 16777216

/*
 * Matrices that lie in the caller's memory: element (o, i) of matrix g is element
 *   g * group_stride + o * row_stride + i
 * of data, o < out_features, i < in_features.
 *   dtype         ES_BF16, or ES_FP8_E4M3 with one scale a matrix: the value is
 *                 scale[g] * code
 *   scale         [groups] fp32 in device memory (4-byte aligned); NULL for ES_BF16.
 *                 In es_project with adapters a scale whose reciprocal is infinite
 *                 (below 2.94e-39) counts as 0. Sums are of codes and scaled in the
 *                 end, so one beyond 2^127 scale is infinite; so is an adapter's part
 *                 beyond that, but for scales outside 2^-32 .. 2^32.
 *   groups        1 .. ES_MAX_EXPERTS
 *   out_features  a multiple of 8, 8 .. 2^20
 *   in_features   a multiple of 8 (FP8: 16), up to 2^17
 *   strides       in elements, multiples of 16 bytes; row_stride at least
 *                 in_features; group_stride, where there are several matrices, at
 *                 least out_features * row_stride
 */
typedef struct {
  const void* data;
  const float* scale;
  uint64_t group_stride;
  uint64_t row_stride;
  int groups;
  int out_features;
  int in_features;
  es_dtype_t dtype;
} es_weights_desc_t;

typedef struct es_weights* es_weights_t;

/*
 * Checks the description and keeps it (no device memory is allocated; the buffers
 * stay the caller's, have to outlive the handle, and may change between calls, as
 * es_perturb changes them). The handle is immutable and may be used from any thread
 * and stream. Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_NO_MEMORY,
 * ES_ERR_CUDA. On error *out is set to NULL.
 */
es_status_t es_weights_create(const es_weights_desc_t* desc, es_weights_t* out);

/* Frees the handle, not the buffers. NULL is a no-op. */
es_status_t es_weights_destroy(es_weights_t weights);

/*
 * Low-rank adapters of one projection: adapter m adds scale[m] * B_m (A_m x).
 *   a      [count] matrices A of [rank][in_features] bf16, a_stride elements apart
 *   b      [count] matrices B of [out_features][rank] bf16, b_stride elements apart
 *   scale  [count] fp32 in device memory (4-byte aligned), or NULL: all 1
 *   count  1 .. 65536
 *   rank   a multiple of 8, 8 .. 128
 * in_features and out_features as in es_weights_desc_t (in_features a multiple of
 * 8); each A and B is contiguous, and strides are multiples of 8.
 */
typedef struct {
  const void* a;
  const void* b;
  const float* scale;
  uint64_t a_stride;
  uint64_t b_stride;
  int count;
  int rank;
  int out_features;
  int in_features;
} es_adapters_desc_t;

typedef struct es_adapters* es_adapters_t;

/* As es_weights_create and es_weights_destroy. */
es_status_t es_adapters_create(const es_adapters_desc_t* desc, es_adapters_t* out);
es_status_t es_adapters_destroy(es_adapters_t adapters);

/*
 * es_project: for each row i of request r, with adapter m = adapter[r],
 *   y_i = W x_i + B_m (scale[m] * (A_m x_i))
 *         (W x_i alone where m is not within 0 .. count - 1),
 * W with its scale. Sums are fp32, A x is kept to 2^-16 of itself, and a result is
 * rounded once. A row depends on its own adapter alone, whatever others hold; in which
 * order B h is summed, and so a result's last bit, also goes by whether the 16 rows
 * around it have one adapter, and by the number of rows.
 *   weights   of one matrix
 *   adapters  of the same sizes, or NULL: y = W x
 *   x         [rows] rows of in_features bf16, x_stride elements apart
 *   y         [rows] rows of out_features bf16, y_stride elements apart; must not
 *             overlap x
 *   start     [requests + 1] (4-byte aligned), from 0 and not decreasing: rows
 *             start[r] .. start[r + 1] - 1 are request r's. Rows from
 *             start[requests] on are neither read nor written. NULL: one row each
 *             (requests = rows).
 *   adapter   [requests] int32 (4-byte aligned); NULL without adapters
 *   rows      0 .. ES_MAX_ROWS; 0 is a no-op
 *   requests  1 .. ES_MAX_SEQUENCES where start or adapter is given, and where
 *             start is NULL not below rows
 *   workspace es_project_workspace() bytes of device memory, zero before its first
 *             use; every call leaves it ready for the next. One workspace serves
 *             any of these calls one after another, and must not be used on two
 *             streams at once. Its 32-bit word at byte ES_PROJECT_GAVE_UP stays 0: a
 *             kernel sets it where a wait of its own ran out (an error of the
 *             library). The outputs of that call, and of later ones with the
 *             workspace, are not to be used then until it has been zeroed again.
 * Strides are multiples of 8, at least a row.
 * Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_WRONG_DEVICE, ES_ERR_CUDA.
 */
typedef struct {
  const void* x;
  void* y;
  const int32_t* start;
  const int32_t* adapter;
  uint64_t x_stride;
  uint64_t y_stride;
  int rows;
  int requests;
} es_project_t;

#define ES_PROJECT_GAVE_UP 4096

es_status_t es_project(es_weights_t weights, es_adapters_t adapters, const es_project_t* args,
                       void* workspace, uint64_t workspace_bytes, void* stream);

/* Bytes of workspace that es_project (with these adapters or NULL) and
   es_project_experts need for up to `rows` rows or slots (0 for a NULL handle or rows
   outside 0 .. ES_MAX_ROWS). Grows with rows. Without adapters es_project, and without rows
   es_project_experts, use only its first ES_PROJECT_GAVE_UP + 256 bytes and take a workspace
   of that size. */
uint64_t es_project_workspace(es_weights_t weights, es_adapters_t adapters, int rows);

/*
 * es_project_experts: slot i, where start[g] <= i < start[g + 1], is a row of
 * matrix g:
 *   z = W_g x_{rows[i]}   (x_i where rows is NULL), W_g with its scale,
 *   y_i = z, or where gated y_i = silu(z_a) * z_b, z_a the first half of z and z_b
 *   the second, silu(v) = v / (1 + exp(-v)).
 * Sums, silu and the product are fp32, and a result is rounded once.
 *   x       [x_rows] rows of in_features bf16, x_stride elements apart
 *   y       [slots] rows of out_features (gated: out_features / 2, a multiple of 8)
 *           bf16, y_stride elements apart; must not overlap x
 *   start   [groups + 1] int32 (4-byte aligned), from 0 and not decreasing. Slots
 *           from start[groups] on are left as they were.
 *   rows    [slots] int32 (4-byte aligned), or NULL (x_rows = slots). A slot whose row is not
 *           within 0 .. x_rows - 1 gets zeros.
 *   slots   0 .. ES_MAX_ROWS; 0 is a no-op, and so is x_rows = 0 without rows
 *   gated   0 or 1
 *   workspace  as for es_project
 * Errors as es_project.
 */
typedef struct {
  const void* x;
  void* y;
  const int32_t* start;
  const int32_t* rows;
  uint64_t x_stride;
  uint64_t y_stride;
  int x_rows;
  int slots;
  int gated;
} es_project_experts_t;

es_status_t es_project_experts(es_weights_t weights, const es_project_experts_t* args,
                               void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * es_route: each token's `top` experts of largest score, largest first, equal
 * scores by the lower index; with p = softmax of the token's scores in fp32,
 *   weights[t][j] = p of the j-th, or with normalise p over the sum of the chosen p.
 * A score of -infinity or NaN is never chosen and has no part in p (+infinity counts
 * as the largest finite number): where fewer than `top` are left, the rest of the
 * token's entries are chosen = -1, weight = 0, place = -1. So a padded token whose
 * scores are all -infinity goes to no expert.
 * Pairs (token, j) are then put in order by expert, and by token within an expert:
 *   start   [experts + 1]: expert e's slots are start[e] .. start[e + 1] - 1
 *   rows    [tokens * top]: the token of each slot; entries from start[experts] on
 *           are left as they were
 *   places  [tokens][top]: the slot of each pair
 * which are es_project_experts' start and rows, and es_combine's places.
 *   scores      [tokens] rows of `experts` elements of dtype (ES_BF16 or ES_FP32),
 *               scores_stride elements apart (any, at least a row; aligned to the element)
 *   chosen, weights  [tokens][top] int32 and fp32
 * The outputs are 4-byte aligned.
 *   tokens      0 .. ES_MAX_ROWS, tokens * top at most ES_MAX_ROWS. 0 tokens: start alone is written.
 *   experts     1 .. ES_MAX_EXPERTS
 *   top         1 .. 32, at most experts
 *   normalise   0 or 1
 *   workspace   es_route_workspace() bytes of device memory; what it holds before
 *               does not matter. Not on two streams at once.
 * Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_CUDA.
 */
typedef struct {
  const void* scores;
  int32_t* chosen;
  float* weights;
  int32_t* start;
  int32_t* rows;
  int32_t* places;
  uint64_t scores_stride;
  int tokens;
  int experts;
  int top;
  int normalise;
  es_dtype_t dtype;
} es_route_t;

es_status_t es_route(const es_route_t* args, void* workspace, uint64_t workspace_bytes,
                     void* stream);

/* Bytes of workspace that es_route needs for up to `tokens` tokens (0 for arguments that it
   refuses). Grows with tokens. */
uint64_t es_route_workspace(int tokens, int experts, int top);

/*
 * es_combine: out_t = sum_j weights[t][j] * y_{places[t][j]} + add_t, in fp32 in
 * ascending j, rounded once. Places outside 0 .. slots - 1 have no part in the sum.
 *   y         [slots] rows of `features` bf16, y_stride elements apart
 *   places    [tokens][top] int32 (4-byte aligned)
 *   weights   [tokens][top] fp32 (4-byte aligned)
 *   add       [tokens] rows, add_stride apart, or NULL; may be out itself, with its
 *             stride, and must not overlap it otherwise
 *   out       [tokens] rows of bf16, out_stride apart; must not overlap y
 *   slots     0 .. ES_MAX_ROWS
 *   tokens    0 .. ES_MAX_ROWS; 0 is a no-op
 *   top       1 .. 32
 *   features  a multiple of 8, 8 .. 2^20; strides multiples of 8, at least a row
 * Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_CUDA.
 */
typedef struct {
  const void* y;
  const int32_t* places;
  const float* weights;
  const void* add;
  void* out;
  uint64_t y_stride;
  uint64_t add_stride;
  uint64_t out_stride;
  int slots;
  int tokens;
  int top;
  int features;
} es_combine_t;

es_status_t es_combine(const es_combine_t* args, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ES_PROJECT_H_ */
