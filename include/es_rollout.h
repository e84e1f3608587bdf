/*
 * es_rollout.h -- C ABI of the rollout operators: what a program needs of its
 * model's attention layer between es_perturb and es_restore (esopt.h), over a
 * paged key/value cache that belongs to the caller.
 *
 *   es_cache_append   norms of the query and key heads, their rotation, and the
 *                     keys and values written to the cache in its storage type
 *   es_attention      the new tokens' queries over the cached keys and values
 *   es_cache_read     cached keys and values back as bf16 rows
 *
 * ES evaluates members forward only, so the operators have no backward pass. A
 * cache holds keys and values of the parameters it was filled with: after an
 * es_perturb, es_restore or es_update its sequences start again.
 *
 * The conventions of esopt.h hold: device memory belongs to the caller, calls are
 * asynchronous on `stream`, run on the current device, return an es_status_t with
 * es_last_error() for the detail, neither allocate nor synchronise (so they can be
 * captured in a CUDA graph; the device arrays are read when the graph runs), and
 * give bit-identical results from call to call. Every buffer has to be device (or
 * managed) memory of the current device, 16-byte aligned except where said.
 *
 * What device arrays hold (lengths, page numbers, positions) cannot be checked on
 * the host. The kernels take every value: nothing is read or written through a
 * page number outside [0, num_pages) or past a row of the page table, and such
 * places hold no tokens.
 */
#ifndef ES_ROLLOUT_H_
#define ES_ROLLOUT_H_

#include <stdint.h>

#include "esopt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest number of sequences in one call. */
#define ES_MAX_SEQUENCES 4096

/*
 * A paged cache. Token s of a page, head h: the `head_dim` elements from
 *   k + page * page_stride + (h * page_size + s) * head_dim     (elements),
 * and the same in v; so one head's page is one contiguous block.
 *   dtype        ES_BF16, or ES_FP8_E4M3 with one fp32 scale per vector:
 *                element = scale * code, with scales of either sign, at
 *                k_scale + page * scale_stride + h * page_size + s
 *                (4-byte aligned); NULL for ES_BF16.
 *   num_pages    1 .. 2^31 - 1
 *   page_size    16, 32, 64 or 128 tokens
 *   kv_heads     1 .. 1024
 *   head_dim     64 or 128
 *   page_stride  elements from one page to the next, in k and in v: at least
 *                kv_heads * page_size * head_dim, a multiple of 16 bytes
 *                (larger where k and v, or layers, share one allocation)
 *   scale_stride floats from one page to the next, at least
 *                kv_heads * page_size; FP8 only
 */
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  uint64_t num_pages;
  uint64_t page_stride;
  uint64_t scale_stride;
  int page_size;
  int kv_heads;
  int head_dim;
  es_dtype_t dtype;
} es_cache_desc_t;

typedef struct es_cache* es_cache_t;

/*
 * Checks the description and keeps it, with what the kernels need of it (no device
 * memory is allocated; the buffers stay the caller's and have to outlive the
 * handle). The handle is immutable and may be used from any thread and stream.
 * Errors: ES_ERR_INVALID_ARG (NULL, a value outside the ranges above, buffers
 * that are not device memory of the current device, scales missing for FP8 or
 * given for bf16), ES_ERR_ALIGNMENT, ES_ERR_NO_MEMORY, ES_ERR_CUDA. On error *out
 * is set to NULL.
 */
es_status_t es_cache_create(const es_cache_desc_t* desc, es_cache_t* out);

/* Frees the handle, not the buffers. NULL is a no-op. */
es_status_t es_cache_destroy(es_cache_t cache);

/*
 * The sequences of a call and their new tokens (device arrays, 4-byte aligned).
 *   pages      [sequences] rows of `pages_per_row` page numbers: token p of
 *              sequence b is in slot p % page_size of page
 *              pages[b * pages_per_row + p / page_size]
 *   seq_len    [sequences] tokens of each sequence, its new tokens included. A
 *              length above pages_per_row * page_size (or 2^31 - 1024) counts as
 *              that, a negative one as 0.
 *   start      [sequences + 1], from 0 and not decreasing: the new tokens of
 *              sequence b are rows start[b] .. start[b + 1] - 1 of the call's
 *              token arrays. They are the sequence's last ones: row start[b] + i
 *              has position seq_len[b] - (start[b + 1] - start[b]) + i. NULL: one
 *              new token for each sequence, in order.
 *   sequences  1 .. ES_MAX_SEQUENCES
 *   tokens     rows of the token arrays, start[sequences]; 0 is a no-op
 *   max_new    an upper bound of the new tokens of one sequence, 1 .. tokens;
 *              the rest of a sequence that has more is left out
 */
typedef struct {
  const int32_t* pages;
  const int32_t* seq_len;
  const int32_t* start;
  int pages_per_row;
  int sequences;
  int tokens;
  int max_new;
} es_batch_t;

/*
 * es_cache_append: for each new token and each head of `qkv`
 *   q, k:  y = x * rsqrt(mean(x^2) + eps) * weight   (per head, over head_dim)
 *          then each pair (y_a, y_b) of the first rotary_dim elements turns into
 *          (y_a c - y_b s, y_b c + y_a s), (c, s) = rope[position][pair];
 *   v:     as it is.
 * Queries go to q_out as bf16, keys and values to the token's place in the cache.
 * Arithmetic is fp32, rounded once (to nearest even). In an FP8 cache a vector's
 * scale is max(max|x| / 448, 2^-126) over its finite elements, and its codes are
 * the E4M3 numbers nearest to x * (1 / scale) in fp32, ties to even, saturating at
 * +-448 (NaN stays NaN). The two fp32 roundings are within 2^-22 of x / scale, so
 * a code is not the nearest to x / scale only where that is as close as this to
 * midway between two codes.
 *   qkv         [tokens] rows of q_heads + 2 * kv_heads heads (queries, keys,
 *               values) of head_dim bf16, qkv_stride elements apart
 *   q_out       [tokens] rows of q_heads heads, q_out_stride elements apart; may
 *               be qkv itself, with its stride, and must not overlap it otherwise
 *   q_weight,   [head_dim] bf16; NULL: these heads are not normalised
 *   k_weight
 *   rope        [rope_rows][rotary_dim / 2] fp32 pairs (cos, sin), or NULL with
 *               rotary_dim 0. A token whose position has no row gets NaN in the
 *               first rotary_dim elements of its queries and keys.
 *   positions   [tokens] (4-byte aligned), or NULL: the position in the sequence.
 *               Only the rotation goes by it.
 *   rotary_dim  a multiple of 16 up to head_dim
 *   interleaved 0: pair i is elements (i, i + rotary_dim / 2); 1: (2i, 2i + 1)
 * q_heads is a multiple of kv_heads, up to 16 per key head. Strides are multiples
 * of 8. A token whose place does not exist writes no key or value. Two sequences
 * that share a page must not both write one slot.
 * Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_NONFINITE (eps),
 * ES_ERR_WRONG_DEVICE, ES_ERR_CUDA.
 */
typedef struct {
  const void* qkv;
  void* q_out;
  const void* q_weight;
  const void* k_weight;
  const float* rope;
  const int32_t* positions;
  uint64_t qkv_stride;
  uint64_t q_out_stride;
  uint64_t rope_rows;
  int q_heads;
  int rotary_dim;
  int interleaved;
  float eps;
} es_append_t;

es_status_t es_cache_append(es_cache_t cache, const es_batch_t* batch, const es_append_t* args,
                            void* stream);

/*
 * The cached keys and values of the batch's tokens (with start = the running sum of
 * seq_len: whole sequences) as [tokens][kv_heads][head_dim] bf16 rows, contiguous;
 * scale * code in fp32, rounded to bf16. A token whose place does not exist reads as 0. Either
 * output may be NULL.
 * Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_WRONG_DEVICE, ES_ERR_CUDA.
 */
es_status_t es_cache_read(es_cache_t cache, const es_batch_t* batch, void* k_out, void* v_out,
                          void* stream);

/*
 * es_attention: for each new token and each query head h (key head
 * h / (q_heads / kv_heads)), over the sequence's cached tokens j that the token sees:
 *   x_j = scale * (q . k_j);  x_j = softcap * tanh(x_j / softcap) where softcap > 0;
 *   x_j = x_j - slopes[h] * |position - j| where slopes is given;
 *   out = sum_j exp(x_j) v_j / sum_j exp(x_j),  lse = ln sum_j exp(x_j).
 * A token at position p sees j in [first, last): first = 0 and last = p + 1
 * (causal) unless given for it, first at least p - window + 1 where window > 0, and
 * never j >= seq_len. So packed documents pass each token's document start as
 * `first`, and a prefix that sees itself whole passes its end as `last`. A token that
 * sees nothing gets out = 0 and lse = -infinity. What a token does not see does not
 * reach it, NaN and infinities included. The new tokens' own keys are read from the
 * cache, so es_cache_append comes first.
 *   q, out     [tokens] rows of q_heads heads of head_dim bf16, q_stride and
 *              out_stride elements apart (multiples of 8); out must not
 *              overlap q
 *   lse        [tokens][q_heads] fp32 (4-byte aligned), or NULL
 *   slopes     [q_heads] fp32 (4-byte aligned), or NULL
 *   first,     [tokens] int32 (4-byte aligned), or NULL
 *   last
 *   softcap    0 for none, or at least 1e-6; above 2^100 it counts as 2^100
 *   workspace  es_attention_workspace() bytes of device memory, zero before its
 *              first use; every call leaves it ready for the next. One workspace
 *              serves calls of any batch one after another, and must not be used
 *              on two streams at once. Its 32-bit word at byte
 *              ES_ATTENTION_GAVE_UP stays 0: a kernel sets it where a wait of
 *              its own ran out (an error of the library). The outputs of
 *              that call, and of later ones with the workspace, are not to
 *              be used then until it has been zeroed again.
 * Scores, exponentials and sums are fp32; keys and values enter the products
 * exactly, and exp(x_j) (times an FP8 value's scale) rounded to bf16, or over FP8
 * caches with max_new * q_heads / kv_heads up to 16 to f16, where those below 2^-28
 * of a token's and head's largest are off by up to 2^-37 of it. (There the elements of
 * q too are f16 times a power of two: exact down to 2^-31 of the head's largest.)
 * Errors: ES_ERR_INVALID_ARG, ES_ERR_ALIGNMENT, ES_ERR_NONFINITE (scale, softcap),
 * ES_ERR_WRONG_DEVICE, ES_ERR_CUDA.
 */
typedef struct {
  const void* q;
  void* out;
  float* lse;
  const float* slopes;
  const int32_t* first;
  const int32_t* last;
  uint64_t q_stride;
  uint64_t out_stride;
  int q_heads;
  int window;
  float scale;
  float softcap;
} es_attention_t;

#define ES_ATTENTION_GAVE_UP 4096

es_status_t es_attention(es_cache_t cache, const es_batch_t* batch, const es_attention_t* args,
                         void* workspace, uint64_t workspace_bytes, void* stream);

/* Bytes of workspace that es_attention needs with this cache and q_heads (0 for a NULL
   cache or a q_heads that es_attention refuses). Independent of the batch. */
uint64_t es_attention_workspace(es_cache_t cache, int q_heads);

#ifdef __cplusplus
}
#endif

#endif /* ES_ROLLOUT_H_ */
