/*
 * vla_paged.h - attention over a paged key/value cache (libvla.so).
 *
 * For models that answer token by token, and for robots whose context outlives
 * one batch, keys and values live in pages of a shared pool: page t of request
 * r is pool page pages[r][t] and holds its tokens t * page_tokens and on. Per
 * layer a step appends its tokens' keys and values (vla_kv_append: rotates
 * queries and keys by their positions on the way) and attends over what the
 * cache then holds (vla_paged_attention); where all requests begin with the
 * same context on the same pages, that part is read once for the batch
 * (vla_shared_attention).
 *
 * Conventions are those of vla.h: device buffers are the caller's, calls
 * validate, enqueue on `stream` and return, results are deterministic, on an
 * error nothing is enqueued and vla_last_error() says why. Work runs on the
 * pool's device, whatever device is current; all buffers must be on it. Calls
 * may be captured into graphs: they allocate nothing and read no device memory
 * on the host. The lengths and pages of a batch are read on the device, so a
 * captured step can be replayed after they changed, within the stated bounds.
 * Two calls that overlap need workspaces of their own and may not write the
 * same cache slots or output rows.
 *
 * Numeric policy: products of bf16 values are exact and summed in fp32; scores,
 * softmax statistics and outputs are fp32 until the one rounding of the result;
 * probabilities are rounded to bf16 before they weigh bf16 values (relative to
 * the row's largest, so an output is off by at most 2^-8 of its row's largest
 * value). Weights are at most 1 until the sum over the values is divided by
 * theirs: values below 2^128 / (keys that the token sees) do not overflow.
 * Rotation angles are reduced in fp64, rotation is fp32. VLA_F32 calls
 * compute in fp32 throughout.
 */
#ifndef VLA_PAGED_H
#define VLA_PAGED_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "vla.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * One layer's pool of pages. Element d of head h of slot s of page p lies at
 * p * page_stride + h * head_stride + s * token_stride + d (elements) of k and
 * of v. Bases are 16-byte aligned, strides are multiples of 16 bytes (a stride
 * along an extent of 1 is not looked at).
 */
typedef struct {
  int device;
  int dtype;                 /* VLA_F32 | VLA_BF16; q, the new k and v and o have it too */
  int n_kv, head_dim;        /* head_dim a multiple of 8 in [8, 256] */
  int page_tokens;           /* a power of two in [1, 65536] */
  int n_pages;
  void *k, *v;
  int64_t page_stride, head_stride, token_stride;
} vla_kv_pool;

/*
 * A ragged batch. Request r brings the tokens start[r] .. start[r + 1] - 1 of
 * the token buffers, which are the last of the kv_len[r] tokens it then has:
 * token i of n has place kv_len[r] - n + i in the cache. Requests may bring no
 * token. Rows of the token buffers from start[n_req] on are neither read nor
 * written. start and kv_len ascend / lie within the bounds; kernels stay
 * within the buffers where they do not (the results of such requests are
 * unspecified). An entry of `pages` outside [0, n_pages) is a page that is not
 * there: nothing is appended to it and no one sees its keys (pages that a
 * window has left behind may be given back and marked -1). Requests may share
 * pages; two tokens that one call appends may not share a slot.
 */
typedef struct {
  int n_req;                 /* >= 1 */
  int n_tok;                 /* rows of the token buffers, >= start[n_req] */
  int max_new;               /* >= the tokens that any request brings */
  int max_len;               /* >= kv_len of any request */
  const int32_t* start;      /* device [n_req + 1] */
  const int32_t* kv_len;     /* device [n_req] */
  const int32_t* pages;      /* device [n_req][pages_stride] */
  int pages_stride;          /* entries a request; max_len fits into them */
} vla_ragged;

/*
 * Append: k and v of the batch's tokens go to their cache slots, k rotated;
 * with q, the rotated q goes to q_out (which may be q itself).
 * Rotation: element pairs (f, f + rot / 2), f < rot / 2, with rot / 2 the sum
 * of the sections; pair f of section a turns by positions[token][a] *
 * rope_base^(-2 f / rot) (sections follow one another in f: time, row and
 * column of image tokens, say). Elements from rot on pass through. n_axes 0:
 * nothing is rotated. positions NULL (n_axes 1): the token's place.
 */
typedef struct {
  const void *k, *v;         /* element (token, head, d) at token * tok_stride + head * head_stride + d */
  int64_t k_tok_stride, k_head_stride, v_tok_stride, v_head_stride;
  int n_q;                   /* query heads; 0: no q */
  const void* q;
  void* q_out;
  int64_t q_tok_stride, q_head_stride, qo_tok_stride, qo_head_stride;
  int n_axes;                /* 0 .. 3 */
  int sections[3];           /* pairs that each axis turns; rot = 2 * their sum, a multiple of 16, <= head_dim */
  const int32_t* positions;  /* device [n_tok][n_axes], or NULL */
  float rope_base;           /* > 1 (n_axes > 0) */
} vla_append_args;

vla_status vla_kv_append(const vla_kv_pool* pool, const vla_ragged* batch, const vla_append_args* args,
                         hipStream_t stream);

/*
 * o = softmax(cap(scale q k^T)) v for every token and query head of the batch
 * (head h uses KV head h / (n_q / n_kv)), over the keys it sees: with causal,
 * the token at place p sees key j when j < prefix[r], or j <= p and (window 0
 * or p - j < window); without, all keys. cap(s) = cap tanh(s / cap) where
 * cap > 0. A token that sees no key (or only scores of -inf) gets zeros.
 * Keys and values that a token does not see never reach its output, whatever
 * their bits.
 */
typedef struct {
  const void* q;             /* [n_tok][n_q][head_dim] by strides, as in vla_append_args */
  void* o;                   /* may not overlap q */
  int64_t q_tok_stride, q_head_stride, o_tok_stride, o_head_stride;
  float* lse;                /* device [n_tok][n_q], written with ln of the softmax's sum (-inf: no key); or NULL */
  int n_q;                   /* a multiple of n_kv */
  float scale;               /* > 0, or 0 for 1 / sqrt(head_dim) */
  float cap;                 /* 0: no cap; else >= 1e-6, with bf16 <= 1e4 (a score is off by a few 2^-24 of it) */
  int causal;                /* 0 or 1 */
  int window;                /* >= 0; 0: none; needs causal */
  const int32_t* prefix;     /* device [n_req], or NULL (none); needs causal */
  void* ws;                  /* device scratch, 16-byte aligned; may be NULL if none is needed */
  size_t ws_bytes;
} vla_attention_args;

/* Bytes of scratch that vla_paged_attention (shared_len 0) or
 * vla_shared_attention needs with these arguments (q, o, ws and the device
 * buffers of the batch are not looked at; of cap and prefix, whether there is
 * one, which changes how the attention is launched). Host only, no GPU needed. */
vla_status vla_attention_workspace(const vla_kv_pool* pool, const vla_ragged* batch, const vla_attention_args* args,
                                   int shared_len, size_t* bytes);

vla_status vla_paged_attention(const vla_kv_pool* pool, const vla_ragged* batch, const vla_attention_args* args,
                               hipStream_t stream);

/*
 * The same for a batch whose requests have their first shared_len tokens on
 * the same pages: the first shared_len / page_tokens entries of all rows of
 * `pages` are equal (those of row 0 are read). shared_len: a multiple of
 * page_tokens, > 0, <= max_len; every request has kv_len >= shared_len + the
 * tokens that it brings, or sees what its kv_len leaves.
 */
vla_status vla_shared_attention(const vla_kv_pool* pool, const vla_ragged* batch, const vla_attention_args* args,
                                int shared_len, hipStream_t stream);

/*
 * Test hook: how such an attention is launched (arguments as of
 * vla_attention_workspace; host only). plan: int[9] = head dim that rows are
 * padded to, then for the whole attention, or for the common context and what
 * follows it: kernel (0 tiles of 16 rows, waves split the keys, 1 tiles of 128
 * rows, waves split them, 2 fp32, 3 as 1 with two groups of waves that split the
 * keys, 4 tiles of 256 rows, 5 as 2 with tiles of 64 or 32 rows, -1 no such part), row tiles, key tiles a range,
 * ranges.
 */
vla_status vla_debug_paged_plan(const vla_kv_pool* pool, const vla_ragged* batch, const vla_attention_args* args,
                                int shared_len, int* plan);

#ifdef __cplusplus
}
#endif
#endif /* VLA_PAGED_H */
