/*
 * sp_serve.h -- what a program that serves a compressed model runs beside its linear layers
 * (libsp, GB300 / sm_103a): the tables of a paged cache, per-head norms with the position rotation,
 * attention over a cache held in 4 bits, and the probabilities of the answer.
 *
 * The paper's deployment measurements (Sec. 3.4) serve whole models; it defines none of these
 * operators, so their definitions stand here.  The conventions of sp.h hold: device pointers of
 * the current device, `stream` a cudaStream_t as void*, asynchronous, a status from every call,
 * nothing allocated and no host synchronisation, so every call can be captured in a CUDA graph.
 * Tables, slots and positions are device data that the host never sees: a kernel checks each
 * index before it uses it, leaves out what lies outside, and records SP_ERR_INVALID_ARG for
 * sp_check.
 *
 * The cache.  Token t of a request lives at slot = table[t / P] * P + t % P, with P tokens to a
 * page and `table` the request's pages in order.  Keys and values are held as 4-bit codes n in
 * 0..15 with one fp16 scale s and one fp16 minimum m per token and key head: value = s * n + m.
 * Block (page, key head) starts at byte (page * kv_heads + head) * P * (D + 8) of the buffer:
 *     [P][D/2]  key codes; byte j of a row holds value 2j in its low half, 2j + 1 in its high half
 *     [P][D/2]  value codes
 *     [P]       keys' (s, m), fp16 each, s first
 *     [P]       values' (s, m)
 * A row x becomes, with its entries clamped to +-2^15 and in fp32 with each operation rounded on
 * its own:
 *     m = fp16(min x)   s = fp16((max x - min x) * (1/15))
 *     n = clamp(rint((x - m) * (1 / s)), 0, 15), or 0 where s = 0
 * and a row with a NaN or an infinity becomes s = 0, m = NaN.  A buffer needs no initial value:
 * what no token was written to takes no part in any result.
 */
#ifndef SP_SERVE_H
#define SP_SERVE_H

#include <stddef.h>
#include <stdint.h>

#include "sp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A cache.  data: pages * kv_heads * page_size * (head_dim + 8) bytes, fewer than 2^63.  page_size 16, 32,
 * 64 or 128, head_dim 64 or 128 (SP_ERR_UNSUPPORTED otherwise). */
typedef struct sp_kv4 {
  void* data;
  int64_t pages;
  int32_t page_size;
  int32_t kv_heads;
  int32_t head_dim;
  int32_t reserved; /* 0 */
} sp_kv4;

/* Bytes of a cache's buffer, from every field but `data`.  Host only. */
sp_status sp_kv4_bytes(const sp_kv4* cache, size_t* bytes);

/* The tables of one step, built on the GPU from the lengths of its requests. */
typedef struct sp_kv_plan_args {
  const int32_t* cached;     /* [requests] tokens that each request holds before the step            */
  const int32_t* new_tokens; /* [requests] tokens that the step adds; < 0: the request has ended     */
  int32_t* table;            /* [requests][width] pages of each request, in order                    */
  int32_t* free_pages;       /* [pages] stack of unused pages, or NULL: `table` is already complete   */
  const int32_t* free_count; /* [1] its height before the step                                       */
  int32_t* next_count;       /* [1] its height after the step (may be free_count)                    */
  int32_t* lens;             /* [requests] tokens after the step (may be `cached`)                   */
  int32_t* cu_q;             /* [requests + 1] first of the step's tokens of each request, their sum */
  int32_t* work;             /* [3 * (requests + 1)] shares of sp_kv4_attend, of its own format      */
  int64_t* slots;            /* [max_tokens] slot of each of the step's tokens; -1 behind the last   */
  int32_t* positions;        /* [max_tokens] position in its request; 0 behind the last              */
  int32_t* status;           /* [1] 0, or why the step does not fit: a sum of SP_PLAN_*              */
  int64_t max_tokens;
  int64_t pages;
  int32_t requests, width;
  int32_t page_size;
  int32_t group;             /* query heads per key head, 1..64, for `work` */
} sp_kv_plan_args;

enum {
  SP_PLAN_PAGES = 1,  /* the stack has too few pages       */
  SP_PLAN_WIDTH = 2,  /* a request outgrows its table row, or all of them what sp_kv4_attend counts */
  SP_PLAN_TOKENS = 4, /* more than max_tokens new tokens   */
  SP_PLAN_INPUT = 8   /* cached or free_count out of range */
};

/* Build the tables of a step.  Ended requests (new_tokens < 0) give their pages back: in the order
 * of the requests, and of each one's table, they go on the stack, and their length becomes 0.
 * Growing requests take the pages that their new length needs beyond the old one off the top of the
 * stack, again in order, and their table rows are extended.  A step that does not fit changes
 * no table, stack or length and has no tokens: cu_q is 0, every slot -1, and *status says why.
 * Unless the step writes over its own inputs (lens = cached, next_count = free_count), the call can
 * be repeated.  SP_ERR_INVALID_ARG for a null pointer (but free_pages, with free_count and
 * next_count), a negative size or a page size that is no power of two; requests == 0 or
 * max_tokens == 0 is allowed.  One launch, or two where max_tokens is large. */
sp_status sp_kv_plan(const sp_kv_plan_args* args, void* stream);

/* Per-head norms of queries and keys with the position rotation, in one pass; keys and values go to
 * the cache's slots in 4 bits, or the keys to a tensor. */
typedef struct sp_rope_args {
  const void* q; /* bf16 [tokens][heads][head_dim], `q_stride` elements from token to token          */
  const void* k; /* bf16 [tokens][kv_heads][head_dim], stride k_stride                               */
  const void* v; /* the same, stride v_stride; NULL without a cache                                  */
  int64_t q_stride, k_stride, v_stride; /* multiples of 8: views of a fused q/k/v row serve         */
  void* q_out;   /* bf16 [tokens][heads][head_dim], contiguous                                       */
  void* k_out;   /* bf16 [tokens][kv_heads][head_dim], contiguous; NULL with a cache                 */
  const sp_kv4* cache;      /* or NULL                                                               */
  const int64_t* slots;     /* [tokens], with a cache; a negative one writes nothing                 */
  const int32_t* positions; /* [tokens] rows of cos_sin                                              */
  const float* cos_sin;     /* fp32 [rows][rot]: rot / 2 cosines, then rot / 2 sines                 */
  int64_t rows;
  const void* q_weight; /* bf16 [head_dim], or NULL: no norm of the queries                          */
  const void* k_weight; /* bf16 [head_dim], or NULL: no norm of the keys                             */
  float eps;
  int32_t tokens, heads, kv_heads;
  int32_t head_dim;     /* 64 or 128 */
  int32_t rot;          /* rotated leading channels: a multiple of 16, at most head_dim */
  int32_t pairs;        /* 0: channel i turns with i + rot / 2; 1: channel 2i with 2i + 1 */
} sp_rope_args;

/* In fp32, each operation rounded on its own and each sum of squares taken by halves (neighbours
 * first, then neighbouring sums), so that an elementwise program gets the same bits:
 *     y = x * (1 / sqrt(sum(x^2) / D + eps)) * weight      (where there is a weight)
 *     (a, b) -> (a * cos - b * sin, b * cos + a * sin)
 * then one rounding to bf16 (q_out, k_out), or to the cache's codes (keys, and the values as they
 * are).  A position outside [0, rows) counts as 0, and a slot outside the cache is left out; both
 * are recorded for sp_check.  One launch.  tokens == 0 returns SP_OK. */
sp_status sp_qk_norm_rope(const sp_rope_args* args, void* stream);

/* The cache's values at n slots, rounded to bf16: k_out, v_out [n][kv_heads][head_dim].  A negative
 * slot reads as zeros; one past the cache too, recorded for sp_check. */
sp_status sp_kv4_read(const sp_kv4* cache, const int64_t* slots, int64_t n, void* k_out, void* v_out, void* stream);

/* Causal attention of a step's tokens over the cache. */
typedef struct sp_attend_args {
  const void* q;  /* bf16 [tokens][heads][head_dim], stride q_stride (a multiple of 8)   */
  void* out;      /* bf16 [tokens][heads][head_dim], stride out_stride (a multiple of 8) */
  int64_t q_stride, out_stride;
  const sp_kv4* cache;
  const int32_t* table; /* [requests][width]                       */
  const int32_t* lens;  /* [requests], this step's tokens included */
  const int32_t* cu_q;  /* [requests + 1]                          */
  const int32_t* work;  /* of sp_kv_plan, for the same group       */
  int64_t tokens;       /* rows of q and out: at least cu_q[requests] */
  int32_t requests, width;
  int32_t heads;        /* a multiple of kv_heads, at most 64 per key head */
  int32_t max_new;      /* at least the largest number of new tokens of a request */
  float scale;          /* of the scores; finite */
  int32_t reserved;     /* 0 */
} sp_attend_args;

/* out = softmax(scale * q . K^T) . V over the values that the cache stands for.  Of a request with
 * L tokens, a of them new, new token i sees the first L - a + i + 1.  Scores, softmax statistics and
 * sums are fp32; queries enter the products exactly (but for entries below 2^-24 of the largest of
 * their own row, which round to 2^-32 of it), weights rounded to fp16, cached keys and values exactly (of
 * a request with more than 32 query rows per key head: values rounded to fp16, and of a key s * n + m the
 * part s * (n - 8), with m + 8 * s exact, so that keys far from zero keep their codes); one rounding to bf16 at
 * the end.  A page that the table does not hold is not read and is recorded for sp_check; what the
 * tokens that would see its keys get is unspecified.  Of a request whose tables do not belong to its
 * lengths nothing is written, and it is recorded.  Rows of `out` behind cu_q[requests] are not written.
 * `workspace` as for sp_linear: sp_kv4_attend_workspace_size bytes, its first
 * SP_WORKSPACE_ZERO_BYTES zero before its first use, calls that share it ordered on one stream; one
 * buffer can serve sp_linear and this call.  Results are bitwise repeatable.  Of a launch that sp_check
 * reports as SP_ERR_TIMEOUT no result is to be used; the workspace is ready for the next call. */
sp_status sp_kv4_attend(const sp_attend_args* args, void* workspace_dev, size_t workspace_bytes, void* stream);

/* Failure-path test (nothing calls it in normal use).  sp_kv4_attend, with warp `warp` of CTA `cta` of its
 * kernel (of the one for many rows, where that runs) first waiting on a shared-memory barrier that nothing completes, and every wait bounded by
 * wait_ms milliseconds.  The warp gives up and records SP_ERR_TIMEOUT, as any whose wait expires; what
 * it would have added to `out` is missing there.  The launch ends by itself, and the workspace is ready
 * for the next call.  A cta or warp that the kernel does not have, or that has no keys to read, gives up
 * nothing.  wait_ms in 1..10000, cta and warp not negative (SP_ERR_INVALID_ARG otherwise); compiled for
 * head_dim 64 and up to 8, or 25 and more, query rows of a request and key head
 * (SP_ERR_UNSUPPORTED otherwise), as variants of the kernels of their own. */
sp_status sp_test_expired_attend(const sp_attend_args* args, void* workspace_dev, size_t workspace_bytes, int32_t cta,
                                 int32_t warp, uint32_t wait_ms, void* stream);

/* Workspace bytes of sp_kv4_attend on the current device, for any batch.  Host only. */
sp_status sp_kv4_attend_workspace_size(int32_t head_dim, size_t* bytes);

/* Log probabilities of given tokens, with the entropy of each row and its most likely entries.
 *   logits     [tokens][vocab] of `dtype`, `stride` elements from row to row (aligned to their own size)
 *   ids        [tokens] int64; a negative one asks for nothing and gets 0, one past the vocabulary
 *              NaN, recorded for sp_check
 *   logp_out   [tokens] fp32: x[id] - log(sum(exp(x)))
 *   entropy_out [tokens] fp32: -sum(p * log p)
 *   top        0..64 entries: top_logp_out fp32 and top_ids_out int64, [tokens][top], by falling
 *              logit, equal ones by rising index; -0 comes below +0, and a NaN counts as the largest;
 *              top <= vocab
 * Sums are fp32 around the row's maximum.  A row of nothing but -inf has log probabilities of -inf and
 * entropy 0; one with a NaN or +inf is NaN.  One launch.  tokens == 0 returns SP_OK. */
typedef enum sp_logits_dtype { SP_LOGITS_BF16 = 0, SP_LOGITS_F32 = 1 } sp_logits_dtype;
sp_status sp_token_logprobs(const void* logits, sp_logits_dtype dtype, int64_t stride, int64_t tokens, int64_t vocab,
                            const int64_t* ids, int32_t top, float* logp_out, float* entropy_out, float* top_logp_out,
                            int64_t* top_ids_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SP_SERVE_H */
