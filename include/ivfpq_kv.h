/*
 * ivfpq_kv.h -- C ABI of the paged 4-bit key/value cache: the search path's idea, boxes
 * that say where to look and short codes that are read exactly, for the vectors that a decoder
 * looks up at every token.
 *
 * A step of a server runs
 *   1. ivfpq_kv_plan       page tables and slot maps, on the GPU, from the requests' lengths;
 *   2. ivfpq_kv_append     keys and values of the new tokens, rounded to 4 bits, into the pages,
 *                          with a box (per channel minimum and maximum of the keys) per page;
 *   3. ivfpq_kv_select     optional: for every new token and kv head the pages with the largest
 *                          inner products, as their boxes let one expect;
 *   4. ivfpq_kv_attention  the new tokens' attention over all pages or over the selected ones.
 *
 * Conventions are those of ivfpq.h: device pointers on the current device, nothing is retained,
 * nothing is allocated, nothing synchronises; kernels go to `hip_stream`; return values are
 * ivfpq_status and ivfpq_last_error() has the text; on an argument error nothing is enqueued.
 * Every size below is checked on the host; what is read from device memory (lengths, page
 * numbers, slots) is checked where it is used: a page or a slot outside the cache is skipped.
 *
 * The cache.  A page holds IVFPQ_KV_PAGE tokens of every kv head.  A held value is c * 2^(b - 127)
 * with a 4-bit c, one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, and one byte b per token, head and
 * 32 channels:
 *   b = exponent bits of max|x| minus 2, in 1 .. 254;  c = x * 2^(127 - b) rounded to the nearest,
 *   of two equally near the one with the even code (0, 1, 2, 4), at most 6.
 * A token with a key or value that is infinite or not a number is held with key scale 255 (its
 * keys are NaN, its values 0, in its box it counts as 0): the result of a row that sees it is NaN, others are not
 * touched.  Bytes of a page and head, D = head_dim, ivfpq_kv_page_bytes in all:
 *   [0, 32 D)       keys    token t, channel c: nibble c & 1 of byte t D/2 + c/2
 *   [32 D, 34 D)    their scales  token t, group p: byte ((t % 16) D/32 + p) 4 + t / 16
 *   [34 D, 66 D)    values  token t, channel c: nibble (c / 16) & 1 of byte (c / 32) 1024 +
 *                   (((t / 4) % 4) 16 + c % 16) 16 + (t / 16) 4 + t % 4
 *   [66 D, 68 D)    their scales  byte (c / 32) 64 + ((t / 4) % 4) 16 + (t / 16) 4 + t % 4
 * which is the order in which a wavefront feeds the matrix units: 16 bytes a lane, contiguous
 * across lanes, and no byte shared by two tokens.
 */
#ifndef IVFPQ_KV_H
#define IVFPQ_KV_H

#include "ivfpq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define IVFPQ_KV_PAGE 64          /* tokens of a page                                  */
#define IVFPQ_KV_MAX_REQUESTS 65536
#define IVFPQ_KV_MAX_SELECT 1024  /* pages selected for a token and kv head            */

typedef enum { IVFPQ_KV_BF16 = 0, IVFPQ_KV_FP16 = 1 } ivfpq_kv_dtype;

/* The caller's memory that holds a cache.  `pages` is filled with zeros once, before its first
 * use, and from then on written by ivfpq_kv_append only. */
typedef struct {
  int64_t n_pages;  /* 1 .. 2^25                                                     */
  int32_t kv_heads; /* 1 .. 1024                                                     */
  int32_t head_dim; /* 64, 96, 128 or 256                                            */
  int32_t dtype;    /* an ivfpq_kv_dtype: the type of the keys, values, queries and results */
  void *pages;      /* device [n_pages][kv_heads][68 * head_dim] bytes, 16-byte aligned */
  uint16_t *boxes;  /* device [n_pages][kv_heads][2][head_dim] bf16, minimum then maximum, 16-byte aligned */
} ivfpq_kv_cache;

/* Bytes of one page, all kv heads; 0 where head_dim or kv_heads is not supported. */
size_t ivfpq_kv_page_bytes(int32_t kv_heads, int32_t head_dim);

/* One step; all arrays on the device.  Tokens are the step's new tokens, request by request; rows
 * max_tokens - q_start[requests] at the end stand for no token. */
typedef struct {
  int32_t requests;    /* 0 .. IVFPQ_KV_MAX_REQUESTS                                         */
  int32_t max_tokens;  /* rows of the per-token arrays                                       */
  int32_t table_width; /* pages that a row of the table has room for, 1 .. 2^20              */
  int32_t *table;      /* [requests][table_width] page numbers; the caller's, kept over steps */
  int32_t *kv_lens;    /* the rest is written by ivfpq_kv_plan and read by the other calls:
                          [requests]      tokens held, the new ones among them               */
  int32_t *q_start;    /* [requests + 1]  first new token of a request                       */
  int64_t *slots;      /* [max_tokens]    page * 64 + place in the page, or -1               */
  int32_t *token_req;  /* [max_tokens]    request, or -1                                     */
  int32_t *positions;  /* [max_tokens]    position in the request, or -1                     */
  int32_t *counts;     /* [2 * requests]  room in which ivfpq_kv_plan counts pages of ended requests, or NULL: every
                          workgroup counts them then, which takes longer with many              */
} ivfpq_kv_step;

/* Page tables and slot maps of a step.
 *   past_lens   [requests]  tokens held (a negative one counts as 0)
 *   new_lens    [requests]  new tokens; negative: the request ends, its pages go back
 *   step->table entries below ceil(past / 64) are the pages held; written from there to
 *               ceil((past + new) / 64), -1 where no page was left
 *   free_pages  [free_capacity] ring of the pages that nobody holds; free_state [3]: first taken
 *               index, first index behind them (both count up), and how many pages were missing.
 *               Pages are taken in the order of requests and positions, those of ended requests
 *               are put behind the others and can be taken from the next step on.  The ring needs
 *               room for every page that it and the tables hold (n_pages of the cache is enough);
 *               what it has no room for is dropped.  free_state_out must not be free_state.
 * Where pages are missing, the table has -1, the tokens have slot -1 and count as held all the same; they are neither
 * stored nor seen by attention, in later steps too.  Such a request gives back the pages that it has when it
 * ends (entries below 0 are no pages); or the step is done again, from the same lengths and state, with fewer new tokens.
 * Written: table and free_pages in place (doing a step again from the same lengths and state
 * gives the same), the step's other arrays (kv_lens: 0 for an ended request) and free_state_out.  A step has to
 * fit: past + new <= 64 * table_width (what is beyond has slot -1 and is not counted as held), and the
 * sum of new <= max_tokens.  kv_lens must not be past_lens.  requests == 0 marks all rows as no token. */
int ivfpq_kv_plan(const ivfpq_kv_step *step, const int32_t *past_lens, const int32_t *new_lens, int32_t *free_pages,
                  int64_t free_capacity, const int64_t *free_state, int64_t *free_state_out, void *hip_stream);

/* Rows [tokens][heads][head_dim] of the cache's type, the channels contiguous; base 16-byte
 * aligned, strides in elements, multiples of 8 (a stride that no index uses is not looked at). */
typedef struct {
  const void *data;
  int64_t token_stride, head_stride;
} ivfpq_kv_rows;

/* Rounds `tokens` keys and values into the cache at `slots` (device int64; outside the cache: the
 * token is left out) and widens the boxes of their pages; a page whose first slot is written
 * starts a new box.  The tokens of one page have to follow each other, slots ascending by one, as
 * the plan lays them out.  k_rounded, v_rounded: NULL or device [tokens][kv_heads][head_dim], the
 * values as they are held (rows of left-out tokens are not written). */
int ivfpq_kv_append(const ivfpq_kv_cache *cache, ivfpq_kv_rows k, ivfpq_kv_rows v, const int64_t *slots, int64_t tokens,
                    void *k_rounded, void *v_rounded, void *hip_stream);

/* For every token and kv head the n_select pages of its request (numbers of table columns) that
 * it looks at, ascending, -1 behind them: d_out device [max_tokens][kv_heads][n_select] int32.
 * A token at position p chooses among the columns 0 .. p / 64, all of them if they are n_select
 * at most; otherwise the first `sinks`, the last `recent` and the best of the rest by
 *   max over the query heads of the kv head of sum_d max(q_d lo_d, q_d hi_d) * 2^e,
 * the lower column first among equals, where q = rint(x * (127 * (1 / max|x|))), each step in fp32, over the
 * channels of these query heads (values that are not finite count as 0; a factor that is not finite is 0), e = exponent of the box's largest corner minus
 * 6, and lo, hi = the corners times 2^-e, rounded outwards.  All whole numbers: the choice does
 * not depend on the order of any sum.  A column without a page in the cache comes last. */
size_t ivfpq_kv_select_workspace_bytes(const ivfpq_kv_cache *cache, const ivfpq_kv_step *step, int32_t heads);
int ivfpq_kv_select(const ivfpq_kv_cache *cache, const ivfpq_kv_step *step, ivfpq_kv_rows q, int32_t heads,
                    int32_t n_select, int32_t sinks, int32_t recent, int32_t *d_out, void *d_workspace,
                    size_t workspace_bytes, void *hip_stream);

/* The new tokens' attention.  Query head h reads kv head h / (heads / kv_heads).  A token at position
 * p sees the held positions j <= p; with a window j > p - window too; with `selected` those whose
 * column is among its list (any order; -1 and columns outside the request are skipped, none may come twice).
 *   out = sum_j softmax_j(scale * q . k_j) v_j,   lse = ln sum_j exp(scale * q . k_j)
 * A row that sees nothing, or stands for no token, has out 0 and lse -inf. */
typedef struct {
  ivfpq_kv_rows q;
  int32_t heads;           /* a multiple of kv_heads                                          */
  int32_t max_new;         /* no request has more new tokens; only chooses the kernel: give 1 for decode, whose kernel
                              is another than that of chunks                                  */
  float scale;             /* finite; sizes below 2^-126 count as 2^-126                      */
  int32_t window;          /* 0: none                                                         */
  const int32_t *selected; /* device [max_tokens][kv_heads][n_select], or NULL                */
  int32_t n_select;
  void *out;               /* device rows of the cache's type, aligned and strided as q; they must not overlap */
  int64_t out_token_stride, out_head_stride;
  float *lse;              /* device [max_tokens][heads], or NULL                             */
} ivfpq_kv_attention_args;

/* Bytes for a call with these arguments (rows, strides and pointers of `args` are not looked at).  What is asked for
 * without a window is enough with one. */
size_t ivfpq_kv_attention_workspace_bytes(const ivfpq_kv_cache *cache, const ivfpq_kv_step *step,
                                          const ivfpq_kv_attention_args *args);
int ivfpq_kv_attention(const ivfpq_kv_cache *cache, const ivfpq_kv_step *step, const ivfpq_kv_attention_args *args,
                       void *d_workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* IVFPQ_KV_H */
