/* maaso_instance.h - C ABI of what a model instance does between its matrix products: the pages of its
 * key/value cache, the write of new keys and values, attention over the pages, and the adjustment of the
 * logits that a token is chosen from.
 *
 * The placer and the distributor (maaso.h) decide from a profile: seconds per decode step against the
 * instance's load, and prefill seconds against the prompt's length.  The entry points here are the parts of
 * such a step that are no plain matrix product, so that an instance's step can be run, and its profile
 * measured, on the card that the placer places it on (maaso_profile_fit takes the samples).
 *
 * Conventions as in maaso.h: functions return MAASO_OK or a negative maaso_status; nothing throws, aborts
 * or prints; DEVICE pointers are caller-owned memory on the instance's device.  Compute calls are
 * asynchronous on the given HIP stream (NULL = the default stream), allocate nothing, free nothing, do no
 * host synchronisation and can be captured into a graph.  An instance serves one call at a time: calls on
 * one stream are ordered by it, a call on another stream than the previous one is ordered behind it with
 * an event, a second thread meanwhile gets MAASO_E_BUSY.  A call that is being captured is not ordered
 * with earlier ones, a call on another stream is not ordered behind a previous call whose stream is being
 * captured by then, and a graph's replays share the instance's workspace with other calls: the caller
 * orders all three (by the event or synchronisation with which it begins the capture, for the first two).
 * Calls that ran at once all the same may have given wrong results; once none runs, maaso_instance_status
 * puts the instance in order again.
 *
 * What the host cannot see (page numbers, rows, lengths, tokens) the kernels check: an entry out of its
 * range is never followed, and raises a bit that maaso_instance_status returns.
 *
 * Sums, softmax statistics and norms are binary32; a result is rounded once to its output's type, and
 * attention's weights to the queries' 16-bit type for the matrix units: half a step of it, relative to each
 * weight (they are 2^(score - m), m a maximum so far that may lag, so at most 2^8).  Results do not depend on
 * the order in which blocks run: a call repeated on the same inputs gives the same bits. */
#ifndef MAASO_INSTANCE_H
#define MAASO_INSTANCE_H

#include "maaso.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MAASO_BF16 = 0,
  MAASO_FP16 = 1,
  MAASO_FP32 = 2,
  MAASO_E4M3 = 3 /* 8 bits, 4 of them exponent, no infinity, largest value 448 */
} maaso_type;

/* bits of maaso_instance_status */
#define MAASO_INST_BAD_PAGE 1u  /* a page number outside the pool, or one given back that nobody held       */
#define MAASO_INST_BAD_ROW 2u   /* a row outside the table, a length outside the row, a fork into a row that
                                   holds tokens                                                              */
#define MAASO_INST_NO_PAGES 4u  /* maaso_kv_extend found too few free pages, or a row too narrow: it did
                                   nothing                                                                   */
#define MAASO_INST_BAD_BOUND 8u /* q_start, group_start, or a start of a list runs backwards or past its end,
                                   or a length passes the bound that the call was given                     */
#define MAASO_INST_BAD_TOKEN 16u /* a token outside the vocabulary, or biases not in ascending order: ignored */
#define MAASO_INST_BAD_POS 32u  /* a position outside the table of angles: taken as the nearest inside      */

#define MAASO_INSTANCE_WORKSPACE_BYTES (256u << 20) /* what workspace_bytes = 0 selects */
#define MAASO_KV_MAX_ROWS 65536u                    /* rows of one call                 */
#define MAASO_KV_MAX_PAGES 16777216u                /* pages of a pool                  */

typedef struct maaso_instance maaso_instance; /* opaque: a device, a workspace, a status word */

/* Creates an instance on `device` with a workspace of workspace_bytes (0: the default above).  A set-up
 * call: it allocates and synchronises.  On error *out is NULL.  Errors: INVALID_ARG, HIP, NOMEM. */
int maaso_instance_create(int device, uint64_t workspace_bytes, maaso_instance** out);
void maaso_instance_destroy(maaso_instance* inst);
/* Synchronises the device, returns the MAASO_INST_* bits raised since the last call in *bits (may be NULL)
 * and clears them.  MAASO_E_INVALID_ARG if there are any, else MAASO_OK.  Errors: INVALID_ARG (no instance),
 * BUSY, HIP; *bits is 0 then. */
int maaso_instance_status(maaso_instance* inst, uint32_t* bits);

/* The pages of a cache: a pool of n_pages pages of page_size tokens, and rows of up to `width` pages.
 * Token t of row r lies in page table[r * width + t / page_size] at place t % page_size.  A page is free
 * when refs[page] == 0; several rows may hold the same page (maaso_kv_fork).  All arrays are DEVICE memory
 * that the caller sets up: refs [n_pages] zeros, table [n_rows * width] -1, length [n_rows] zeros for an
 * empty pool. */
typedef struct {
  uint32_t n_pages, page_size; /* page_size: 16, 32, 64 or 128 */
  uint32_t n_rows, width;
  int32_t* refs;   /* [n_pages] rows that hold the page                  */
  int32_t* table;  /* [n_rows * width] page numbers, -1 where there is none */
  int32_t* length; /* [n_rows] tokens                                    */
} maaso_kv_pages;

/* The cache itself, DEVICE memory.  A page of one layer holds, for each key head, page_size rows of
 * head_dim elements in k and head_dim rows of page_size elements in v (values lie token by token along a
 * row, so that both products of attention read whole rows).  Pages of a layer lie page_stride elements
 * apart and layers layer_stride, in k and in v alike; k, v and the strides' bytes are multiples of 16. */
typedef struct {
  uint32_t type;     /* maaso_type: BF16, FP16 or E4M3                                                     */
  uint32_t n_layers, n_pages, n_kv_heads;
  uint32_t page_size; /* 16, 32, 64 or 128 */
  uint32_t head_dim;  /* 64, 128 or 256    */
  uint64_t page_stride, layer_stride;
  void* k;
  void* v;
  const float* k_scale; /* [n_kv_heads] what an E4M3 value is multiplied by, or NULL for 1; NULL for the */
  const float* v_scale; /*   other types                                                                 */
} maaso_kv_cache;

/* Grows rows: rows[i] (DEVICE, [n], each at most once) gets q_start[i + 1] - q_start[i] tokens more
 * (q_start: DEVICE, [n + 1], from 0 up to n_tok).  Pages are taken lowest number first, for the rows in
 * their order.  A row whose last page is partly filled and held by others as well takes a page of its own
 * for it (also when all its holders grow in one call: then it is free afterwards), and copies[2 * i],
 * copies[2 * i + 1] (DEVICE, [2 * n]) are the pages to copy from and to with maaso_kv_copy, before the rows
 * grow again; -1, -1 where there is none.  slot[t] (DEVICE, [n_tok]) receives page * page_size + place of
 * each new token, pos[t] its position in its row (DEVICE, [n_tok], may be NULL).
 * With too few free pages, a row too narrow, or anything out of range, nothing is changed, slot, pos and
 * copies are -1, and a status bit is raised.  Errors: INVALID_ARG, SHAPE, WORKSPACE, BUSY, HIP. */
int maaso_kv_extend(maaso_instance* inst, const maaso_kv_pages* pages, const int32_t* rows, uint32_t n,
                    const int32_t* q_start, uint32_t n_tok, int64_t* slot, int32_t* pos, int32_t* copies,
                    void* hip_stream);

/* Row children[i] becomes a copy of row parents[i], sharing all its pages (DEVICE, [n] each; the children
 * hold no tokens, are distinct, and are no parents of the same call).  A child that holds tokens, or a row
 * out of range, is left alone and raises MAASO_INST_BAD_ROW.  Errors: INVALID_ARG, SHAPE, BUSY, HIP. */
int maaso_kv_fork(maaso_instance* inst, const maaso_kv_pages* pages, const int32_t* parents,
                  const int32_t* children, uint32_t n, void* hip_stream);

/* Row rows[i] keeps its first keep[i] tokens (DEVICE, [n] each, rows distinct); the pages behind them are
 * given back and their table entries become -1.  keep[i] == 0 frees the row; a row with no more than
 * keep[i] tokens stays as it is.  Errors: INVALID_ARG, SHAPE, BUSY, HIP. */
int maaso_kv_trim(maaso_instance* inst, const maaso_kv_pages* pages, const int32_t* rows,
                  const int32_t* keep, uint32_t n, void* hip_stream);

/* Packs the pool: its n_live held pages get the numbers 0 .. n_live - 1.  Pages below n_live stay, the i-th
 * held page from n_live on becomes the i-th free one below it.  refs_out [n_pages] and table_out
 * [n_rows * width] receive the new state (they may be pages->refs and pages->table themselves), n_live [1]
 * the number of held pages, moves [2 * (n_pages / 2)] the pages to copy from and to, -1 behind the last: no
 * page is both, so that one maaso_kv_copy moves them all.  All DEVICE.
 * Errors: INVALID_ARG, SHAPE, WORKSPACE, BUSY, HIP. */
int maaso_kv_compact(maaso_instance* inst, const maaso_kv_pages* pages, int32_t* refs_out,
                     int32_t* table_out, int32_t* moves, int32_t* n_live, void* hip_stream);

/* Copies page pairs[2 * i] to page pairs[2 * i + 1] in k and v of every layer (DEVICE, [2 * n]; a pair with
 * a negative number is skipped).  No page may be written twice, or both written and read.
 * Errors: INVALID_ARG, SHAPE, BUSY, HIP. */
int maaso_kv_copy(maaso_instance* inst, const maaso_kv_cache* cache, const int32_t* pairs, uint32_t n,
                  void* hip_stream);

/* New tokens' queries, keys and values.  For each token t and each head of q and k:
 *   y = x / sqrt(mean(x^2) + eps) * weight         (where a weight is given, else y = x)
 *   (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin)   for the rotary / 2 pairs of the first `rotary` elements,
 *   (a, b) = (i, i + rotary / 2), or (2 i, 2 i + 1) where `interleaved` is not 0; the angle of pair i at
 *   position p is given by cos_sin[p * rotary + i] and cos_sin[p * rotary + rotary / 2 + i].
 * Queries go to q_out, keys and the values as they are into the cache's layer at slot[t] (negative: not
 * written).  In a cache of 8 bits a value x is held as x / scale, rounded to the nearest, at most 448 in
 * magnitude. */
typedef struct {
  uint32_t type;                       /* of q, k, v, the weights and q_out: BF16 or FP16     */
  uint32_t n_tok, n_heads;             /* n_heads: of q                                        */
  uint32_t rotary;                     /* 0 (no rotation) .. head_dim, a multiple of 16        */
  uint32_t interleaved;
  uint32_t n_pos;                      /* rows of cos_sin                                      */
  float eps;
  const void* q;                       /* [n_tok][n_heads][head_dim]; the heads of a token lie head_dim    */
  const void* k;                       /* [n_tok][n_kv_heads][head_dim]  elements apart, its tokens        */
  const void* v;                       /* [n_tok][n_kv_heads][head_dim]  *_stride                          */
  uint64_t q_stride, k_stride, v_stride, q_out_stride;
  void* q_out;                         /* may be q, with the same stride                       */
  const void* q_weight;                /* [head_dim] or NULL                                   */
  const void* k_weight;                /* [head_dim] or NULL                                   */
  const float* cos_sin;                /* [n_pos][rotary]; may be NULL when rotary == 0        */
  const int32_t* pos;                  /* [n_tok]; may be NULL when rotary == 0                */
  const int64_t* slot;                 /* [n_tok]                                              */
} maaso_kv_append_args;
int maaso_kv_append(maaso_instance* inst, const maaso_kv_cache* cache, uint32_t layer,
                    const maaso_kv_append_args* a, void* hip_stream);

/* Attention of n sequences' newest tokens to all that their rows hold.  Sequence i is row rows[i] of the
 * pages (rows NULL: row i) and has the queries q_start[i] .. q_start[i + 1] - 1, which are the last tokens of
 * the row: query j of n_q sees the keys before position length - n_q + j + 1.  Query head h reads key head
 * h / (n_heads / n_kv_heads).  The sequences need not fill n_tok, and may have no queries (idle places of a captured
 * step): queries before q_start[0] or from q_start[n] on are of no sequence, and their out and lse are left as they are.
 *   out = sum_t softmax_t(scale * q . k_t) v_t,   lse = log sum_t exp(scale * q . k_t)
 * A query that sees no key gets out = 0, lse = -infinity.  What lies behind the keys that a query sees
 * has no part in its result, whatever it holds, infinities and NaN included.
 *
 * Sequences that begin alike: group g is the sequences group_start[g] .. group_start[g + 1] - 1, whose first
 * shared[g] tokens are the same (forked rows hold the same pages for them): these keys are read once for
 * the whole group, from the row of its first sequence, and multiplied with all its queries at once.
 * Sequences outside every group share nothing.
 *
 * max_q, max_len and max_shared bound the queries of a sequence, the length of a row and the tokens
 * shared; what lies beyond is left out and raises MAASO_INST_BAD_BOUND: queries from max_q on are left as
 * they are, keys from max_len on are seen by nobody, and the others' results are as without them.
 * total_len is the sum of the rows' lengths or an estimate of it (0: unknown); only the division of the
 * work depends on it.
 * Errors: INVALID_ARG, SHAPE, WORKSPACE (parts of long or shared rows do not fit), BUSY, HIP. */
typedef struct {
  uint32_t type;                 /* of q and out: BF16 or FP16; the cache has the same, or E4M3  */
  uint32_t n, n_tok, n_heads;
  uint32_t n_groups;             /* 0: no groups                                                  */
  uint32_t max_q, max_len, max_shared;
  uint64_t total_len;
  float scale;
  const void* q;                 /* [n_tok][n_heads][head_dim], tokens q_stride elements apart    */
  void* out;                     /* [n_tok][n_heads][head_dim], tokens out_stride elements apart  */
  uint64_t q_stride, out_stride; /* multiples of 8, as the pointers are of 16 bytes               */
  float* lse;                    /* [n_tok][n_heads] or NULL                                      */
  const int32_t* q_start;        /* [n + 1], DEVICE as all below                                  */
  const int32_t* rows;           /* [n] or NULL                                                   */
  const int32_t* group_start;    /* [n_groups + 1]                                                */
  const int32_t* shared;         /* [n_groups]                                                    */
} maaso_kv_attention_args;
int maaso_kv_attention(maaso_instance* inst, const maaso_kv_cache* cache, uint32_t layer,
                       const maaso_kv_pages* pages, const maaso_kv_attention_args* a, void* hip_stream);

/* Logits as the next token is chosen from.  For token v of row r, said c times in the row's history:
 *   x = logits[r][v]
 *   if c > 0: x = x > 0 ? x / repetition : x * repetition;  x = x - (frequency * c + presence)
 *   x = x + bias (where v is listed);  x = x / temperature;  x = -infinity where the mask's bit is 0
 * in binary32, one rounding per operation, rounded to the type of out.  chosen[r] is the token of the
 * largest x before that rounding, the lowest of equals, NaN never; -1 if none is above -infinity. */
typedef struct {
  uint32_t type, out_type;      /* BF16, FP16 or FP32; out_type FP32 or type                               */
  uint32_t n, vocab;
  uint64_t stride, out_stride;  /* elements between rows                                                   */
  const void* logits;           /* [n][vocab], DEVICE as all below                                         */
  void* out;                    /* [n][vocab], may be logits if type and stride are; or NULL               */
  int32_t* chosen;              /* [n] or NULL (not both)                                                  */
  const float* repetition;      /* [n] each, or NULL for 1, 0, 0, 1; repetition and temperature > 0        */
  const float* frequency;
  const float* presence;
  const float* temperature;
  const int32_t* history;       /* tokens, history_start [n + 1] into them, or both NULL                   */
  const int32_t* history_start;
  uint32_t n_history;           /* elements of history                                                     */
  uint32_t n_bias;              /* elements of bias_token and bias_value                                   */
  const int32_t* bias_token;    /* ascending within a row; bias_start [n + 1] into them, or all NULL       */
  const float* bias_value;
  const int32_t* bias_start;
  const uint32_t* mask;         /* [n_mask][(vocab + 31) / 32], bit v % 32 of word v / 32: allowed; or NULL */
  const int32_t* mask_row;      /* [n] the row's mask, negative: none; NULL: mask r for row r              */
  uint32_t n_mask;
} maaso_logits_args;
int maaso_logits_adjust(maaso_instance* inst, const maaso_logits_args* a, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MAASO_INSTANCE_H */
