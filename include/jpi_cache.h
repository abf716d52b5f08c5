/* libjpi operators of a paged KV cache in 8 bits: norms of queries and keys with
 * their rotation, room for sequences in a pool of pages, writing keys and values
 * into it, attention over it, and the moves of its pages.
 *
 * The operators of include/jpi_prefix.h work on dense caches in the models' own
 * types.  These are for programs that hold many sequences (texts or rollouts
 * sampled from one observation) of unequal and growing lengths: a sequence's
 * slots lie in pages that a table names, pages may belong to several sequences
 * at once, and a code of 8 bits stands for each element.  A step of such a
 * program is jpi_cache_resize (room for the new tokens), then for each layer
 * jpi_norm_rope (or jpi_rope), jpi_cache_append and jpi_cache_attention, these two
 * with n_new and q_len the lengths after the resize less those before it: 0 for a
 * sequence that the pool had no pages for; jpi_cache_reorder forks, frees and
 * reorders sequences between steps, and jpi_cache_compact moves the pages in use
 * together.
 *
 * Conventions as include/jpi_prefix.h: no handle and no state, the caller's
 * memory and stream, nothing allocated, only kernels enqueued (so a call may be
 * captured into a graph), errors found on the host before that, jpi_view for
 * strided arrays, outputs that overlap neither each other nor, but where a call
 * says so, an input.  Lengths, tables and counts are int32 on the device and are
 * read when the kernels run; lengths outside [0, max_pages * page] count as the
 * nearer end.  The text of the last failure on the calling thread is
 * jpi_cache_last_error().
 */
#ifndef JPI_CACHE_H_
#define JPI_CACHE_H_

#include <stddef.h>
#include <stdint.h>

#include "jpi.h"
#include "jpi_prefix.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Text of the last failure of a call of this header on the calling thread ("" if none). */
const char* jpi_cache_last_error(void);

/* ---- the pool --------------------------------------------------------------
 * One layer's K and V in n_pages pages of `page` slots each.  The element of
 * page p, KV head h, slot t (0 .. page - 1) and dim d is code * scale with its
 * code at byte
 *   K: ((p * n_kv_heads + h) * (head_dim / 16) + d / 16) * page * 16 + t * 16 + d % 16,
 *   V: (((p * n_kv_heads + h) * (page / 16) + t / 16) * head_dim + d) * 16 + t % 16,
 * and its scale at [p * n_kv_heads + h] of k_scale or v_scale: pieces of 16 bytes
 * are what a lane of the matrix instructions takes, so attention reads them
 * straight into registers.  JPI_E4M3: 1 sign, 4 exponent and 3 fraction bits, up
 * to 448, NaN but no infinity; JPI_INT8: two's complement.  Scales may be any
 * finite numbers >= 0; a page whose scale is NaN holds NaN.  NaN codes are not
 * allowed in slots of a sequence (jpi_cache_append never writes one). */
typedef enum { JPI_E4M3 = 0, JPI_INT8 = 1 } jpi_code;

typedef struct {
  int code;                 /* jpi_code */
  int n_kv_heads, head_dim; /* n_kv_heads 1 .. 1024; head_dim 64, 128 or 256 */
  int n_pages, page;        /* n_pages 1 .. 2^24; page 16, 32, 64 or 128 */
  void *k, *v;              /* 16-byte aligned */
  float *k_scale, *v_scale;
} jpi_cache_pool;

/* Sequence s holds slots 0 .. len[s] - 1; slot j is slot j % page of the page
 * with number table[s * table_stride + j / page].  Entries behind the last slot
 * are not read.  An entry outside [0, n_pages) names no page: attention takes its
 * slots for NaN, append writes nothing there, and the page moves pass it by. */
typedef struct {
  int n_seqs, max_pages;    /* n_seqs 1 .. 65536; max_pages 1 .. 2^22 */
  int64_t table_stride;     /* >= max_pages */
  const int32_t* table;     /* device */
  const int32_t* len;       /* device [n_seqs] */
} jpi_cache_seqs;

/* ---- norms of queries and keys with their rotation --------------------------
 * Each head of q and k is normed and then turned as by jpi_rope:
 *   y = x * (sum_d x_d^2 / head_dim + eps)^-1/2 * (weight + offset),
 * offset 1 with unit_offset != 0, else 0; a NULL weight counts as 1 - offset
 * (the norm alone).  All of it in fp32 (the angle as in jpi_rope), rounded once; a
 * head whose squares sum past fp32 (elements of 2^60 and more) comes out 0.
 * q_weight, k_weight: device [head_dim] of type weight_dtype (JPI_BF16 or JPI_F32),
 * that of head h at + h * weight_stride elements (0: all heads share one).
 * eps > 0, also as a float.  Everything else, the errors too, as jpi_rope; a
 * rotation alone and a norm alone are jpi_rope and rot_dim 2 at position 0. */
typedef struct {
  const void *q_weight, *k_weight;
  jpi_dtype weight_dtype;
  int unit_offset;
  int64_t weight_stride;
  double eps;
} jpi_head_norm;

jpi_status jpi_norm_rope(const jpi_head_norm* norm, const jpi_rope_config* cfg, jpi_dtype dt, int batch, int tokens,
                         const int32_t* positions, int64_t pos_stride, const jpi_view* q, const jpi_view* q_out, int q_heads,
                         const jpi_view* k, const jpi_view* k_out, int k_heads, void* stream);

/* ---- writing keys and values ------------------------------------------------
 * Token t < n_new[s] of sequence s becomes its slot seqs->len[s] + t (len is what
 * the sequence holds before the call; it is not changed).  For each page and KV
 * head with new slots, K and V each for itself: A = max |x| of its new tokens, M =
 * 127 (JPI_INT8) or 448 (JPI_E4M3).
 *   - The scale stays if the page has slots before the new ones and A <= M * scale.
 *     Otherwise it becomes 2^e, e >= -126 the least with M * 2^e >= A, and codes of
 *     slots before the new ones become round(code * (old scale / new scale)).
 *   - New codes are round(x / scale).  Roundings are to nearest, ties to even.
 *   - Where A is not finite, or the old scale is NaN, the scale becomes NaN and the
 *     new codes 0: the page holds NaN until it is free again.
 * Scales that are powers of two make every step but the rounding exact, and
 * halving an e4m3 code of 2^-5 or more loses nothing.  Slots that are neither new nor rescaled
 * are left as they were; tokens past max_pages * page slots, and those of pages
 * that are none, are dropped.  A page that the call writes to may belong to one
 * sequence only: jpi_cache_resize sees to it for as many tokens as it lengthened
 * the sequence by, and not for one that it left as it was.  k, v: [n_seqs][tokens]
 * [n_kv_heads][head_dim] of type dt; n_new: device [n_seqs], or NULL for `tokens`
 * each; values outside [0, tokens] count as the nearer end.  Any alignment and
 * strides; 16-byte aligned rows are fastest.  tokens 0: nothing is done.  Errors:
 * JPI_ERR_ARG (NULL, values out of the ranges above, alignment, negative strides),
 * JPI_ERR_SHAPE (more than 2^31 - 1 tokens, or workgroups of 256 threads for pages x
 * KV heads that no launch holds), JPI_ERR_DTYPE, JPI_ERR_HIP. */
jpi_status jpi_cache_append(const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, jpi_dtype dt, int tokens, const jpi_view* k,
                            const jpi_view* v, const int32_t* n_new, void* stream);

/* ---- attention --------------------------------------------------------------
 * Row i (query i < n = q_len[s] of sequence s, head h) is at position p = len[s] -
 * n + i.  Query head h reads KV head h / (n_heads / n_kv_heads).  A row sees the
 * slots j < len[s], with causal != 0 those with j <= p only, and with window > 0
 * of these the ones with j > p - window or j < sinks.  Over what it sees
 *   s_ij = scale * q_i . k_j,  lse_i = log sum_j exp(s_ij),
 *   out_i = sum_j exp(s_ij - lse_i) v_j.
 * A row that sees nothing has out 0 and lse -inf.  Rows i >= q_len[s] of out and
 * lse are left as they were.  NaN in slots that a row does not see does not reach it.
 * In bf16 probabilities are taken in two bf16 parts for the product with V, 2^-16 of
 * each at most lost, and rounded to one, 2^-8, where a call has many rows; calls of
 * fewer than 64 rows on a KV head (q_rows * n_heads / n_kv_heads) take two always.
 * fp32 queries and probabilities are taken in three, which lose nothing (codes are
 * exact in bf16).  Sums are fp32, and the one over V is divided at the end: elements
 * of q past 2^100, or of V past 2^80, may take them out of its range. */
typedef struct {
  jpi_dtype dtype;         /* JPI_BF16 or JPI_F32: q and out */
  int q_rows, n_heads;     /* q_rows >= 1; n_heads a multiple of the pool's n_kv_heads */
  int causal;
  int window, sinks;       /* >= 0; window (0: none) needs causal, sinks needs window */
  float scale;             /* > 0, scale / ln 2 finite (usually head_dim^-1/2) */
  jpi_view q;              /* [n_seqs][q_rows][n_heads][head_dim] */
  const int32_t* q_len;    /* device [n_seqs], or NULL: q_rows each; outside [0, q_rows]: the nearer end */
  jpi_view out;            /* as q */
  float* lse;              /* device [n_seqs][q_rows][n_heads], or NULL */
} jpi_cache_attn;

/* Bytes of workspace that the call with these sizes wants (0: none); pointers are not looked at. */
jpi_status jpi_cache_attention_workspace(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs,
                                         size_t* bytes);

/* workspace: device memory of at least that many bytes, 16-byte aligned, that no
 * other running call uses (its contents need not be kept or cleared).  q and out
 * have to be 16-byte aligned with strides of whole multiples of 16 bytes.  The
 * sum's order depends on the sizes and lengths alone: equal calls give equal bits.
 * Errors: JPI_ERR_ARG (NULL, values out of the ranges above, alignment, a
 * workspace that is too small, out at q's address), JPI_ERR_SHAPE (more than 2^30
 * rows n_seqs * q_rows * n_heads, or more workgroups than a launch holds),
 * JPI_ERR_DTYPE, JPI_ERR_HIP. */
jpi_status jpi_cache_attention(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, void* workspace,
                               size_t workspace_bytes, void* stream);

/* How a call with these sizes is cut, for tests that want a certain cut, for each
 * (sequence, KV head): workgroups of 128 rows that pass the keys through a ring in
 * LDS, or (groups 0) tiles of 16 rows and ranges of their keys.  Errors as the
 * workspace query. */
jpi_status jpi_debug_cache_plan(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, int* groups,
                                int* tiles, int* ranges);
/* And how many waves a workgroup has: 4 or 8. */
jpi_status jpi_debug_cache_waves(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, int* waves);

/* ---- moves of pages ---------------------------------------------------------
 * refs: device int32 [n_pages], the number of sequences that hold each page; a
 * page whose count is <= 0 is free.  The calls read seqs->table, seqs->len and
 * refs and write table_out (row stride table_out_stride >= max_pages), len_out and
 * refs_out whole: rows to their max_pages entries, -1 where the sequence holds
 * nothing.  Each of the three may be its input (same address and stride) or memory
 * that overlaps no input.  Where pages change their place their contents move in
 * all `layers` layers of a pool: layer l's k, v, k_scale and v_scale lie n_pages
 * pages behind layer l - 1's.  pool NULL: counts and tables alone.  workspace: as
 * for jpi_cache_attention. */
typedef struct {
  jpi_cache_seqs seqs;
  const int32_t* refs;
  int32_t* table_out;
  int64_t table_out_stride;
  int32_t *len_out, *refs_out; /* len_out is not used by jpi_cache_compact */
  int n_pages, page;           /* as the pool's, if there is one */
} jpi_cache_moves;

/* Bytes of workspace that any of the three calls below wants with these sizes. */
jpi_status jpi_cache_moves_workspace(const jpi_cache_moves* m, size_t* bytes);

/* Sequence s is to hold new_len[s] slots (device int32; negative: as many as now;
 * more than max_pages * page: that many).  A shorter one gives its last pages back.
 * A longer one takes free pages; if its last page is partly filled and its count is
 * above 1, that page is copied into a free one first, so that new slots never lie
 * in a page that others hold.  Free pages (those with a count <= 0 before the call)
 * are taken in ascending order, by the sequences in their order, the copy before
 * the new ones.  A sequence that needs pages is served if the needs up to and with
 * its own are no more than the free pages; otherwise it stays as it was, its last
 * page shared as before: nothing may be appended to it.  short_out (device int32 [1],
 * or NULL): how many free pages all needs together lacked.
 * Pages that the call sets free serve from the next call on.  seqs->len and
 * new_len may not overlap len_out unless they are len_out itself. */
jpi_status jpi_cache_resize(const jpi_cache_moves* m, const jpi_cache_pool* pool, int layers, const int32_t* new_len,
                            int32_t* short_out, void* workspace, size_t workspace_bytes, void* stream);

/* Sequence s takes over what sequence parents[s] (device int32) holds before the
 * call; a parent outside [0, n_seqs) leaves it empty.  Nothing is copied: forks
 * share pages until they grow. */
jpi_status jpi_cache_reorder(const jpi_cache_moves* m, const int32_t* parents, void* workspace, size_t workspace_bytes, void* stream);

/* Pages in use get the numbers 0 .. n_live - 1: the i-th of them (ascending) whose
 * number is n_live or more moves to the i-th free one below n_live.  All entries of
 * the table that name pages are renumbered, behind a sequence's last slot too;
 * len is not read.  n_live_out: device int32 [1], or NULL. */
jpi_status jpi_cache_compact(const jpi_cache_moves* m, const jpi_cache_pool* pool, int layers, int32_t* n_live_out,
                             void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* JPI_CACHE_H_ */
