/* libjpi operators of a prefix cache: rotary positions, attention of a batch
 * that shares a prefix, the weight that its queries lay on each prefix slot,
 * and eviction of the lightest slots.
 *
 * jpi_bind_prefix gives every rollout a prefix KV of its own.  These calls are
 * for programs that hold one prefix for many rollouts (several candidate action
 * chunks, or several sampled texts, of one observation): rotary positions turn
 * queries and keys before the keys enter the cache; the shared attention reads
 * the prefix once for all rollouts of a group and each rollout's own tail
 * behind it; its row sums (lse) give the weight of each slot; eviction keeps
 * the heaviest slots, in their order, and what it leaves can be bound to a
 * jpi_ctx (jpi_prefix_buffers, jpi_bind_prefix) or attended to again.
 *
 * Conventions as include/jpi.h (status codes, streams as hipStream_t values,
 * bf16 as raw 16-bit patterns), and:
 *   - No handle and no state: every call takes device memory of the caller on
 *     the current HIP device, allocates nothing, enqueues kernels only (no
 *     memory sets or copies) and does not synchronise, so it may be captured
 *     into a graph.  Calls may run at once on several streams or threads as
 *     long as they share no output and no workspace.
 *   - Errors are found on the host before anything is enqueued (JPI_ERR_ARG,
 *     JPI_ERR_SHAPE, JPI_ERR_DTYPE); JPI_ERR_HIP reports a launch that failed.
 *     The text of the last failure on the calling thread is
 *     jpi_prefix_last_error().
 *   - Arrays are given as jpi_view: element (o, r, h, d) of
 *     [outer][row][head][head_dim] lies at data[o * outer + r * row + h * head
 *     + d].  Strides are in elements and may be in any order, but not negative;
 *     an input's may be 0.  Outputs may not overlap each other, themselves or,
 *     but where a call says so, an input; what shows it at first sight (equal
 *     addresses, a stride of 0) is JPI_ERR_ARG.
 *   - Lengths are int32 arrays on the device (or NULL: all slots).  They are
 *     read when the kernels run; values outside [0, slots] count as the nearer
 *     end.  Slots at or past a length are never read, so they may hold
 *     anything, NaN included.
 *   - Softmax statistics, sums and scores are fp32; bf16 outputs are rounded
 *     once (round to nearest even).
 */
#ifndef JPI_PREFIX_H_
#define JPI_PREFIX_H_

#include <stddef.h>
#include <stdint.h>

#include "jpi.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void* data;
  int64_t outer, row, head; /* strides in elements; head_dim elements are contiguous */
} jpi_view;

/* Text of the last failure of a call of this header on the calling thread ("" if none). */
const char* jpi_prefix_last_error(void);

/* ---- rotary positions ------------------------------------------------------
 * The first rot_dim of a head's head_dim elements are pairs (x, y) that are
 * turned by the angle a_i = position * f_i:
 *   (x, y) -> amplitude * (x cos a_i - y sin a_i, x sin a_i + y cos a_i),
 * i = 0 .. rot_dim / 2 - 1; elements from rot_dim on are copied.  Pairs are
 * (i, i + rot_dim / 2) with JPI_ROPE_HALF (the layout of this library's models)
 * and (2i, 2i + 1) with JPI_ROPE_INTERLEAVED.
 *   f_i = base^(-2 i / rot_dim), and for contexts past the trained one
 *   JPI_ROPE_LINEAR: f_i / factor (positions interpolated);
 *   JPI_ROPE_BASE: with base * factor^(rot_dim / (rot_dim - 2)) for base;
 *   JPI_ROPE_PARTS: f_i (g + (1 - g) / factor), g = clamp((r - beta_slow) /
 *     (beta_fast - beta_slow), 0, 1), r = trained * f_i / (2 pi) the turns of
 *     pair i within the trained context.
 * inverse != 0 turns by -a_i with the same amplitude: the transposed map, which
 * is the gradient of the forward call with respect to its input; with amplitude
 * 1 it also undoes it, and positions (which may be negative) can be differences,
 * to move cached keys.  Angles are formed in 64 bits, so that far positions lose
 * nothing that fp32 sines and cosines could show. */
typedef enum { JPI_ROPE_HALF = 0, JPI_ROPE_INTERLEAVED = 1 } jpi_rope_layout;
typedef enum { JPI_ROPE_PLAIN = 0, JPI_ROPE_LINEAR = 1, JPI_ROPE_BASE = 2, JPI_ROPE_PARTS = 3 } jpi_rope_scaling;

typedef struct {
  int head_dim;  /* even, 2 .. 512 */
  int rot_dim;   /* even, 2 .. head_dim */
  int layout;    /* jpi_rope_layout */
  int scaling;   /* jpi_rope_scaling */
  int inverse;
  double base;   /* > 1 */
  double factor; /* >= 1; ignored by JPI_ROPE_PLAIN */
  double trained, beta_fast, beta_slow; /* JPI_ROPE_PARTS: trained > 0, beta_fast > beta_slow >= 0 */
  double amplitude;                     /* finite, as a float too */
} jpi_rope_config;

/* Turn q [batch][tokens][q_heads][head_dim] into q_out and, where k is not NULL,
 * k [batch][tokens][k_heads][head_dim] into k_out, in one launch.  An output may
 * be its input (same data and strides, but for dimensions of size 1); other
 * overlaps of an output with an input or with itself are not allowed (a stride of
 * 0 on an input is: all heads read the same row).  positions: device int32, token t of batch b at
 * positions[b * pos_stride + t] (pos_stride 0: shared by the batch), or NULL for
 * 0, 1, 2 ...  Any alignment and strides; 16-byte aligned rows are fastest.
 * batch or tokens 0: nothing is done.  Errors: JPI_ERR_ARG (NULL, values out of
 * the ranges above, a negative stride, q_heads or k_heads < 1), JPI_ERR_SHAPE
 * (more than 2^31 - 1 tokens in all), JPI_ERR_DTYPE, JPI_ERR_HIP. */
jpi_status jpi_rope(const jpi_rope_config* cfg, jpi_dtype dt, int batch, int tokens, const int32_t* positions,
                    int64_t pos_stride, const jpi_view* q, const jpi_view* q_out, int q_heads, const jpi_view* k,
                    const jpi_view* k_out, int k_heads, void* stream);

/* ---- attention of a batch that shares a prefix -----------------------------
 * batch = n_groups * group rollouts; rollout b belongs to group b / group and
 * attends to that group's prefix K and V and to its own tail (suffix) behind it.
 * Query head h reads KV head h / (n_heads / n_kv_heads).  For a row i (query
 * i < q_rows of rollout b, head h), over the prefix slots j <
 * prefix_len[b / group] and the tail slots j < suffix_len[b]:
 *   s_ij = scale * q_i . k_j,  lse_i = log sum_j exp(s_ij),
 *   out_i = sum_j exp(s_ij - lse_i) v_j.
 * causal != 0: the tail's last q_rows keys are the queries' own, so row i sees
 * tail slots j <= suffix_len[b] - q_rows + i only (the prefix always whole).  A
 * row that sees no key has out 0 and lse -inf.  Keys are used as they are
 * (already rotated); in bf16 the probabilities are rounded to bf16 for the
 * product with V, while the row sum and lse take them in fp32.  Rollouts do not
 * affect each other: NaN or infinity in one rollout's queries or tail stays in
 * the rows that see it (of which it may reach every element). */
typedef struct {
  jpi_dtype dtype;                     /* JPI_BF16 or JPI_F32: q, keys, values and out */
  int n_groups, group, q_rows;         /* each >= 1 */
  int n_heads, n_kv_heads, head_dim;   /* n_heads a multiple of n_kv_heads; head_dim 64, 128 or 256 */
  int prefix, suffix;                  /* slots per group and per rollout, >= 0 */
  int causal;
  float scale;                         /* > 0, scale / ln 2 finite (usually head_dim^-1/2) */
  jpi_view q;                          /* [batch][q_rows][n_heads][head_dim] */
  jpi_view k_prefix, v_prefix;         /* [n_groups][prefix][n_kv_heads][head_dim]; not read if prefix is 0 */
  jpi_view k_suffix, v_suffix;         /* [batch][suffix][n_kv_heads][head_dim]; not read if suffix is 0 */
  const int32_t* prefix_len;           /* device [n_groups], or NULL */
  const int32_t* suffix_len;           /* device [batch], or NULL */
  jpi_view out;                        /* [batch][q_rows][n_heads][head_dim]; not used by jpi_prefix_weight */
  float* lse;                          /* device [batch][q_rows][n_heads]; may be NULL in jpi_shared_attention */
} jpi_shared_attn;

/* Bytes of workspace that the call with these arguments wants (0: none).  Only
 * sizes and types are looked at, not the pointers.  The same for
 * jpi_prefix_weight.  Errors as the calls themselves. */
jpi_status jpi_shared_attention_workspace(const jpi_shared_attn* a, size_t* bytes);
jpi_status jpi_prefix_weight_workspace(const jpi_shared_attn* a, size_t* bytes);

/* out and lse as above.  workspace: device memory of at least
 * jpi_shared_attention_workspace bytes, 16-byte aligned, that no other running
 * call uses (its contents need not be kept or cleared).  Data pointers have to
 * be 16-byte aligned and strides whole multiples of 16 bytes; rows of K and V
 * may lie at most 2^24 elements apart.  out must not overlap any input.
 * Errors: JPI_ERR_ARG (NULL, values out of the ranges above, alignment, a
 * workspace that is too small, out at an input's address), JPI_ERR_SHAPE (more
 * than 2^30 rows, 2^27 slots of one prefix or tail, 2^22 prefixes x KV heads, or
 * 2^30 prefix slots x KV heads in all; or more workgroups than a launch holds,
 * which takes millions of rows over millions of slots), JPI_ERR_DTYPE,
 * JPI_ERR_HIP. */
jpi_status jpi_shared_attention(const jpi_shared_attn* a, void* workspace, size_t workspace_bytes, void* stream);

/* The weight that the rows lay on each prefix slot, accumulated:
 *   weight_out[g][kv][j] = decay * weight_in[g][kv][j]
 *                          + sum over the group's rows i of heads on kv of exp(s_ij - lse_i)
 * for j < prefix_len[g]; other slots of weight_out are left as they were.
 * weight_in, weight_out: device fp32 [n_groups][n_kv_heads][prefix]; weight_in
 * may be NULL (zero) or weight_out itself.  a->lse holds the rows' lse from
 * jpi_shared_attention over the same keys (a row whose lse is -inf adds
 * nothing); a->v_prefix, the tail, causal and out are not used.  The sum's order
 * is fixed: equal calls give equal bits.  Errors as jpi_shared_attention, and
 * JPI_ERR_ARG for a decay that is not finite. */
jpi_status jpi_prefix_weight(const jpi_shared_attn* a, const float* weight_in, float decay, float* weight_out,
                             void* workspace, size_t workspace_bytes, void* stream);

/* How a call with these sizes is cut, for tests that want a certain cut:
 * of_weight 0, jpi_shared_attention: waves of a workgroup (32 rows each), row
 * tiles of a (prefix, KV head), ranges of its keys.  of_weight 1,
 * jpi_prefix_weight: waves, key tiles, ranges of its rows.  Errors as the
 * workspace queries. */
jpi_status jpi_debug_prefix_plan(const jpi_shared_attn* a, int of_weight, int* waves, int* tiles, int* ranges);

/* ---- eviction by weight ----------------------------------------------------
 * n_outer x n_heads sequences of up to `slots` cache slots, e.g. layer x
 * rollout, KV head.  A sequence of n = len[o] slots keeps all of them if n <=
 * keep; otherwise the first n_first, the last n_last, and of the others the
 * keep - n_first - n_last with the largest weight (equal weights: the lower
 * slot; NaN counts as -inf; -0 as 0).  Kept slots keep their order: new slot t
 * takes old slot index[t], and index, K, V and weights of new slots t <
 * min(n, keep) are written, while what lies behind them in the outputs is left
 * as it was.  len_out[o] = min(n, keep). */
typedef struct {
  jpi_dtype dtype;
  int n_outer, n_heads, head_dim;  /* n_outer >= 0, the others >= 1 (head_dim up to 4096) */
  int slots, keep;                 /* slots >= 0, keep >= 1 */
  int n_first, n_last;             /* >= 0, together at most keep */
  const float* weight;             /* device, weight[(o * n_heads + h) * weight_stride + j] */
  int64_t weight_stride;           /* >= slots */
  const int32_t* len;              /* device [n_outer], or NULL */
  jpi_view k, v;                   /* [n_outer][slots][n_heads][head_dim] */
  jpi_view k_out, v_out;           /* [n_outer][min(keep, slots)][n_heads][head_dim] */
  float* weight_out;               /* device, stride weight_out_stride >= min(keep, slots); may be NULL */
  int64_t weight_out_stride;
  int32_t* index;                  /* device [n_outer][n_heads][keep] */
  int32_t* len_out;                /* device [n_outer]; may be NULL or len itself */
} jpi_evict_args;

/* k_out, v_out and weight_out may be k, v and weight themselves (same data and
 * strides, but for dimensions of size 1: the cache is compacted where it lies)
 * or memory that overlaps no input; K and V may not overlap each other.  Any
 * alignment; 16-byte aligned rows are fastest.  Errors: JPI_ERR_ARG (NULL, values
 * out of the ranges above), JPI_ERR_SHAPE (more than 2^26 slots, 2^20 sequences
 * n_outer * n_heads, or 2^40 bytes of K), JPI_ERR_DTYPE, JPI_ERR_HIP. */
jpi_status jpi_evict(const jpi_evict_args* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* JPI_PREFIX_H_ */
