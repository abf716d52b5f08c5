// C entry points of the operators of a paged 8-bit cache (include/jpi_cache.h): argument checks, then the launches.
#include <math.h>

#include "jpi_cache_internal.h"

using namespace jpi;

namespace {

thread_local ErrorText fail{};

bool known_page(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }

// sizes and types of a pool
jpi_status check_pool(const char* call, const jpi_cache_pool* p) {
  if (!p) return fail(JPI_ERR_ARG, "%s: NULL pool", call);
  if (p->code != JPI_E4M3 && p->code != JPI_INT8) return fail(JPI_ERR_DTYPE, "%s: code must be JPI_E4M3 or JPI_INT8", call);
  if (p->n_kv_heads < 1 || p->n_kv_heads > 1024) return fail(JPI_ERR_ARG, "%s: n_kv_heads must be 1 .. 1024", call);
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256)
    return fail(JPI_ERR_ARG, "%s: head_dim must be 64, 128 or 256", call);
  if (!known_page(p->page)) return fail(JPI_ERR_ARG, "%s: page must be 16, 32, 64 or 128", call);
  if (p->n_pages < 1 || p->n_pages > 1 << 24) return fail(JPI_ERR_ARG, "%s: n_pages must be 1 .. 2^24", call);
  return JPI_OK;
}

jpi_status check_pool_data(const char* call, const jpi_cache_pool* p) {
  if (!p->k || !p->v || !p->k_scale || !p->v_scale) return fail(JPI_ERR_ARG, "%s: NULL data of the pool", call);
  if (((uintptr_t)p->k | (uintptr_t)p->v) & 15) return fail(JPI_ERR_ARG, "%s: codes must be 16-byte aligned", call);
  if (p->k == p->v || p->k_scale == p->v_scale) return fail(JPI_ERR_ARG, "%s: K and V of the pool are one", call);
  return JPI_OK;
}

jpi_status check_seqs(const char* call, const jpi_cache_seqs* q) {
  if (!q) return fail(JPI_ERR_ARG, "%s: NULL sequences", call);
  if (q->n_seqs < 1 || q->n_seqs > 65536) return fail(JPI_ERR_ARG, "%s: n_seqs must be 1 .. 65536", call);
  if (q->max_pages < 1 || q->max_pages > 1 << 22)  // 2^29 slots at most
    return fail(JPI_ERR_ARG, "%s: max_pages must be 1 .. 2^22", call);
  if (q->table_stride < q->max_pages) return fail(JPI_ERR_ARG, "%s: table_stride below max_pages", call);
  return JPI_OK;
}

jpi_status check_tables(const char* call, const jpi_cache_seqs* q) {
  if (!q->table || !q->len) return fail(JPI_ERR_ARG, "%s: NULL table or len", call);
  return JPI_OK;
}

jpi_status check_workspace(const char* call, size_t need, const void* ws, size_t bytes) {
  if (need == 0) return JPI_OK;
  if (!ws || bytes < need)
    return fail(JPI_ERR_ARG, "%s: workspace of %zu bytes wanted, %zu given", call, need, ws ? bytes : (size_t)0);
  if ((uintptr_t)ws & 15) return fail(JPI_ERR_ARG, "%s: workspace must be 16-byte aligned", call);
  return JPI_OK;
}

// everything about an attention's arguments that does not depend on pointers
jpi_status check_attention(const char* call, const jpi_cache_attn* a, const jpi_cache_pool* p, const jpi_cache_seqs* q) {
  if (!a) return fail(JPI_ERR_ARG, "%s: NULL arguments", call);
  if (!known(a->dtype)) return fail(JPI_ERR_DTYPE, "%s: dtype must be JPI_BF16 or JPI_F32", call);
  jpi_status st;
  if ((st = check_pool(call, p)) != JPI_OK || (st = check_seqs(call, q)) != JPI_OK) return st;
  if (a->q_rows < 1) return fail(JPI_ERR_ARG, "%s: q_rows must be >= 1", call);
  if (a->n_heads < 1 || a->n_heads % p->n_kv_heads != 0)
    return fail(JPI_ERR_ARG, "%s: n_heads must be a multiple of n_kv_heads", call);
  if (a->window < 0 || a->sinks < 0) return fail(JPI_ERR_ARG, "%s: negative window or sinks", call);
  if ((a->window > 0 && !a->causal) || (a->sinks > 0 && a->window == 0))
    return fail(JPI_ERR_ARG, "%s: window needs causal, sinks needs window", call);
  // the kernels take scores in powers of two
  if (!isfinite(a->scale * 1.44269504f) || !(a->scale > 0.f))
    return fail(JPI_ERR_ARG, "%s: scale, and scale / ln 2, must be finite and > 0", call);
  if ((double)q->n_seqs * a->q_rows * a->n_heads > 1073741824.0) return fail(JPI_ERR_SHAPE, "%s: more than 2^30 rows", call);
  if (!cache_attention_fits(*a, *p, *q)) return fail(JPI_ERR_SHAPE, "%s: more workgroups than one launch holds", call);
  return JPI_OK;
}

jpi_status check_rows(const char* call, const char* what, const jpi_view& v, int es) {
  if (!v.data) return fail(JPI_ERR_ARG, "%s: %s is NULL", call, what);
  if (negative(v)) return fail(JPI_ERR_ARG, "%s: %s has a negative stride", call, what);
  if (!aligned16(v, es)) return fail(JPI_ERR_ARG, "%s: %s must be 16-byte aligned, its strides too", call, what);
  return JPI_OK;
}

jpi_status check_moves_sizes(const char* call, const jpi_cache_moves* m) {
  if (!m) return fail(JPI_ERR_ARG, "%s: NULL arguments", call);
  if (!known_page(m->page)) return fail(JPI_ERR_ARG, "%s: page must be 16, 32, 64 or 128", call);
  if (m->n_pages < 1 || m->n_pages > 1 << 24) return fail(JPI_ERR_ARG, "%s: n_pages must be 1 .. 2^24", call);
  const jpi_status st = check_seqs(call, &m->seqs);
  if (st != JPI_OK) return st;
  if ((int64_t)m->seqs.n_seqs * (m->seqs.max_pages + 1) > INT32_MAX || !moves_fit(*m))
    return fail(JPI_ERR_SHAPE, "%s: tables of 2^31 entries or more", call);
  return JPI_OK;
}

jpi_status check_moves(const char* call, const jpi_cache_moves* m, const jpi_cache_pool* pool, int layers, bool lengths, const void* ws,
                       size_t bytes) {
  jpi_status st = check_moves_sizes(call, m);
  if (st != JPI_OK) return st;
  const jpi_cache_seqs& q = m->seqs;
  if (!q.table || !m->refs || !m->table_out || !m->refs_out || (lengths && (!q.len || !m->len_out)))
    return fail(JPI_ERR_ARG, "%s: NULL table, len or refs, or an output of theirs", call);
  if (m->table_out_stride < q.max_pages) return fail(JPI_ERR_ARG, "%s: table_out_stride below max_pages", call);
  if (m->table_out == q.table && m->table_out_stride != q.table_stride && q.n_seqs > 1)
    return fail(JPI_ERR_ARG, "%s: in place, table and table_out need the same stride", call);
  const void *in[3] = {q.table, m->refs, lengths ? q.len : nullptr}, *out[3] = {m->table_out, m->refs_out, lengths ? m->len_out : nullptr};
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 3; ++j)
      if (out[i] && i != j && (out[i] == in[j] || out[i] == out[j]))
        return fail(JPI_ERR_ARG, "%s: an output is where another array is", call);
  if (pool) {
    if ((st = check_pool(call, pool)) != JPI_OK || (st = check_pool_data(call, pool)) != JPI_OK) return st;
    if (pool->n_pages != m->n_pages || pool->page != m->page)
      return fail(JPI_ERR_ARG, "%s: n_pages or page is not the pool's", call);
    if (layers < 1 || layers > 65536) return fail(JPI_ERR_ARG, "%s: layers must be 1 .. 65536", call);
  }
  return check_workspace(call, moves_bytes(*m), ws, bytes);
}

}  // namespace

extern "C" {

const char* jpi_cache_last_error(void) { return fail.text; }

jpi_status jpi_norm_rope(const jpi_head_norm* norm, const jpi_rope_config* cfg, jpi_dtype dt, int batch, int tokens,
                         const int32_t* positions, int64_t pos_stride, const jpi_view* q, const jpi_view* q_out, int q_heads,
                         const jpi_view* k, const jpi_view* k_out, int k_heads, void* stream) {
  const char* call = "jpi_norm_rope";
  if (!norm) return fail(JPI_ERR_ARG, "%s: NULL argument", call);
  if (!known(norm->weight_dtype)) return fail(JPI_ERR_DTYPE, "%s: weight_dtype must be JPI_BF16 or JPI_F32", call);
  if (!((float)norm->eps > 0.f) || !isfinite((float)norm->eps))
    return fail(JPI_ERR_ARG, "%s: eps must be finite and > 0 as a float", call);
  if (norm->weight_stride < 0) return fail(JPI_ERR_ARG, "%s: negative weight_stride", call);
  RopeLaunch l{};
  const jpi_status st =
      check_rope(fail, call, cfg, dt, batch, tokens, positions, pos_stride, q, q_out, q_heads, k, k_out, k_heads, l);
  if (st != JPI_OK || batch == 0 || tokens == 0) return st;
  const NormWeights nw{{norm->q_weight, norm->k_weight}, norm->weight_stride, norm->unit_offset ? 1.f : 0.f, (float)norm->eps};
  return fail.launched(call, launch_norm_rope(dt, norm->weight_dtype, l, nw, (hipStream_t)stream));
}

jpi_status jpi_cache_append(const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, jpi_dtype dt, int tokens, const jpi_view* k,
                            const jpi_view* v, const int32_t* n_new, void* stream) {
  const char* call = "jpi_cache_append";
  jpi_status st;
  if ((st = check_pool(call, pool)) != JPI_OK || (st = check_seqs(call, seqs)) != JPI_OK) return st;
  if (!known(dt)) return fail(JPI_ERR_DTYPE, "%s: dtype must be JPI_BF16 or JPI_F32", call);
  if (tokens < 0) return fail(JPI_ERR_ARG, "%s: negative tokens", call);
  if ((int64_t)seqs->n_seqs * tokens > INT32_MAX) return fail(JPI_ERR_SHAPE, "%s: more than 2^31 - 1 tokens", call);
  if (!append_fits(*pool, *seqs, tokens)) return fail(JPI_ERR_SHAPE, "%s: more workgroups than one launch holds", call);
  if (tokens == 0) return JPI_OK;
  if ((st = check_pool_data(call, pool)) != JPI_OK || (st = check_tables(call, seqs)) != JPI_OK) return st;
  if (!k || !v || !k->data || !v->data) return fail(JPI_ERR_ARG, "%s: k or v is NULL", call);
  if (negative(*k) || negative(*v)) return fail(JPI_ERR_ARG, "%s: negative stride", call);
  return fail.launched(call, launch_append(*pool, *seqs, dt, tokens, *k, *v, n_new, (hipStream_t)stream));
}

jpi_status jpi_cache_attention_workspace(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs,
                                         size_t* bytes) {
  const char* call = "jpi_cache_attention_workspace";
  if (!bytes) return fail(JPI_ERR_ARG, "%s: NULL bytes", call);
  *bytes = 0;
  const jpi_status st = check_attention(call, a, pool, seqs);
  if (st == JPI_OK) *bytes = cache_attention_bytes(*a, *pool, *seqs);
  return st;
}

jpi_status jpi_debug_cache_plan(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, int* groups,
                                int* tiles, int* ranges) {
  const char* call = "jpi_debug_cache_plan";
  if (!groups || !tiles || !ranges) return fail(JPI_ERR_ARG, "%s: NULL argument", call);
  const jpi_status st = check_attention(call, a, pool, seqs);
  if (st != JPI_OK) return st;
  const CachePlan p = cache_plan(*a, *pool, *seqs);
  *groups = p.groups, *tiles = p.tiles, *ranges = p.splits;
  return JPI_OK;
}

jpi_status jpi_debug_cache_waves(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, int* waves) {
  const char* call = "jpi_debug_cache_waves";
  if (!waves) return fail(JPI_ERR_ARG, "%s: NULL argument", call);
  const jpi_status st = check_attention(call, a, pool, seqs);
  if (st == JPI_OK) *waves = cache_plan(*a, *pool, *seqs).waves;
  return st;
}

jpi_status jpi_cache_attention(const jpi_cache_attn* a, const jpi_cache_pool* pool, const jpi_cache_seqs* seqs, void* workspace,
                               size_t workspace_bytes, void* stream) {
  const char* call = "jpi_cache_attention";
  jpi_status st = check_attention(call, a, pool, seqs);
  if (st != JPI_OK) return st;
  if ((st = check_pool_data(call, pool)) != JPI_OK || (st = check_tables(call, seqs)) != JPI_OK) return st;
  const int es = a->dtype == JPI_BF16 ? 2 : 4;
  if ((st = check_rows(call, "q", a->q, es)) != JPI_OK || (st = check_rows(call, "out", a->out, es)) != JPI_OK) return st;
  if ((st = check_workspace(call, cache_attention_bytes(*a, *pool, *seqs), workspace, workspace_bytes)) != JPI_OK) return st;
  if (a->out.data == a->q.data) return fail(JPI_ERR_ARG, "%s: out may not be q", call);
  if (folded(a->out, seqs->n_seqs, a->q_rows, a->n_heads)) return fail(JPI_ERR_ARG, "%s: out has a stride of 0", call);
  return fail.launched(call, launch_cache_attention(*a, *pool, *seqs, workspace, (hipStream_t)stream));
}

jpi_status jpi_cache_moves_workspace(const jpi_cache_moves* m, size_t* bytes) {
  const char* call = "jpi_cache_moves_workspace";
  if (!bytes) return fail(JPI_ERR_ARG, "%s: NULL bytes", call);
  *bytes = 0;
  const jpi_status st = check_moves_sizes(call, m);
  if (st == JPI_OK) *bytes = moves_bytes(*m);
  return st;
}

jpi_status jpi_cache_resize(const jpi_cache_moves* m, const jpi_cache_pool* pool, int layers, const int32_t* new_len,
                            int32_t* short_out, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "jpi_cache_resize";
  const jpi_status st = check_moves(call, m, pool, layers, true, workspace, workspace_bytes);
  if (st != JPI_OK) return st;
  if (!new_len) return fail(JPI_ERR_ARG, "%s: NULL new_len", call);
  return fail.launched(call, launch_resize(*m, pool, layers, new_len, short_out, workspace, (hipStream_t)stream));
}

jpi_status jpi_cache_reorder(const jpi_cache_moves* m, const int32_t* parents, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "jpi_cache_reorder";
  const jpi_status st = check_moves(call, m, nullptr, 0, true, workspace, workspace_bytes);
  if (st != JPI_OK) return st;
  if (!parents) return fail(JPI_ERR_ARG, "%s: NULL parents", call);
  if (parents == m->len_out) return fail(JPI_ERR_ARG, "%s: an output is where another array is", call);
  return fail.launched(call, launch_reorder(*m, parents, workspace, (hipStream_t)stream));
}

jpi_status jpi_cache_compact(const jpi_cache_moves* m, const jpi_cache_pool* pool, int layers, int32_t* n_live_out,
                             void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "jpi_cache_compact";
  const jpi_status st = check_moves(call, m, pool, layers, false, workspace, workspace_bytes);
  if (st != JPI_OK) return st;
  return fail.launched(call, launch_compact(*m, pool, layers, n_live_out, workspace, (hipStream_t)stream));
}

}  // extern "C"
