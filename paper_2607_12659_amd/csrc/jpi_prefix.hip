// C entry points of the prefix-cache operators (include/jpi_prefix.h): argument checks, then the launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <cstdint>

#include "jpi_prefix_internal.h"

using namespace jpi;

namespace {

thread_local char g_err[256] = "";  // no allocation on the error path: nothing here can throw

__attribute__((format(printf, 2, 3))) jpi_status fail(jpi_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return st;
}

jpi_status launched(const char* call, hipError_t e) {
  if (e == hipSuccess) return JPI_OK;
  (void)hipGetLastError();
  return fail(JPI_ERR_HIP, "%s: %s", call, hipGetErrorString(e));
}

bool known(jpi_dtype dt) { return dt == JPI_BF16 || dt == JPI_F32; }
bool negative(const jpi_view& v) { return v.outer < 0 || v.row < 0 || v.head < 0; }
bool aligned16(const jpi_view& v, int es) {
  return ((uintptr_t)v.data & 15) == 0 && (v.outer * es) % 16 == 0 && (v.row * es) % 16 == 0 && (v.head * es) % 16 == 0;
}
// the same places for [outer][rows][heads]: strides of a dimension of size 1 are not used
bool same(const jpi_view& a, const jpi_view& b, int outer, int rows, int heads) {
  return (outer <= 1 || a.outer == b.outer) && (rows <= 1 || a.row == b.row) && (heads <= 1 || a.head == b.head);
}

// an output of which several elements are one
bool folded(const jpi_view& v, int outer, int rows, int heads) {
  return (outer > 1 && v.outer == 0) || (rows > 1 && v.row == 0) || (heads > 1 && v.head == 0);
}
// one of a pair of tensors is written where the other one is read or written
bool crossed(const jpi_view* const in[2], const jpi_view* const out[2]) {
  return out[0]->data == out[1]->data || out[0]->data == in[1]->data || out[1]->data == in[0]->data;
}

// everything about the arguments that does not depend on pointers
jpi_status check_sizes(const char* call, const jpi_shared_attn* a, bool (*launches_fit)(const jpi_shared_attn&)) {
  if (!a) return fail(JPI_ERR_ARG, "%s: NULL arguments", call);
  if (!known(a->dtype)) return fail(JPI_ERR_DTYPE, "%s: dtype must be JPI_BF16 or JPI_F32", call);
  if (a->n_groups < 1 || a->group < 1 || a->q_rows < 1)
    return fail(JPI_ERR_ARG, "%s: n_groups, group and q_rows must be >= 1", call);
  if (a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads != 0)
    return fail(JPI_ERR_ARG, "%s: n_heads must be a multiple of n_kv_heads", call);
  if (a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256)
    return fail(JPI_ERR_ARG, "%s: head_dim must be 64, 128 or 256", call);
  if (a->prefix < 0 || a->suffix < 0) return fail(JPI_ERR_ARG, "%s: negative prefix or suffix", call);
  // the kernels take scores in powers of two
  if (!isfinite(a->scale * 1.44269504f) || !(a->scale > 0.f))
    return fail(JPI_ERR_ARG, "%s: scale, and scale / ln 2, must be finite and > 0", call);
  const double rows = (double)a->n_groups * a->group * a->q_rows * a->n_heads;
  if (rows > 1073741824.0 || a->prefix > 1 << 27 || a->suffix > 1 << 27 || (int64_t)a->n_groups * a->n_kv_heads > 1 << 22 ||
      (double)a->n_groups * a->n_kv_heads * a->prefix > 1073741824.0)
    return fail(JPI_ERR_SHAPE, "%s: more than 2^30 rows, 2^27 slots, 2^22 prefixes x KV heads or 2^30 slots in all", call);
  if (!launches_fit(*a)) return fail(JPI_ERR_SHAPE, "%s: more workgroups than one launch holds", call);
  return JPI_OK;
}

jpi_status check_view(const char* call, const char* what, const jpi_view& v, int es, bool keys) {
  if (!v.data) return fail(JPI_ERR_ARG, "%s: %s is NULL", call, what);
  if (negative(v)) return fail(JPI_ERR_ARG, "%s: %s has a negative stride", call, what);
  if (!aligned16(v, es)) return fail(JPI_ERR_ARG, "%s: %s must be 16-byte aligned, its strides too", call, what);
  if (keys && v.row > 1 << 24) return fail(JPI_ERR_ARG, "%s: rows of %s lie more than 2^24 elements apart", call, what);
  return JPI_OK;
}

jpi_status check_workspace(const char* call, size_t need, const void* ws, size_t bytes) {
  if (need == 0) return JPI_OK;
  if (!ws || bytes < need)
    return fail(JPI_ERR_ARG, "%s: workspace of %zu bytes wanted, %zu given", call, need, ws ? bytes : (size_t)0);
  if ((uintptr_t)ws & 15) return fail(JPI_ERR_ARG, "%s: workspace must be 16-byte aligned", call);
  return JPI_OK;
}

}  // namespace

extern "C" {

const char* jpi_prefix_last_error(void) { return g_err; }

jpi_status jpi_rope(const jpi_rope_config* cfg, jpi_dtype dt, int batch, int tokens, const int32_t* positions,
                    int64_t pos_stride, const jpi_view* q, const jpi_view* q_out, int q_heads, const jpi_view* k,
                    const jpi_view* k_out, int k_heads, void* stream) {
  const char* call = "jpi_rope";
  if (!cfg || !q || !q_out || (k && !k_out)) return fail(JPI_ERR_ARG, "%s: NULL argument", call);
  if (!known(dt)) return fail(JPI_ERR_DTYPE, "%s: dtype must be JPI_BF16 or JPI_F32", call);
  const jpi_rope_config& c = *cfg;
  if (c.head_dim < 2 || c.head_dim > 512 || c.head_dim % 2 != 0)
    return fail(JPI_ERR_ARG, "%s: head_dim must be even, 2 .. 512", call);
  if (c.rot_dim < 2 || c.rot_dim > c.head_dim || c.rot_dim % 2 != 0)
    return fail(JPI_ERR_ARG, "%s: rot_dim must be even, 2 .. head_dim", call);
  if (c.layout != JPI_ROPE_HALF && c.layout != JPI_ROPE_INTERLEAVED) return fail(JPI_ERR_ARG, "%s: unknown layout", call);
  if (c.scaling < JPI_ROPE_PLAIN || c.scaling > JPI_ROPE_PARTS) return fail(JPI_ERR_ARG, "%s: unknown scaling", call);
  if (!isfinite(c.base) || c.base <= 1.0) return fail(JPI_ERR_ARG, "%s: base must be finite and > 1", call);
  if (!isfinite((float)c.amplitude)) return fail(JPI_ERR_ARG, "%s: amplitude must be finite as a float", call);
  if (c.scaling != JPI_ROPE_PLAIN && (!isfinite(c.factor) || c.factor < 1.0))
    return fail(JPI_ERR_ARG, "%s: factor must be finite and >= 1", call);
  if (c.scaling == JPI_ROPE_BASE && c.rot_dim == 2)
    return fail(JPI_ERR_ARG, "%s: JPI_ROPE_BASE needs rot_dim > 2", call);
  if (c.scaling == JPI_ROPE_PARTS && (!(c.trained > 0.0) || !isfinite(c.trained) || !(c.beta_slow >= 0.0) ||
                                      !(c.beta_fast > c.beta_slow) || !isfinite(c.beta_fast)))
    return fail(JPI_ERR_ARG, "%s: JPI_ROPE_PARTS needs trained > 0 and beta_fast > beta_slow >= 0", call);
  if (batch < 0 || tokens < 0 || pos_stride < 0) return fail(JPI_ERR_ARG, "%s: negative size", call);
  if (q_heads < 1 || q_heads > 65536 || (k && (k_heads < 1 || k_heads > 65536)))
    return fail(JPI_ERR_ARG, "%s: heads must be 1 .. 65536", call);
  if ((int64_t)batch * tokens > INT32_MAX) return fail(JPI_ERR_SHAPE, "%s: more than 2^31 - 1 tokens", call);
  if (batch == 0 || tokens == 0) return JPI_OK;
  const jpi_view* in[2] = {q, k};
  const jpi_view* out[2] = {q_out, k_out};
  RopeLaunch l{};
  for (int i = 0; i < (k ? 2 : 1); ++i) {
    if (!in[i]->data || !out[i]->data) return fail(JPI_ERR_ARG, "%s: NULL data", call);
    if (negative(*in[i]) || negative(*out[i])) return fail(JPI_ERR_ARG, "%s: negative stride", call);
    if (in[i]->data == out[i]->data && !same(*in[i], *out[i], batch, tokens, i ? k_heads : q_heads))
      return fail(JPI_ERR_ARG, "%s: in place, input and output need the same strides", call);
    if (folded(*out[i], batch, tokens, i ? k_heads : q_heads)) return fail(JPI_ERR_ARG, "%s: an output has a stride of 0", call);
    l.t[i] = RopeTensor{in[i]->data, out[i]->data, in[i]->outer, in[i]->row, in[i]->head, out[i]->outer, out[i]->row,
                        out[i]->head, i ? k_heads : q_heads};
  }
  if (k && crossed(in, out)) return fail(JPI_ERR_ARG, "%s: q_out or k_out is where another tensor is", call);
  l.pos = positions;
  l.pos_stride = pos_stride;
  l.batch = batch;
  l.tokens = tokens;
  l.head_dim = c.head_dim;
  l.rot_dim = c.rot_dim;
  l.interleaved = c.layout == JPI_ROPE_INTERLEAVED;
  l.inverse = c.inverse != 0;
  l.scaling = c.scaling;
  const double grow = c.scaling == JPI_ROPE_BASE ? (double)c.rot_dim / (c.rot_dim - 2) * log2(c.factor) : 0.0;
  l.log2_step = (log2(c.base) + grow) * 2.0 / c.rot_dim;
  l.factor = c.factor;
  l.trained = c.trained;
  l.beta_fast = c.beta_fast;
  l.beta_slow = c.beta_slow;
  l.amplitude = (float)c.amplitude;
  return launched(call, launch_rope(dt, l, (hipStream_t)stream));
}

jpi_status jpi_shared_attention_workspace(const jpi_shared_attn* a, size_t* bytes) {
  const char* call = "jpi_shared_attention_workspace";
  if (!bytes) return fail(JPI_ERR_ARG, "%s: NULL bytes", call);
  *bytes = 0;
  const jpi_status st = check_sizes(call, a, shared_attention_fits);
  if (st == JPI_OK) *bytes = shared_attention_bytes(*a);
  return st;
}

jpi_status jpi_prefix_weight_workspace(const jpi_shared_attn* a, size_t* bytes) {
  const char* call = "jpi_prefix_weight_workspace";
  if (!bytes) return fail(JPI_ERR_ARG, "%s: NULL bytes", call);
  *bytes = 0;
  const jpi_status st = check_sizes(call, a, prefix_weight_fits);
  if (st == JPI_OK) *bytes = prefix_weight_bytes(*a);
  return st;
}

jpi_status jpi_debug_prefix_plan(const jpi_shared_attn* a, int of_weight, int* waves, int* tiles, int* ranges) {
  const char* call = "jpi_debug_prefix_plan";
  if (!waves || !tiles || !ranges) return fail(JPI_ERR_ARG, "%s: NULL argument", call);
  const jpi_status st = check_sizes(call, a, of_weight ? prefix_weight_fits : shared_attention_fits);
  if (st != JPI_OK) return st;
  const PrefixPlan p = of_weight ? weight_plan(*a) : shared_plan(*a);
  *waves = p.waves, *tiles = p.tiles, *ranges = p.splits;
  return JPI_OK;
}

jpi_status jpi_shared_attention(const jpi_shared_attn* a, void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "jpi_shared_attention";
  jpi_status st = check_sizes(call, a, shared_attention_fits);
  if (st != JPI_OK) return st;
  const int es = a->dtype == JPI_BF16 ? 2 : 4;
  if ((st = check_view(call, "q", a->q, es, false)) != JPI_OK) return st;
  if ((st = check_view(call, "out", a->out, es, false)) != JPI_OK) return st;
  if (a->prefix > 0) {
    if ((st = check_view(call, "k_prefix", a->k_prefix, es, true)) != JPI_OK) return st;
    if ((st = check_view(call, "v_prefix", a->v_prefix, es, true)) != JPI_OK) return st;
  }
  if (a->suffix > 0) {
    if ((st = check_view(call, "k_suffix", a->k_suffix, es, true)) != JPI_OK) return st;
    if ((st = check_view(call, "v_suffix", a->v_suffix, es, true)) != JPI_OK) return st;
  }
  if ((st = check_workspace(call, shared_attention_bytes(*a), workspace, workspace_bytes)) != JPI_OK) return st;
  if (a->out.data == a->q.data || (a->prefix > 0 && (a->out.data == a->k_prefix.data || a->out.data == a->v_prefix.data)) ||
      (a->suffix > 0 && (a->out.data == a->k_suffix.data || a->out.data == a->v_suffix.data)))
    return fail(JPI_ERR_ARG, "%s: out may not be an input", call);
  if (folded(a->out, a->n_groups * a->group, a->q_rows, a->n_heads)) return fail(JPI_ERR_ARG, "%s: out has a stride of 0", call);
  return launched(call, launch_shared_attention(*a, workspace, (hipStream_t)stream));
}

jpi_status jpi_prefix_weight(const jpi_shared_attn* a, const float* weight_in, float decay, float* weight_out,
                             void* workspace, size_t workspace_bytes, void* stream) {
  const char* call = "jpi_prefix_weight";
  jpi_status st = check_sizes(call, a, prefix_weight_fits);
  if (st != JPI_OK) return st;
  if (!isfinite(decay)) return fail(JPI_ERR_ARG, "%s: decay must be finite", call);
  if (a->prefix == 0) return JPI_OK;
  if (!weight_out || !a->lse) return fail(JPI_ERR_ARG, "%s: weight_out or lse is NULL", call);
  const int es = a->dtype == JPI_BF16 ? 2 : 4;
  if ((st = check_view(call, "q", a->q, es, false)) != JPI_OK) return st;
  if ((st = check_view(call, "k_prefix", a->k_prefix, es, true)) != JPI_OK) return st;
  if ((st = check_workspace(call, prefix_weight_bytes(*a), workspace, workspace_bytes)) != JPI_OK) return st;
  return launched(call, launch_prefix_weight(*a, weight_in, decay, weight_out, workspace, (hipStream_t)stream));
}

jpi_status jpi_evict(const jpi_evict_args* a, void* stream) {
  const char* call = "jpi_evict";
  if (!a) return fail(JPI_ERR_ARG, "%s: NULL arguments", call);
  if (!known(a->dtype)) return fail(JPI_ERR_DTYPE, "%s: dtype must be JPI_BF16 or JPI_F32", call);
  if (a->n_outer < 0 || a->n_heads < 1 || a->head_dim < 1 || a->head_dim > 4096 || a->slots < 0 || a->keep < 1)
    return fail(JPI_ERR_ARG, "%s: size out of range", call);
  if (a->n_first < 0 || a->n_last < 0 || (int64_t)a->n_first + a->n_last > a->keep)
    return fail(JPI_ERR_ARG, "%s: n_first + n_last must be 0 .. keep", call);
  if (a->slots > 1 << 26 || (int64_t)a->n_outer * a->n_heads > 1 << 20 ||
      (double)a->n_outer * a->n_heads * a->slots * a->head_dim * (a->dtype == JPI_BF16 ? 2 : 4) > 1099511627776.0)
    return fail(JPI_ERR_SHAPE, "%s: more than 2^26 slots, 2^20 sequences or 2^40 bytes of K", call);
  if (a->n_outer == 0) return JPI_OK;
  if (a->slots > 0 && (!a->weight || !a->index)) return fail(JPI_ERR_ARG, "%s: weight or index is NULL", call);
  const int most = a->keep < a->slots ? a->keep : a->slots;
  if (a->weight_stride < a->slots || (a->weight_out && a->weight_out_stride < most))
    return fail(JPI_ERR_ARG, "%s: weight stride below the number of slots", call);
  if (a->weight_out && a->weight_out == a->weight && a->weight_out_stride != a->weight_stride && a->n_outer * a->n_heads > 1)
    return fail(JPI_ERR_ARG, "%s: in place, the weights need the same stride", call);
  const jpi_view* in[2] = {&a->k, &a->v};
  const jpi_view* out[2] = {&a->k_out, &a->v_out};
  for (int i = 0; i < 2; ++i) {
    if (a->slots > 0 && (!in[i]->data || !out[i]->data)) return fail(JPI_ERR_ARG, "%s: NULL data", call);
    if (negative(*in[i]) || negative(*out[i])) return fail(JPI_ERR_ARG, "%s: negative stride", call);
    if (most > 0 && in[i]->data == out[i]->data && !same(*in[i], *out[i], a->n_outer, most, a->n_heads))
      return fail(JPI_ERR_ARG, "%s: in place, input and output need the same strides", call);
    if (folded(*out[i], a->n_outer, most, a->n_heads)) return fail(JPI_ERR_ARG, "%s: an output has a stride of 0", call);
  }
  if (most > 0 && crossed(in, out)) return fail(JPI_ERR_ARG, "%s: k_out or v_out is where another tensor is", call);
  return launched(call, launch_evict(*a, (hipStream_t)stream));
}

}  // extern "C"
