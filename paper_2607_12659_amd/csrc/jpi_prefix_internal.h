// Launches of the prefix-cache operators (include/jpi_prefix.h), which checks their arguments first.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include <cstdint>

#include "../../include/jpi_prefix.h"

namespace jpi {

// The text of a header's last failure on a thread; no allocation on the error path: nothing here can throw
struct ErrorText {
  char text[256];
  __attribute__((format(printf, 3, 4))) jpi_status operator()(jpi_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return st;
  }
  jpi_status launched(const char* call, hipError_t e) {
    if (e == hipSuccess) return JPI_OK;
    (void)hipGetLastError();
    return (*this)(JPI_ERR_HIP, "%s: %s", call, hipGetErrorString(e));
  }
};

inline bool known(jpi_dtype dt) { return dt == JPI_BF16 || dt == JPI_F32; }
inline bool negative(const jpi_view& v) { return v.outer < 0 || v.row < 0 || v.head < 0; }
inline bool aligned16(const jpi_view& v, int es) {
  return ((uintptr_t)v.data & 15) == 0 && (v.outer * es) % 16 == 0 && (v.row * es) % 16 == 0 && (v.head * es) % 16 == 0;
}
// an output of which several elements are one
inline bool folded(const jpi_view& v, int outer, int rows, int heads) {
  return (outer > 1 && v.outer == 0) || (rows > 1 && v.row == 0) || (heads > 1 && v.head == 0);
}

struct RopeTensor {
  const void* src;
  void* dst;
  int64_t so, sr, sh;  // strides of src, in elements: batch, token, head
  int64_t d_o, dr, dh;
  int heads;
};

struct RopeLaunch {
  RopeTensor t[2];  // queries, keys (heads 0: none)
  const int32_t* pos;
  int64_t pos_stride;
  int batch, tokens, head_dim, rot_dim;
  bool interleaved, inverse;
  int scaling;
  double log2_step;  // f_i = 2^(-i * log2_step)
  double factor, trained, beta_fast, beta_slow;
  float amplitude;
};
// The checks of jpi_rope's arguments, and its launch (l.batch or l.tokens 0: nothing to do)
jpi_status check_rope(ErrorText& fail, const char* call, const jpi_rope_config* cfg, jpi_dtype dt, int batch, int tokens,
                      const int32_t* positions, int64_t pos_stride, const jpi_view* q, const jpi_view* q_out, int q_heads,
                      const jpi_view* k, const jpi_view* k_out, int k_heads, RopeLaunch& l);
hipError_t launch_rope(jpi_dtype dt, const RopeLaunch& l, hipStream_t s);

// how a call is cut: 32-row waves of a workgroup, row tiles and ranges of keys (weights: key tiles and ranges of rows)
struct PrefixPlan {
  int waves, tiles, splits;
};
PrefixPlan shared_plan(const jpi_shared_attn& a);
PrefixPlan weight_plan(const jpi_shared_attn& a);
// whether every launch of the call holds its workgroups
bool shared_attention_fits(const jpi_shared_attn& a);
bool prefix_weight_fits(const jpi_shared_attn& a);

size_t shared_attention_bytes(const jpi_shared_attn& a);
hipError_t launch_shared_attention(const jpi_shared_attn& a, void* ws, hipStream_t s);

size_t prefix_weight_bytes(const jpi_shared_attn& a);
hipError_t launch_prefix_weight(const jpi_shared_attn& a, const float* w_in, float decay, float* w_out, void* ws,
                                hipStream_t s);

hipError_t launch_evict(const jpi_evict_args& a, hipStream_t s);

}  // namespace jpi
