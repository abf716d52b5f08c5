// Launches of the prefix-cache operators (include/jpi_prefix.h), which checks their arguments first.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/jpi_prefix.h"

namespace jpi {

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
