// What the kernels that turn heads by their positions share (jpi_rope.hip, jpi_norm_rope.hip).
#pragma once

#include "jpi_device.h"
#include "jpi_prefix_internal.h"

namespace jpi {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TABLE = 1024;  // (cos, sin) of a workgroup at most: four tokens of 256 pairs

// f_i / 2 pi: turns per position of pair i
__device__ __forceinline__ double rope_turns(const RopeLaunch& l, int i) {
  constexpr double inv_2pi = 0.15915494309189533577;
  const double f = exp2(-(double)i * l.log2_step);
  double g = f;
  if (l.scaling == JPI_ROPE_LINEAR) {
    g = f / l.factor;
  } else if (l.scaling == JPI_ROPE_PARTS) {
    const double r = l.trained * f * inv_2pi;
    const double keep = fmin(1.0, fmax(0.0, (r - l.beta_slow) / (l.beta_fast - l.beta_slow)));
    g = f * (keep + (1.0 - keep) / l.factor);
  }
  return g * inv_2pi;
}

// N consecutive elements: one piece where they are aligned to their size, else one by one
template <typename T, int N, bool VEC>
struct Piece {
  typedef T vec __attribute__((ext_vector_type(N)));
  T v[N];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC) {
      const vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = x[e];
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = p[e];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (VEC) {
      vec x;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = v[e];
      *reinterpret_cast<vec*>(p) = x;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) p[e] = v[e];
    }
  }
};

// (cos, sin) of the `here` tokens from tok0 on, token after token, by the whole workgroup
__device__ __forceinline__ void rope_table(const RopeLaunch& l, int tok0, int here, float2* table) {
  const int pairs = l.rot_dim >> 1;
  int have = -1;
  double f = 0.0;
  for (int e = threadIdx.x; e < here * pairs; e += ROPE_THREADS) {
    const int tt = e / pairs, i = e - tt * pairs, n = tok0 + tt;
    if (i != have) f = rope_turns(l, i), have = i;
    const int b = n / l.tokens, t = n - b * l.tokens;
    const double turns = (double)(l.pos ? l.pos[b * l.pos_stride + t] : t) * f;
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    table[e] = float2{l.amplitude * cs, l.inverse ? -l.amplitude * sn : l.amplitude * sn};
  }
}

}  // namespace
}  // namespace jpi
