// Norms of queries and keys with their rotation (jpi_norm_rope, include/jpi_cache.h).
//
// y = x (sum x^2 / D + eps)^-1/2 (w + offset), then pairs of y turned by their
// angle: every element is read and written once, so the call is bound by memory
// as jpi_rope is.  A head is held in the registers of a few neighbouring lanes
// between the sum of its squares and its rotation; a workgroup takes a few tokens
// whose table of (cos, sin), and the weights that all heads share, it keeps in LDS.
// The norm costs a pass through the lanes for each head and no memory.  336 MB in
// and out of fp32, 67 us, 5.0 TB/s (half of it from the last cache); a token alone
// 4.1 us, a launch and its chain of reads.  Heads off 16-byte boundaries go element by
// element: 8000 tokens of 9 heads of 256 take 19 us in bf16 and 25 in fp32, 39 and 42
// so; with weights of each head 20 and 27.
#include <algorithm>

#include "jpi_cache_internal.h"
#include "jpi_rope_device.h"

namespace jpi {
namespace {

constexpr int MAX_DIM = 512;

template <typename W>
__device__ __forceinline__ float factor_at(const void* w, int64_t i, float offset) {
  return w ? (float)reinterpret_cast<const W*>(w)[i] + offset : 1.f;
}

// N factors of one head from dim d on: the shared ones of LDS, or the head's own
template <int N, bool VEC, typename W>
__device__ __forceinline__ void factors(float (&f)[N], const float* shared, const void* own, int64_t at, int d, float offset) {
  if (own) {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = factor_at<W>(own, at + d + e, offset);
  } else if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(shared + d + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[e + i] = x[i];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = shared[d + e];
  }
}

// Sum over the neighbouring lanes of a head, a power of two of them, the same in each
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  if (lanes >= 16) {
    v = group16_sum(v);
    if (lanes >= 32) v += __shfl_xor(v, 16, 64);
    return lanes == 64 ? halves_sum(v) : v;
  }
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// A unit is N elements of a head, with JPI_ROPE_HALF and their N partners half a rotation further on; lane c of the
// `lanes` (a power of two) of a head has units c, c + lanes ...: U at most.
template <typename T, typename W, int N, bool VEC, bool INTER, int U, int B>
__global__ __launch_bounds__(ROPE_THREADS) void k_norm_rope(RopeLaunch l, NormWeights nw, int first, int n_tok, int tile, int lanes) {
  __shared__ float2 table[ROPE_TABLE];
  __shared__ __align__(16) float shared_w[2][MAX_DIM];
  const int pairs = l.rot_dim >> 1;
  const int tok0 = first + (int)blockIdx.x * tile, here = min(tile, n_tok - tok0);
  const bool per_head = nw.stride != 0;

  if (!per_head) {
    for (int i = threadIdx.x; i < l.head_dim; i += ROPE_THREADS) {
      shared_w[0][i] = factor_at<W>(nw.w[0], i, nw.offset);
      shared_w[1][i] = factor_at<W>(nw.w[1], i, nw.offset);
    }
  }
  rope_table(l, tok0, here, table);
  __syncthreads();

  const unsigned rot_units = (INTER ? l.rot_dim : pairs) / N, units = rot_units + (l.head_dim - l.rot_dim) / N;
  const unsigned heads = l.t[0].heads + l.t[1].heads, c0 = threadIdx.x & (lanes - 1);
  const unsigned step = ROPE_THREADS / lanes, rows = here * heads;
  const float inv_dim = 1.f / (float)l.head_dim;
  const unsigned o0 = (unsigned)tok0 / (unsigned)l.tokens, t0 = tok0 - o0 * l.tokens;
  const bool one = here == 1;
  // B heads of a group of lanes at a time, whose loads are on their way together
  for (unsigned r0 = threadIdx.x / lanes; r0 < rows; r0 += B * step) {  // a head's lanes leave together
    Piece<T, N, VEC> lo[B][U], hi[B][U];
    T* dst[B];
    unsigned tt[B], h[B];
    bool key[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const unsigned r = min(r0 + b * step, rows - 1);
      tt[b] = one ? 0 : r / heads;
      const unsigned hh = r - tt[b] * heads;
      key[b] = hh >= (unsigned)l.t[0].heads;
      const RopeTensor& x = l.t[key[b]];
      h[b] = key[b] ? hh - l.t[0].heads : hh;
      unsigned o = o0, t = t0 + tt[b];
      if (t >= (unsigned)l.tokens) {
        const unsigned by = here <= l.tokens ? 1 : t / (unsigned)l.tokens;
        o += by, t -= by * l.tokens;
      }
      const T* src = reinterpret_cast<const T*>(x.src) + o * x.so + t * x.sr + h[b] * x.sh;
      dst[b] = reinterpret_cast<T*>(x.dst) + o * x.d_o + t * x.dr + h[b] * x.dh;
      if (r0 + b * step >= rows) continue;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned c = c0 + u * lanes;
        if (c >= units) continue;
        lo[b][u].load(src + (c < rot_units ? (int)c * N : l.rot_dim + (int)(c - rot_units) * N));
        if (!INTER && c < rot_units) hi[b][u].load(src + pairs + (int)c * N);
      }
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (r0 + b * step >= rows) break;
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned c = c0 + u * lanes;
        if (c >= units) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          sum = fmaf((float)lo[b][u].v[e], (float)lo[b][u].v[e], sum);
          if (!INTER && c < rot_units) sum = fmaf((float)hi[b][u].v[e], (float)hi[b][u].v[e], sum);
        }
      }
      sum = lanes_sum(sum, lanes);
      const float f = rsqrtf(sum * inv_dim + nw.eps);
      const void* own = per_head ? nw.w[key[b]] : nullptr;
      const float* w = shared_w[key[b]];
      const bool plain = per_head && !own;  // no weight of its own where the other tensor has one for each head
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned c = c0 + u * lanes;
        if (c >= units) continue;
        const bool turn = c < rot_units;
        const int d = turn ? (int)c * N : l.rot_dim + (int)(c - rot_units) * N;
        Piece<T, N, VEC>&x = lo[b][u], &y = hi[b][u];
        float wl[N];
        if (plain) {
#pragma unroll
          for (int e = 0; e < N; ++e) wl[e] = 1.f;
        } else {
          factors<N, VEC, W>(wl, w, own, h[b] * nw.stride, d, nw.offset);
        }
        if (!turn) {
#pragma unroll
          for (int e = 0; e < N; ++e) x.v[e] = from_f32<T>((float)x.v[e] * f * wl[e]);
          x.store(dst[b] + d);
        } else if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const float2 cs = table[tt[b] * pairs + (d + e) / 2];
            const float p = (float)x.v[e] * f * wl[e], q = (float)x.v[e + 1] * f * wl[e + 1];
            x.v[e] = from_f32<T>(p * cs.x - q * cs.y);
            x.v[e + 1] = from_f32<T>(p * cs.y + q * cs.x);
          }
          x.store(dst[b] + d);
        } else {
          float wh[N];
          if (plain) {
#pragma unroll
            for (int e = 0; e < N; ++e) wh[e] = 1.f;
          } else {
            factors<N, VEC, W>(wh, w, own, h[b] * nw.stride, pairs + d, nw.offset);
          }
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 cs = table[tt[b] * pairs + d + e];
            const float p = (float)x.v[e] * f * wl[e], q = (float)y.v[e] * f * wh[e];
            x.v[e] = from_f32<T>(p * cs.x - q * cs.y);
            y.v[e] = from_f32<T>(p * cs.y + q * cs.x);
          }
          x.store(dst[b] + d);
          y.store(dst[b] + pairs + d);
        }
      }
    }
  }
}

template <typename T>
bool whole_pieces(const RopeLaunch& l) {
  constexpr int N = 16 / sizeof(T);
  const int unit = l.interleaved ? l.rot_dim : l.rot_dim / 2;
  int64_t any = unit % N | (l.head_dim - l.rot_dim) % N;
  for (const RopeTensor& t : l.t)
    if (t.heads) {
      any |= (t.so | t.sr | t.sh | t.d_o | t.dr | t.dh) % N;
      any |= (int64_t)(((uintptr_t)t.src | (uintptr_t)t.dst) & 15);
    }
  return any == 0;
}

template <typename T, typename W, int N, bool VEC, bool INTER>
void launch_units(const RopeLaunch& l, const NormWeights& nw, unsigned grid, int first, int n, int tile, hipStream_t s) {
  const int units = (INTER ? l.rot_dim : l.rot_dim / 2) / N + (l.head_dim - l.rot_dim) / N;
  int lanes = 1;
  while (lanes < units && lanes < 64) lanes <<= 1;
  // units of a lane at most: 512 dims in pieces of 4 are two of 64 lanes, in single elements eight
  if constexpr (VEC) {
    if (units <= lanes) k_norm_rope<T, W, N, VEC, INTER, 1, 2><<<grid, ROPE_THREADS, 0, s>>>(l, nw, first, n, tile, lanes);
    else k_norm_rope<T, W, N, VEC, INTER, 2, 1><<<grid, ROPE_THREADS, 0, s>>>(l, nw, first, n, tile, lanes);
  } else {
    k_norm_rope<T, W, N, VEC, INTER, 8, 1><<<grid, ROPE_THREADS, 0, s>>>(l, nw, first, n, tile, lanes);
  }
}

template <typename T, typename W>
hipError_t norm_rope_typed(const RopeLaunch& l, const NormWeights& nw, hipStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const int n = l.batch * l.tokens;
  const int64_t bytes = (int64_t)(l.t[0].heads + l.t[1].heads) * l.head_dim * sizeof(T);
  const int tile = (int)std::min<int64_t>({(16384 + bytes - 1) / bytes, ROPE_TABLE / (l.rot_dim / 2), std::max(1, n / 512)});
  const int64_t most = (int64_t)tile << 22;  // tokens of a launch, whose threads are counted in 32 bits
  for (int64_t first = 0; first < n; first += most) {
    const unsigned grid = (unsigned)((std::min(most, n - first) + tile - 1) / tile);
    if (whole_pieces<T>(l)) {
      if (l.interleaved) launch_units<T, W, N, true, true>(l, nw, grid, (int)first, n, tile, s);
      else launch_units<T, W, N, true, false>(l, nw, grid, (int)first, n, tile, s);
    } else if (l.interleaved) {
      launch_units<T, W, 2, false, true>(l, nw, grid, (int)first, n, tile, s);
    } else {
      launch_units<T, W, 1, false, false>(l, nw, grid, (int)first, n, tile, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_norm_rope(jpi_dtype dt, jpi_dtype weight_dt, const RopeLaunch& l, const NormWeights& nw, hipStream_t s) {
  if (weight_dt == JPI_BF16)
    return dt == JPI_BF16 ? norm_rope_typed<bf16, bf16>(l, nw, s) : norm_rope_typed<float, bf16>(l, nw, s);
  return dt == JPI_BF16 ? norm_rope_typed<bf16, float>(l, nw, s) : norm_rope_typed<float, float>(l, nw, s);
}

}  // namespace jpi
