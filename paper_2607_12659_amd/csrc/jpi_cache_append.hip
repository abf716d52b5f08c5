// Writing keys and values into the pages of an 8-bit cache (jpi_cache_append, include/jpi_cache.h).
//
// One workgroup takes one (sequence, page, KV head) of K or of V: it alone knows
// that page's scale.  It takes the maximum of its new tokens, settles the scale,
// and writes codes: K in pieces of 16 dims of a slot, which are 16 neighbours of
// the token's row, V in pieces of 16 slots of a dim, which a lane collects from 16
// rows that a wave reads along the dims.  Pieces of which only some slots are new
// are read, changed and written back.  The second reading of the tokens comes from
// L2.  Bound by memory for many tokens, by the chain of dependent reads (length,
// table, tokens) for few.
#include <algorithm>

#include "jpi_cache_device.h"

namespace jpi {
namespace {

constexpr int THREADS = 256;

struct AppendArgs {
  const void* src[2];  // K, V
  int64_t outer[2], row[2], head[2];
  uint8_t* codes[2];
  float* scale[2];
  const int32_t *table, *len, *n_new;
  int64_t table_stride;
  int n_pages, kv, cap, lg_page, tokens, count, lg_dim;
};

// the largest of a value over the workgroup
__device__ __forceinline__ u32 block_max(u32 v, u32* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = max(v, (u32)__shfl_xor((int)v, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}

template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, bool vec, float (&f)[N]) {
  typedef T piece __attribute__((ext_vector_type(16 / sizeof(T))));
  constexpr int E = 16 / sizeof(T);
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; i += E) {
      const piece x = *reinterpret_cast<const piece*>(p + i);
#pragma unroll
      for (int e = 0; e < E; ++e) f[i + e] = (float)x[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = (float)p[i];
  }
}

template <typename T, bool E4M3>
__global__ __launch_bounds__(THREADS) void k_append(AppendArgs a, bool vec) {
  typedef Code<E4M3> C;
  __shared__ u32 red[4];
  unsigned id = blockIdx.x;
  const bool values = id & 1;
  id >>= 1;
  const int h = id % a.kv;
  id /= a.kv;
  const int nth = id % a.count, s = id / a.count;
  const int page = 1 << a.lg_page, dh = 1 << a.lg_dim;

  const int start = clamp_len(a.len[s], a.cap);
  const int n = a.n_new ? clamp_len(a.n_new[s], a.tokens) : a.tokens;
  const int end = (int)min((int64_t)start + n, (int64_t)a.cap);
  const int64_t number = (int64_t)(start >> a.lg_page) + nth, base = number << a.lg_page;
  if (base >= end || start >= end) return;
  const int lo = (int)max((int64_t)start - base, (int64_t)0), hi = (int)min((int64_t)end - base, (int64_t)page);
  const int at = a.table[s * a.table_stride + number];
  if ((unsigned)at >= (unsigned)a.n_pages) return;

  const int64_t row = a.row[values];
  const T* src = reinterpret_cast<const T*>(a.src[values]) + s * a.outer[values] + h * a.head[values] + (base - start) * row;
  const int64_t where = (int64_t)at * a.kv + h;
  uint8_t* codes = a.codes[values] + (where << (a.lg_page + a.lg_dim));
  float* scale = a.scale[values] + where;
  const float old = *scale;

  // magnitudes as integers: those of NaN are above infinity's, which are above all others
  u32 top = 0;
  const int pieces = dh >> 4, lg_pieces = a.lg_dim - 4;
  for (int i = threadIdx.x; i < (hi - lo) << lg_pieces; i += THREADS) {
    float f[16];
    load_row<T, 16>(src + (lo + (i >> lg_pieces)) * row + ((i & (pieces - 1)) << 4), vec, f);
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __builtin_bit_cast(u32, f[e]) & 0x7fffffffu);
  }
  top = block_max(top, red);

  const bool had = lo > 0, spoilt = top >= 0x7f800000u || (had && old != old);
  float now = old;
  if (spoilt) now = __builtin_nanf("");
  else if (!had || !(__builtin_bit_cast(float, top) <= C::TOP * old)) now = scale_for<E4M3>(top);
  const bool rescale = had && !spoilt && now != old;
  const float ratio = rescale ? old / now : 1.f;
  const bool zero = spoilt || now == 0.f;
  if (threadIdx.x == 0) *scale = now;  // everybody has read the old one before the maximum's barrier

  const int from = rescale ? 0 : lo;
  if (!values) {
    for (int i = threadIdx.x; i < (hi - from) << lg_pieces; i += THREADS) {
      const int slot = from + (i >> lg_pieces), c = i & (pieces - 1);
      u32x4* p = reinterpret_cast<u32x4*>(codes + (((int64_t)(c << a.lg_page) + slot) << 4));
      float f[16];
      if (slot >= lo) {
        load_row<T, 16>(src + slot * row + (c << 4), vec, f);
#pragma unroll
        for (int e = 0; e < 16; ++e) f[e] = zero ? 0.f : f[e] / now;
      } else {
        const u32x4 w = *p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float g[4];
          C::decode4(w[e], g);
#pragma unroll
          for (int j = 0; j < 4; ++j) f[4 * e + j] = g[j] * ratio;
        }
      }
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = C::encode4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
      *p = w;
    }
  } else {
    const int g0 = from >> 4, groups = ((hi + 15) >> 4) - g0;
    for (int i = threadIdx.x; i < groups << a.lg_dim; i += THREADS) {
      const int g = g0 + (i >> a.lg_dim), d = i & (dh - 1), slot0 = g << 4;
      u32x4* p = reinterpret_cast<u32x4*>(codes + (((int64_t)(g << a.lg_dim) + d) << 4));
      u32x4 w = {0, 0, 0, 0};
      if (slot0 < lo || slot0 + 16 > hi) w = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float f[4], was[4];
        u32 keep = 0;
        C::decode4(w[e], was);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = slot0 + 4 * e + j;
          f[j] = 0.f;
          if (slot >= lo && slot < hi) {
            const float x = (float)src[slot * row + d];
            f[j] = zero ? 0.f : x / now;
          } else if (rescale && slot < lo) {
            f[j] = was[j] * ratio;
          } else {
            keep |= 255u << (8 * j);
          }
        }
        w[e] = (w[e] & keep) | (C::encode4(f[0], f[1], f[2], f[3]) & ~keep);
      }
      *p = w;
    }
  }
}

// pages that the new tokens of a sequence touch at most
int pages_touched(const jpi_cache_pool& p, int tokens) { return (int)(((int64_t)tokens + p.page - 2) / p.page) + 1; }

}  // namespace

bool append_fits(const jpi_cache_pool& p, const jpi_cache_seqs& q, int tokens) {
  return (double)q.n_seqs * pages_touched(p, tokens) * p.n_kv_heads * 2 < (double)(1 << 24);
}

hipError_t launch_append(const jpi_cache_pool& p, const jpi_cache_seqs& q, jpi_dtype dt, int tokens, const jpi_view& k,
                         const jpi_view& v, const int32_t* n_new, hipStream_t s) {
  AppendArgs a{};
  const jpi_view* in[2] = {&k, &v};
  for (int i = 0; i < 2; ++i) a.src[i] = in[i]->data, a.outer[i] = in[i]->outer, a.row[i] = in[i]->row, a.head[i] = in[i]->head;
  a.codes[0] = (uint8_t*)p.k, a.codes[1] = (uint8_t*)p.v;
  a.scale[0] = p.k_scale, a.scale[1] = p.v_scale;
  a.table = q.table, a.len = q.len, a.n_new = n_new, a.table_stride = q.table_stride;
  a.n_pages = p.n_pages, a.kv = p.n_kv_heads, a.cap = q.max_pages * p.page, a.tokens = tokens, a.count = pages_touched(p, tokens);
  a.lg_page = __builtin_ctz(p.page), a.lg_dim = __builtin_ctz(p.head_dim);
  const int es = dt == JPI_BF16 ? 2 : 4;
  const bool vec = aligned16(k, es) && aligned16(v, es);
  const unsigned grid = (unsigned)((int64_t)q.n_seqs * a.count * a.kv * 2);
  if (dt == JPI_BF16) {
    if (p.code == JPI_E4M3) k_append<bf16, true><<<grid, THREADS, 0, s>>>(a, vec);
    else k_append<bf16, false><<<grid, THREADS, 0, s>>>(a, vec);
  } else {
    if (p.code == JPI_E4M3) k_append<float, true><<<grid, THREADS, 0, s>>>(a, vec);
    else k_append<float, false><<<grid, THREADS, 0, s>>>(a, vec);
  }
  return hipGetLastError();
}

}  // namespace jpi
