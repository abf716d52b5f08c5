// Writing keys and values into the pages of an 8-bit cache (jpi_cache_append, include/jpi_cache.h).
//
// One workgroup takes one (sequence, page, KV head) of K or of V: it alone knows
// that page's scale.  It takes the maximum of its new tokens, settles the scale,
// and writes codes: K in pieces of 16 dims of a slot, which are 16 neighbours of
// the token's row, V in pieces of 16 slots of a dim, which a lane collects from 16
// rows that a wave reads along the dims.  Pieces of which only some slots are new
// are read, changed and written back.  Bound by the chain of dependent reads
// (length, table, tokens and scale) where tokens are few: one of 64 sequences takes
// 6.0 us, 816 of eight sequences, 10 MB in all, 7.5; by memory where they are many:
// 4096 of eight sequences in 8 heads of 128 dims, 201 MB, 45 us, 4.4 TB/s.
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

// 16 neighbours
template <typename T>
__device__ __forceinline__ void load_row(const T* p, bool vec, T (&x)[16]) {
  constexpr int E = 16 / sizeof(T);
  typedef T piece __attribute__((ext_vector_type(E)));
  if (vec) {
#pragma unroll
    for (int i = 0; i < 16; i += E) {
      const piece y = *reinterpret_cast<const piece*>(p + i);
#pragma unroll
      for (int e = 0; e < E; ++e) x[i + e] = y[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = p[i];
  }
}

// P: pieces of 16 codes of a page and head that a thread takes at most.  Their tokens stay in registers between the maximum
// and the codes: read a second time from L2, 816 tokens of 256 dims for eight sequences took 11 us instead of 7.5.
template <typename T, bool E4M3, int P>
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

  // A piece of K: 16 dims of a slot, neighbours of its row; of V: 16 slots of a dim.  The thread's pieces that have new slots:
  const int lg_units = values ? a.lg_dim : a.lg_dim - 4, first = values ? lo >> 4 : lo;
  const int count = ((values ? (hi + 15) >> 4 : hi) - first) << lg_units;
  T x[P][16];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int i = threadIdx.x + k * THREADS;
    if (i >= count) continue;
    const int major = first + (i >> lg_units), unit = i & ((1 << lg_units) - 1);
    if (!values) {
      load_row(src + major * row + (unit << 4), vec, x[k]);
    } else if (hi - lo == 1) {  // a decoded token: sixteen loads with masks took half a us more
      const T y = src[lo * row + unit];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[k][e] = (lo & 15) == e ? y : (T)0.f;
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int slot = (major << 4) + e;
        x[k][e] = slot >= lo && slot < hi ? src[slot * row + unit] : (T)0.f;
      }
    }
  }
  // magnitudes as integers: those of NaN are above infinity's, which are above all others
  u32 top = 0;
#pragma unroll
  for (int k = 0; k < P; ++k)
    if ((int)threadIdx.x + k * THREADS < count) {
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max(top, __builtin_bit_cast(u32, (float)x[k][e]) & 0x7fffffffu);
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

  // codes of a piece of K are at (unit, slot), of V at (16 slots, dim)
  auto place = [&](int major, int unit) {
    return reinterpret_cast<u32x4*>(codes + ((int64_t)(values ? (major << a.lg_dim) + unit : (unit << a.lg_page) + major) << 4));
  };
  auto rescaled = [&](u32 w) {
    float f[4];
    C::decode4(w, f);
    return C::encode4(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
  };
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int i = threadIdx.x + k * THREADS;
    if (i >= count) continue;
    const int major = first + (i >> lg_units), unit = i & ((1 << lg_units) - 1), slot0 = values ? major << 4 : lo;
    u32x4* p = place(major, unit);
    const bool partly = values && (slot0 < lo || slot0 + 16 > hi);
    u32x4 was = {0, 0, 0, 0}, w;
    if (partly) was = *p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = zero ? 0.f : (float)x[k][4 * e + j] / now;
      w[e] = C::encode4(f[0], f[1], f[2], f[3]);
      if (partly) {
        u32 fresh = 0, older = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = slot0 + 4 * e + j;
          fresh |= slot >= lo && slot < hi ? 255u << (8 * j) : 0u;
          older |= rescale && slot < lo ? 255u << (8 * j) : 0u;
        }
        w[e] = (w[e] & fresh) | (rescaled(was[e]) & older) | (was[e] & ~(fresh | older));
      }
    }
    *p = w;
  }
  if (rescale) {  // pieces of slots before the new ones alone
    for (int i = threadIdx.x; i < first << lg_units; i += THREADS) {
      u32x4* p = place(i >> lg_units, i & ((1 << lg_units) - 1));
      u32x4 w = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = rescaled(w[e]);
      *p = w;
    }
  }
}

template <typename T, bool E4M3>
void launch_pieces(const AppendArgs& a, bool vec, unsigned grid, hipStream_t s) {
  const int most = std::min(1 << a.lg_page, (a.tokens + 15) / 16 * 16 + 16);  // slots of whole pieces of V that the tokens can touch
  const int pieces = ((most << a.lg_dim) / 16 + THREADS - 1) / THREADS;
  if (pieces <= 1) k_append<T, E4M3, 1><<<grid, THREADS, 0, s>>>(a, vec);
  else if (pieces <= 2) k_append<T, E4M3, 2><<<grid, THREADS, 0, s>>>(a, vec);
  else if (pieces <= 4) k_append<T, E4M3, 4><<<grid, THREADS, 0, s>>>(a, vec);
  else k_append<T, E4M3, 8><<<grid, THREADS, 0, s>>>(a, vec);
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
    if (p.code == JPI_E4M3) launch_pieces<bf16, true>(a, vec, grid, s);
    else launch_pieces<bf16, false>(a, vec, grid, s);
  } else {
    if (p.code == JPI_E4M3) launch_pieces<float, true>(a, vec, grid, s);
    else launch_pieces<float, false>(a, vec, grid, s);
  }
  return hipGetLastError();
}

}  // namespace jpi
