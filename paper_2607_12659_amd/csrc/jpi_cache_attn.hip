// Attention over a paged cache in 8 bits (jpi_cache_attention, include/jpi_cache.h).
//
// The query rows of a sequence that read one KV head (tokens x the heads on it)
// are tiles of 32; a workgroup's four waves take one row tile and share out its
// keys in tiles of 32, wave w the tiles w, w + 4 ..., and join their sums in LDS.
// Where there are few row tiles the keys are cut into ranges as well, by the
// sequence's own length, and k_cache_join adds them up.
//
// Products use 32 x 32 matrix instructions in bf16 with the operands swapped, S^T
// = K q^T and O^T = V^T P^T: one query row in each lane (lane % 32), a half wave
// (lane / 32) of a row's keys each.  Codes are exact in bf16 (eight significant
// bits hold -128 .. 127 and every e4m3 number), so a page's scale can wait: that of
// K goes into the score, that of V into the probability, both one number per 16
// keys.  fp32 queries and probabilities are taken in three bf16 parts, whose 24
// bits lose nothing, for three products each: 2/5 of the bf16 rate would be left
// of them, the fp32 instructions have 1/16.
//
// The pages' layout gives a lane its operands in pieces of 16 bytes, and a half
// wave's are 512 bytes in a row, so K and V go from memory to registers without
// LDS: 16 dims of a key, 16 keys of a dim.  Row i of S^T takes key 16 ((i >> 2) & 1)
// + 4 (i >> 3) + (i & 3) of the tile, so that register r of half h of the product is
// key 16 h + r: a half's keys are one piece of V, with one page and one scale.
#include <algorithm>
#include <type_traits>

#include "jpi_cache_device.h"

namespace jpi {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int WAVES = 4, TILE = 32;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr float HEADROOM = 16.f;  // log2 of the most that a probability may exceed its row's reference by

struct CacheArgs {
  const void* q;
  int64_t q_outer, q_row, q_head;
  void* out;
  int64_t o_outer, o_row, o_head;
  float* lse;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table, *len, *q_len;
  int64_t table_stride;
  int n_seqs, kv, group, q_rows, n_heads;  // group: query heads of a KV head
  int n_pages, lg_page, cap;
  int causal, window, sinks;
  float qscale;  // scale / ln 2
  int splits, row_tiles;
  float* part;     // [workgroup][32 rows][head_dim]
  float2* stats;   // [workgroup][32 rows]: reference, sum
};

// What a row tile sees, in tiles of its keys: the first `sink_tiles` and those from lo_tile to hi_tile
struct Span {
  int len, nq, rows, i0, i1, pos0, sink_tiles, lo_tile, count;
  __device__ __forceinline__ int tile(int n) const { return n < sink_tiles ? n : n - sink_tiles + lo_tile; }
};

__device__ __forceinline__ Span span_of(const CacheArgs& a, int s, int rt) {
  Span x;
  x.len = clamp_len(a.len[s], a.cap);
  x.nq = a.q_len ? clamp_len(a.q_len[s], a.q_rows) : a.q_rows;
  x.rows = x.nq * a.group;
  x.i0 = rt * TILE / a.group;
  x.i1 = min(x.nq - 1, (rt * TILE + TILE - 1) / a.group);
  x.pos0 = x.len - x.nq;
  const int hi = a.causal ? min(max(x.pos0 + x.i1 + 1, 0), x.len) : x.len;
  const int hi_tile = (hi + TILE - 1) / TILE;
  x.lo_tile = a.window ? min((int)(max((int64_t)x.pos0 + x.i0 - a.window + 1, (int64_t)0) / TILE), hi_tile) : 0;
  x.sink_tiles = a.window ? min((min(a.sinks, hi) + TILE - 1) / TILE, x.lo_tile) : 0;
  x.count = x.sink_tiles + hi_tile - x.lo_tile;
  return x;
}

// Tiles of a range, and how many ranges have any (one at least): a wave gets a tile each where there are as many
__device__ __forceinline__ int per_range(int count, int splits) { return max((count + splits - 1) / splits, WAVES); }
__device__ __forceinline__ int ranges_of(int count, int per) { return max(1, (count + per - 1) / per); }

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// x in PARTS parts of bf16: the largest first
template <int PARTS>
__device__ __forceinline__ void split8(const float* x, bf16x8 (&part)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float rest = x[e];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      part[p][e] = (__bf16)rest;
      if (p + 1 < PARTS) rest -= (float)part[p][e];
    }
  }
}

// The raw pieces of a tile and its scales
template <int DH>
struct Raw {
  u32x4 k[DH / 32], v[DH / 32];
  float ks, vs;
};

template <int DH, bool E4M3, typename T>
__global__ __launch_bounds__(64 * WAVES) void k_cache_attn(CacheArgs a) {
  typedef Code<E4M3> C;
  constexpr int PARTS = sizeof(T) == 2 ? 1 : 3, STEPS = DH / 16, DT = DH / 32;
  constexpr int ROUND = DT < 4 ? DT : 4;  // 32-dim tiles that are joined at once
  __shared__ __align__(16) f32x4 join[WAVES][ROUND][4][64];
  __shared__ float2 wave_stats[WAVES][TILE];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int pairs = a.n_seqs * a.kv;
  const int pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
  const int split = rest % a.splits, rt = rest / a.splits;
  const int s = pair / a.kv, h = pair - s * a.kv;
  const Span x = span_of(a, s, rt);
  if (rt * TILE >= x.rows) return;
  const int per = per_range(x.count, a.splits), ranges = ranges_of(x.count, per);
  if (split >= ranges) return;
  const int last = min(x.count, (split + 1) * per);

  // the lane's row, and the slots that it sees
  const int r = min(rt * TILE + col, x.rows - 1), token = r / a.group, head = h * a.group + (r - token * a.group);
  const int see_hi = a.causal ? min(x.pos0 + token + 1, x.len) : x.len;
  const int64_t see_lo = a.window ? (int64_t)x.pos0 + token - a.window + 1 : 0;
  // tiles from slot full_lo up to slot full_hi are seen whole by all rows
  const int full_hi = a.causal ? min(x.pos0 + x.i0 + 1, x.len) : x.len;
  const int64_t full_lo = a.window ? (int64_t)x.pos0 + x.i1 - a.window + 1 : 0;

  bf16x8 q[PARTS][STEPS];
  {
    const T* p = reinterpret_cast<const T*>(a.q) + s * a.q_outer + token * a.q_row + head * a.q_head + 16 * half;
#pragma unroll
    for (int kk = 0; kk < STEPS; ++kk) {
      const T* at = p + (kk >> 1) * 32 + (kk & 1) * 8;
      if constexpr (PARTS == 1) {
        q[0][kk] = *reinterpret_cast<const bf16x8*>(at);
      } else {
        float f[8];
        const f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = lo[e], f[4 + e] = hi[e];
        bf16x8 part[PARTS];
        split8<PARTS>(f, part);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) q[i][kk] = part[i];
      }
    }
  }

  const int page = 1 << a.lg_page;
  const int64_t page_bytes = (int64_t)page * DH;
  const int32_t* table = a.table + s * a.table_stride;
  const int key = ((col >> 2) & 1) * 16 + (col >> 3) * 4 + (col & 3);  // the tile's key that the lane loads for K

  // pages of the two 16-key halves of a tile; -1 past the length, where nothing is read
  auto pages = [&](int t, int (&id)[2]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int slot = t * TILE + 16 * e;
      id[e] = slot < x.len ? table[slot >> a.lg_page] : -2;
    }
  };
  auto load = [&](int t, const int (&id)[2], Raw<DH>& raw) {
    const int kid = (col >> 2) & 1 ? id[1] : id[0], vid = half ? id[1] : id[0];
    const bool vok = (unsigned)vid < (unsigned)a.n_pages;
    const int64_t kat = (int64_t)((unsigned)kid < (unsigned)a.n_pages ? kid : 0) * a.kv + h;
    const int64_t vat = (int64_t)(vok ? vid : 0) * a.kv + h;
    const uint8_t* kp = a.k + kat * page_bytes + (((half << a.lg_page) + ((t * TILE + key) & (page - 1))) << 4);
    const uint8_t* vp = a.v + vat * page_bytes + ((((t * TILE + 16 * half) & (page - 1)) * DH) + (col << 4));
#pragma unroll
    for (int kk = 0; kk < DT; ++kk) raw.k[kk] = *reinterpret_cast<const u32x4*>(kp + ((int64_t)kk << (a.lg_page + 5)));
#pragma unroll
    for (int d = 0; d < DT; ++d) raw.v[d] = *reinterpret_cast<const u32x4*>(vp + d * 512);
    // a number that names no page: its slots are NaN; past the length nothing is seen
    raw.ks = vok ? a.k_scale[vat] : vid == -2 ? 0.f : __builtin_nanf("");
    raw.vs = vok ? a.v_scale[vat] : vid == -2 ? 0.f : __builtin_nanf("");
  };

  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float m_ref = -INFINITY, sum = 0.f;

  int n = split * per + wave;
  Raw<DH> raw;
  int id[2];
  if (n < last) {
    pages(x.tile(n), id);
    load(x.tile(n), id, raw);
    if (n + WAVES < last) pages(x.tile(n + WAVES), id);
  }
  for (; n < last; n += WAVES) {
    const int t = x.tile(n);
    const Raw<DH> cur = raw;
    if (n + WAVES < last) {
      load(x.tile(n + WAVES), id, raw);
      if (n + 2 * WAVES < last) pages(x.tile(n + 2 * WAVES), id);
    }

    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < STEPS; ++kk) {
      const u32x4 w = cur.k[kk >> 1];
      const bf16x8 codes = kk & 1 ? C::widen8(w[2], w[3]) : C::widen8(w[0], w[1]);
#pragma unroll
      for (int p = PARTS - 1; p >= 0; --p) sc = mfma(codes, q[p][kk], sc);
    }

    const int slot0 = t * TILE;
    const bool whole = slot0 + TILE <= full_hi && (slot0 >= full_lo || slot0 + TILE <= a.sinks);
    const float f = a.qscale * cur.ks;
    u32 seen = 0xffffu;
    if (!whole) {
      seen = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = slot0 + 16 * half + e;
        seen |= (j < see_hi && (j >= see_lo || j < a.sinks) ? 1u : 0u) << e;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      sc[e] *= f;
      if (!whole) sc[e] = seen >> e & 1 ? sc[e] : -INFINITY;
      top = fmaxf(top, sc[e]);
    }
    top = halves_max(top);
    if (__any(top > m_ref + HEADROOM || (m_ref == -INFINITY && top > -INFINITY))) {
      const float now = fmaxf(m_ref, top);
      const float g = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref - now);
      if (now > -INFINITY) {
        sum *= g;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= g;
        m_ref = now;
      }
    }
    const float ref = m_ref == -INFINITY ? 0.f : m_ref;
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(sc[e] - ref);
      sum += p[e];
      p[e] *= cur.vs;
      if (!whole) p[e] = seen >> e & 1 ? p[e] : 0.f;  // 0 * NaN
    }
    bf16x8 pp[2][PARTS];
    split8<PARTS>(p, pp[0]);
    split8<PARTS>(p + 8, pp[1]);

    // codes past the length may be anything
    const int valid = x.len - slot0 - 16 * half;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      u32x4 w = cur.v[d];
      if (slot0 + TILE > x.len) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int bytes = min(max(valid - 4 * e, 0), 4);
          w[e] &= bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1;
        }
      }
      const bf16x8 c0 = C::widen8(w[0], w[1]), c1 = C::widen8(w[2], w[3]);
#pragma unroll
      for (int i = PARTS - 1; i >= 0; --i) o[d] = mfma(c0, pp[0][i], o[d]);
#pragma unroll
      for (int i = PARTS - 1; i >= 0; --i) o[d] = mfma(c1, pp[1][i], o[d]);
    }
  }
  sum = halves_sum(sum);

  // the four waves' sums, brought to one reference and added in their order
  if (half == 0) wave_stats[wave][col] = float2{m_ref, sum};
  __syncthreads();
  float ref = -INFINITY, total = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) ref = fmaxf(ref, wave_stats[w][col].x);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float2 st = wave_stats[w][col];
    total += (st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - ref)) * st.y;
  }
  const float mine = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref - ref);
  const bool here = rt * TILE + col < x.rows, final = ranges == 1;
  const float norm = !final ? 1.f : total == 0.f ? 0.f : 1.f / total;
  float* part = a.part + ((int64_t)blockIdx.x * TILE + col) * DH;
  T* out = reinterpret_cast<T*>(a.out) + s * a.o_outer + token * a.o_row + head * a.o_head;
  if (wave == 0 && half == 0 && here) {
    if (!final) a.stats[(int64_t)blockIdx.x * TILE + col] = float2{ref, total};
    else if (a.lse) a.lse[((int64_t)s * a.q_rows + token) * a.n_heads + head] = total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * LN2;
  }
#pragma unroll
  for (int d0 = 0; d0 < DT; d0 += ROUND) {
    if (d0) __syncthreads();
#pragma unroll
    for (int d = 0; d < ROUND; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = o[d0 + d][4 * j + e] * mine;
        join[wave][d][j][lane] = y;
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ROUND; ++i) {  // ROUND * 4 pieces over the four waves
      const int piece = i * WAVES + wave, d = piece >> 2, j = piece & 3;
      f32x4 y = join[0][d][j][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) y += join[w][d][j][lane];
      if (!here) continue;
      const int at = (d0 + d) * 32 + 8 * j + 4 * half;
      y *= norm;
      if (!final) {
        *reinterpret_cast<f32x4*>(part + at) = y;
      } else if constexpr (sizeof(T) == 2) {
        typedef bf16 b4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<b4*>(out + at) = b4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
      } else {
        *reinterpret_cast<f32x4*>(out + at) = y;
      }
    }
  }
}

// One row of a row tile whose keys were cut into ranges: a workgroup adds up the ranges that have any.  Lanes take four dims
// each, groups of DH / 4 of them one range after the other, and the groups' sums are added in their order.
template <int DH, typename T>
__global__ __launch_bounds__(256) void k_cache_join(CacheArgs a) {
  constexpr int LANES = DH / 4, GROUPS = 256 / LANES;
  __shared__ __align__(16) f32x4 sums[GROUPS][LANES];
  const int pairs = a.n_seqs * a.kv, per_tile = min(TILE, a.q_rows * a.group);
  const int pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
  const int col = rest % per_tile, rt = rest / per_tile;
  const int s = pair / a.kv, h = pair - s * a.kv;
  const Span x = span_of(a, s, rt);
  const int r = rt * TILE + col;
  if (r >= x.rows) return;
  const int ranges = ranges_of(x.count, per_range(x.count, a.splits));
  if (ranges == 1) return;
  const int token = r / a.group, head = h * a.group + (r - token * a.group);
  // range i of the row tile is workgroup (rt * splits + i) * pairs + pair
  const int64_t at = ((int64_t)rt * a.splits * pairs + pair) * TILE + col, step = (int64_t)pairs * TILE;

  float ref = -INFINITY, total = 0.f;
  for (int i = threadIdx.x & 63; i < ranges; i += 64) ref = fmaxf(ref, a.stats[at + i * step].x);
  ref = wave_max(ref);
  for (int i = threadIdx.x & 63; i < ranges; i += 64) {
    const float2 st = a.stats[at + i * step];
    total += (st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - ref)) * st.y;
  }
  total = wave_sum(total);

  const int d4 = threadIdx.x % LANES, group = threadIdx.x / LANES;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = group; i < ranges; i += GROUPS) {
    const float m = a.stats[at + i * step].x;
    const float g = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - ref);
    y += g * *reinterpret_cast<const f32x4*>(a.part + (at + i * step) * DH + 4 * d4);
  }
  sums[group][d4] = y;
  __syncthreads();
  if (threadIdx.x >= LANES) return;
#pragma unroll
  for (int g = 1; g < GROUPS; ++g) y += sums[g][d4];
  y *= total == 0.f ? 0.f : 1.f / total;
  T* out = reinterpret_cast<T*>(a.out) + s * a.o_outer + token * a.o_row + head * a.o_head + 4 * d4;
  if constexpr (sizeof(T) == 2) {
    typedef bf16 b4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<b4*>(out) = b4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
  } else {
    *reinterpret_cast<f32x4*>(out) = y;
  }
  if (threadIdx.x == 0 && a.lse)
    a.lse[((int64_t)s * a.q_rows + token) * a.n_heads + head] = total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * LN2;
}

template <int DH, bool E4M3, typename T>
void launch_typed(const CacheArgs& a, unsigned grid, unsigned rows, hipStream_t s) {
  k_cache_attn<DH, E4M3, T><<<grid, 64 * WAVES, 0, s>>>(a);
  if (a.splits > 1) k_cache_join<DH, T><<<rows, 256, 0, s>>>(a);
}

template <int DH, bool E4M3>
void launch_code(const CacheArgs& a, bool f32, unsigned grid, unsigned rows, hipStream_t s) {
  if (f32) launch_typed<DH, E4M3, float>(a, grid, rows, s);
  else launch_typed<DH, E4M3, bf16>(a, grid, rows, s);
}

template <int DH>
void launch_dim(const CacheArgs& a, int code, bool f32, unsigned grid, unsigned rows, hipStream_t s) {
  if (code == JPI_E4M3) launch_code<DH, true>(a, f32, grid, rows, s);
  else launch_code<DH, false>(a, f32, grid, rows, s);
}

int64_t workgroups(const CachePlan& plan, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  return (int64_t)q.n_seqs * p.n_kv_heads * plan.tiles * plan.splits;
}

}  // namespace

CachePlan cache_plan(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  const int group = a.n_heads / p.n_kv_heads;
  const int64_t tiles = ((int64_t)a.q_rows * group + TILE - 1) / TILE, units = (int64_t)q.n_seqs * p.n_kv_heads * tiles;
  int64_t most = (int64_t)q.max_pages * p.page;
  if (a.window) most = std::min<int64_t>(most, (int64_t)a.window + a.sinks + TILE / group + 2 * TILE);
  const int64_t key_tiles = (most + TILE - 1) / TILE;
  const int64_t splits = std::min<int64_t>({256, 512 / units, key_tiles / WAVES});
  return {WAVES, (int)tiles, (int)std::max<int64_t>(1, splits)};
}

bool cache_attention_fits(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  const CachePlan plan = cache_plan(a, p, q);
  return workgroups(plan, p, q) < 1 << 24 && (plan.splits == 1 || (int64_t)q.n_seqs * a.n_heads * a.q_rows < 1 << 24);
}

size_t cache_attention_bytes(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  const CachePlan plan = cache_plan(a, p, q);
  if (plan.splits == 1) return 0;
  return (size_t)workgroups(plan, p, q) * TILE * (p.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_cache_attention(const jpi_cache_attn& c, const jpi_cache_pool& p, const jpi_cache_seqs& q, void* ws,
                                  hipStream_t s) {
  const CachePlan plan = cache_plan(c, p, q);
  CacheArgs a{};
  a.q = c.q.data, a.q_outer = c.q.outer, a.q_row = c.q.row, a.q_head = c.q.head;
  a.out = c.out.data, a.o_outer = c.out.outer, a.o_row = c.out.row, a.o_head = c.out.head;
  a.lse = c.lse;
  a.k = (const uint8_t*)p.k, a.v = (const uint8_t*)p.v, a.k_scale = p.k_scale, a.v_scale = p.v_scale;
  a.table = q.table, a.len = q.len, a.q_len = c.q_len, a.table_stride = q.table_stride;
  a.n_seqs = q.n_seqs, a.kv = p.n_kv_heads, a.group = c.n_heads / p.n_kv_heads, a.q_rows = c.q_rows, a.n_heads = c.n_heads;
  a.n_pages = p.n_pages, a.lg_page = __builtin_ctz(p.page), a.cap = q.max_pages * p.page;
  a.causal = c.causal != 0, a.window = c.window, a.sinks = c.sinks;
  a.qscale = c.scale * LOG2E;
  a.splits = plan.splits, a.row_tiles = plan.tiles;
  const int64_t wgs = workgroups(plan, p, q);
  a.part = (float*)ws;
  a.stats = (float2*)((char*)ws + (size_t)wgs * TILE * p.head_dim * sizeof(float));
  const unsigned rows = (unsigned)((int64_t)q.n_seqs * p.n_kv_heads * plan.tiles * std::min(TILE, a.q_rows * a.group));
  const bool f32 = c.dtype == JPI_F32;
  switch (p.head_dim) {
    case 64: launch_dim<64>(a, p.code, f32, (unsigned)wgs, rows, s); break;
    case 128: launch_dim<128>(a, p.code, f32, (unsigned)wgs, rows, s); break;
    default: launch_dim<256>(a, p.code, f32, (unsigned)wgs, rows, s);
  }
  return hipGetLastError();
}

}  // namespace jpi
