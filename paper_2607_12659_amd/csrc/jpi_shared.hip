// Attention of a batch that shares a prefix, and the weight of its slots
// (jpi_shared_attention, jpi_prefix_weight, include/jpi_prefix.h).
//
// All query rows of a group that read one KV head (rollouts x query rows x the
// heads on that KV head) form one matrix against one key sequence: the prefix,
// which every row sees, and behind it the tails of the rollouts, each seen by
// its own rows only.  A workgroup takes 32 rows per wave and a range of 32-key
// tiles of that sequence, so each prefix tile that it loads serves all its rows,
// whichever rollouts they belong to.  A running maximum and sum per row give the
// softmax in one pass; ranges of one row tile are joined by k_shared_merge.
//
// Products use 32 x 32 matrix instructions with the operands swapped:
// S^T = K q^T puts one query row in each lane (lane % 32) and 16 of the tile's
// keys in its registers, register r <-> key 8 (r / 4) + 4 (lane / 32) + r % 4, so
// the row maximum and sum are in-lane but for one lane swap, and P^T is the B
// operand of O^T = V^T P^T without leaving its registers.
#include <algorithm>
#include <type_traits>

#include "jpi_device.h"
#include "jpi_prefix_internal.h"

namespace jpi {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32;
typedef u32 u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int KEYS = 32;          // keys per tile
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr float HEADROOM = 16.f;  // log2 of the most that a probability may exceed its row's reference by

// A tile of 32 rows (keys, or queries) of DH elements in LDS, in 16-byte chunks.  Chunk c of row r lies at
// chunk place(r, c) of the row: the permutations keep the lanes of one LDS read in different banks.
template <typename T, int DH>
struct Tile {
  static constexpr int CE = 16 / sizeof(T);      // elements of a chunk
  static constexpr int CPR = DH / CE;            // chunks of a row
  static constexpr int KS = CPR / 2;             // chunk pairs (the two lane halves) of a row
  static constexpr int NT = DH / 32;             // 32-wide output tiles
  static constexpr int BYTES = KEYS * DH * (int)sizeof(T);
  typedef T chunk __attribute__((ext_vector_type(CE)));
  // 32 rows at one chunk: 16 rows fill the 64 banks
  static __device__ __forceinline__ int place(int r, int c) { return c ^ (CPR >= 16 ? r & 15 : (r >> 1) & 7); }
  // V as the transposed operand.  bf16: four consecutive keys at 64 bytes; fp32: keys r and r + 4 at 128 bytes
  static __device__ __forceinline__ int place_v(int r, int c) {
    if constexpr (sizeof(T) == 4) return c ^ ((r >> 2) & 1) * 8;
    return c ^ (CPR >= 16 ? (r & 3) << 2 : ((r >> 1) & 1) << 2);
  }
};

template <typename T>
__device__ __forceinline__ f32x16 mfma_chunk(const typename Tile<T, 64>::chunk& a, const typename Tile<T, 64>::chunk& b,
                                             f32x16 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
}

// the larger of this lane's value and that of the lane 32 away (one swap; the pair is copied before the bit casts,
// since a bit cast of an element of the returned vector reads element 0 for both)
__device__ __forceinline__ void halves(float v, float& a, float& b) {
  const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(u32, v), __builtin_bit_cast(u32, v), false, false);
  const u32 x = p[0], y = p[1];
  a = __builtin_bit_cast(float, x);
  b = __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float halves_max(float v) {
  float a, b;
  halves(v, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float halves_sum(float v) {
  float a, b;
  halves(v, a, b);
  return a + b;
}

struct View {
  const char* data;
  int64_t outer, row, head;  // bytes
};

struct SharedLaunch {
  View q, kp, vp, ks, vs, out;
  const int32_t *plen, *slen;
  float* lse;
  float* part;    // [splits][rows in all][DH]: a range's sum of p v (null: the output is written directly)
  float2* stats;  // [splits][rows in all]: its reference and sum of p
  int n_groups, group, q_rows, n_heads, n_kv, per_kv, prefix, suffix;
  int causal, splits, row_tiles;
  float qscale;  // scale * log2(e): scores in powers of two
};

// Rows of a (group, KV head): r = (rollout of the group * q_rows + query) * per_kv + head of the KV head.
struct Row {
  int b, i, h;  // rollout in the batch, query, head; b < 0: past the last row
};
__device__ __forceinline__ Row row_of(const SharedLaunch& l, int g, int kv, int r) {
  if (r >= l.group * l.q_rows * l.per_kv) return Row{-1, 0, 0};
  const int qi = (int)((unsigned)r / (unsigned)l.per_kv), bl = (int)((unsigned)qi / (unsigned)l.q_rows);
  return Row{g * l.group + bl, qi - bl * l.q_rows, kv * l.per_kv + r - qi * l.per_kv};
}

__device__ __forceinline__ int clamp_len(const int32_t* len, int i, int most) {
  return len ? max(0, min(len[i], most)) : most;
}

// One 32-key tile for this wave's 32 rows.  `lim`: keys of the tile below it are visible to the lane's row.  `mixed`:
// only lanes with `mine` take the result (rows of other rollouts keep theirs, whatever this tile's V holds).
// The row's reference is the maximum of the first tile with a visible key; it moves up, and the row's sums are
// rescaled, only when a later score exceeds it by more than 2^HEADROOM.
template <typename T, int DH>
__device__ __forceinline__ void tile_step(const char* kt, const char* vt, const typename Tile<T, DH>::chunk (&q)[Tile<T, DH>::KS],
                                          f32x16 (&o)[Tile<T, DH>::NT], float& m_ref, float& l_run, float qscale, int lim,
                                          bool mixed, bool mine) {
  using TL = Tile<T, DH>;
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  f32x16 s;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
  for (int k = 0; k < TL::KS; ++k) {
    const auto a = *reinterpret_cast<const typename TL::chunk*>(kt + (col * TL::CPR + TL::place(col, 2 * k + half)) * 16);
    s = mfma_chunk<T>(a, q[k], s);
  }
  if (__any(lim < KEYS)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + 4 * half + (r & 3) < lim ? s[r] : -INFINITY;
  }
  float m = -INFINITY;
#pragma unroll
  for (int r = 0; r < 16; ++r) m = fmaxf(m, s[r]);
  m = halves_max(m) * qscale;
  const bool over = m > m_ref + HEADROOM || (m_ref == -INFINITY && m > -INFINITY);
  if (__any(over)) {
    const float f = over ? __builtin_amdgcn_exp2f(m_ref - m) : 1.f;
    l_run *= f;
#pragma unroll
    for (int t = 0; t < TL::NT; ++t) o[t] *= f;
    m_ref = over ? m : m_ref;
  }
  const float ref = m_ref == -INFINITY ? 0.f : m_ref;  // nothing seen yet: every probability is 2^-inf
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], qscale, -ref));
    sum += s[r];
  }
  l_run += sum;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // 16 keys: registers 8u .. 8u + 7
      bf16x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = static_cast<bf16>(s[8 * u + e]);
      // transposed reads: the 16 lanes of a group address 4 keys x 16 dims and get 4 keys of one dim each
      const int grp = lane >> 4, at = lane & 15;
      const int key0 = 16 * u + 4 * half + (at >> 2), dim = 16 * (grp & 1) + 4 * (at & 3);
#pragma unroll
      for (int t = 0; t < TL::NT; ++t) {
        const int c = 4 * t + (dim >> 3), sub = (dim & 4) * 2;
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(vt + (key0 * TL::CPR + TL::place_v(key0, c)) * 16 + sub));
        const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(vt + ((key0 + 8) * TL::CPR + TL::place_v(key0 + 8, c)) * 16 + sub));
        typedef short i16x8 __attribute__((ext_vector_type(8)));
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        const f32x16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, o[t], 0, 0, 0);
        if (mixed) {
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t][r] = mine ? n[r] : o[t][r];
        } else {
          o[t] = n;
        }
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < TL::NT; ++t) {
      f32x16 n = o[t];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = 8 * (r >> 2) + 4 * half + (r & 3), d = 32 * t + col;
        const float v = *reinterpret_cast<const float*>(vt + (key * TL::CPR + TL::place_v(key, d >> 2)) * 16 + (d & 3) * 4);
        n = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[r], n, 0, 0, 0);
      }
      if (mixed) {
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = mine ? n[r] : o[t][r];
      } else {
        o[t] = n;
      }
    }
  }
}

template <typename T, int DH, int NW>
__global__ __launch_bounds__(64 * NW) void k_shared(SharedLaunch l) {
  using TL = Tile<T, DH>;
  constexpr int ROWS = 32 * NW;
  __shared__ __attribute__((aligned(1024))) char lds[2 * TL::BYTES];
  __shared__ int cum[ROWS + 1];  // tail tiles of the rollouts that this row tile touches, summed up
  char* const kt = lds;
  char* const vt = lds + TL::BYTES;

  // items (group, KV head, range, row tile): row tiles of one range are neighbours, and neighbours share an XCD's L2
  const int item = (int)(blockIdx.x % 8) * (int)(gridDim.x / 8) + (int)(blockIdx.x / 8);
  if (item >= l.n_groups * l.n_kv * l.splits * l.row_tiles) return;
  const int rt = item % l.row_tiles, split = item / l.row_tiles % l.splits, gk = item / (l.row_tiles * l.splits);
  const int g = gk / l.n_kv, kv = gk - g * l.n_kv;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, half = lane >> 5;
  const int n_rows = l.group * l.q_rows * l.per_kv, r0 = rt * ROWS;
  const Row me = row_of(l, g, kv, r0 + w * 32 + (lane & 31));

  typename TL::chunk q[TL::KS];
  {
    const char* p = l.q.data + max(me.b, 0) * l.q.outer + me.i * l.q.row + me.h * l.q.head;
#pragma unroll
    for (int k = 0; k < TL::KS; ++k) {
      if (me.b >= 0) q[k] = *reinterpret_cast<const typename TL::chunk*>(p + (2 * k + half) * 16);
      else
#pragma unroll
        for (int e = 0; e < TL::CE; ++e) q[k][e] = (T)0.f;
    }
  }

  // the key sequence: prefix tiles, then the tiles of each rollout's tail
  const int plen = clamp_len(l.plen, g, l.prefix), np = (plen + KEYS - 1) / KEYS;
  const int b0 = g * l.group + r0 / (l.q_rows * l.per_kv);
  const int nb = l.suffix ? g * l.group + (min(r0 + ROWS, n_rows) - 1) / (l.q_rows * l.per_kv) - b0 + 1 : 0;
  if (tid == 0) cum[0] = 0;
  for (int t = tid; t < nb; t += 64 * NW) cum[t + 1] = (clamp_len(l.slen, b0 + t, l.suffix) + KEYS - 1) / KEYS;
  __syncthreads();
  if (tid == 0)
    for (int t = 0; t < nb; ++t) cum[t + 1] += cum[t];
  __syncthreads();
  const int total = np + cum[nb];
  const int t0 = (int)((int64_t)split * total / l.splits), t1 = (int)((int64_t)(split + 1) * total / l.splits);

  f32x16 o[TL::NT];
#pragma unroll
  for (int t = 0; t < TL::NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f;
  const int own_len = me.b >= 0 && l.suffix ? clamp_len(l.slen, me.b, l.suffix) : 0;
  const int own_lim = l.causal ? min(own_len, own_len - l.q_rows + me.i + 1) : own_len;

  int seg = 0;  // rollout of the current tail tile
  for (int t = t0; t < t1; ++t) {
    const char *kb, *vb;
    int64_t kr, vr;
    int n, lim;
    bool mixed = false, mine = true;
    if (t < np) {
      const int j = t * KEYS;
      kr = l.kp.row, vr = l.vp.row;
      kb = l.kp.data + g * l.kp.outer + kv * l.kp.head + j * kr;
      vb = l.vp.data + g * l.vp.outer + kv * l.vp.head + j * vr;
      lim = n = min(KEYS, plen - j);
    } else {
      while (t - np >= cum[seg + 1]) ++seg;
      const int j = (t - np - cum[seg]) * KEYS, b = b0 + seg;
      kr = l.ks.row, vr = l.vs.row;
      kb = l.ks.data + b * l.ks.outer + kv * l.ks.head + j * kr;
      vb = l.vs.data + b * l.vs.outer + kv * l.vs.head + j * vr;
      n = min(KEYS, clamp_len(l.slen, b, l.suffix) - j);
      mine = me.b == b;
      mixed = !__all(mine);
      lim = mine ? own_lim - j : 0;
    }
    __syncthreads();
    for (int c = tid; c < KEYS * TL::CPR; c += 64 * NW) {
      const int r = c / TL::CPR, cc = c - r * TL::CPR;
      u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
      if (r < n) {
        x = *reinterpret_cast<const u32x4*>(kb + r * kr + cc * 16);
        y = *reinterpret_cast<const u32x4*>(vb + r * vr + cc * 16);
      }
      *reinterpret_cast<u32x4*>(kt + (r * TL::CPR + TL::place(r, cc)) * 16) = x;
      *reinterpret_cast<u32x4*>(vt + (r * TL::CPR + TL::place_v(r, cc)) * 16) = y;
    }
    __syncthreads();
    if (__any(lim > 0)) tile_step<T, DH>(kt, vt, q, o, m_ref, l_run, l.qscale, lim, mixed, mine);
  }

  l_run = halves_sum(l_run);
  if (me.b < 0) return;
  const int64_t row = ((int64_t)me.b * l.q_rows + me.i) * l.n_heads + me.h;
  const float ref = m_ref == -INFINITY ? 0.f : m_ref;
  if (l.part) {
    const int64_t at = (int64_t)split * l.n_groups * l.group * l.q_rows * l.n_heads + row;
    if (half == 0) l.stats[at] = l_run == 0.f ? float2{-INFINITY, 0.f} : float2{ref, l_run};
    if (l_run == 0.f) return;
#pragma unroll
    for (int t = 0; t < TL::NT; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<f32x4*>(l.part + at * DH + 32 * t + 8 * k + 4 * half) =
            f32x4{o[t][4 * k], o[t][4 * k + 1], o[t][4 * k + 2], o[t][4 * k + 3]};
    return;
  }
  if (half == 0 && l.lse) l.lse[row] = l_run == 0.f ? -INFINITY : (ref + log2f(l_run)) * LN2;
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  T* out = reinterpret_cast<T*>(const_cast<char*>(l.out.data) + me.b * l.out.outer + me.i * l.out.row + me.h * l.out.head);
  typedef T quad __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int t = 0; t < TL::NT; ++t)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      quad x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(o[t][4 * k + e] * inv);
      *reinterpret_cast<quad*>(out + 32 * t + 8 * k + 4 * half) = x;
    }
}

// Join of a row's ranges, one wave per row: the ranges' sums brought to their largest reference.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_shared_merge(SharedLaunch l) {
  constexpr int N = DH / 64;
  typedef float vec __attribute__((ext_vector_type(N)));
  typedef T tvec __attribute__((ext_vector_type(N)));
  const int64_t rows = (int64_t)l.n_groups * l.group * l.q_rows * l.n_heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int s = 0; s < l.splits; ++s) m = fmaxf(m, l.stats[s * rows + row].x);
  float sum = 0.f;
  vec o;
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = 0.f;
  for (int s = 0; s < l.splits; ++s) {
    const float2 st = l.stats[s * rows + row];
    if (st.x == -INFINITY) continue;  // a range without a visible key wrote nothing
    const float f = __builtin_amdgcn_exp2f(st.x - m);
    sum += st.y * f;
    o += f * *reinterpret_cast<const vec*>(l.part + (s * rows + row) * DH + lane * N);
  }
  const float inv = m == -INFINITY ? 0.f : 1.f / sum;
  const int h = (int)(row % l.n_heads);
  const int64_t qi = row / l.n_heads, b = qi / l.q_rows, i = qi - b * l.q_rows;
  tvec x;
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = from_f32<T>(o[e] * inv);
  *reinterpret_cast<tvec*>(const_cast<char*>(l.out.data) + b * l.out.outer + i * l.out.row + h * l.out.head +
                           lane * N * sizeof(T)) = x;
  if (lane == 0 && l.lse) l.lse[row] = m == -INFINITY ? -INFINITY : (m + log2f(sum)) * LN2;
}

// ---------------------------------------------------------------------------
// weight of the prefix slots
// ---------------------------------------------------------------------------
// A wave keeps 32 keys in registers and reads the rows, 32 at a time, from LDS: S = q K^T puts one key in each lane,
// and the sum over rows stays in its register.  Ranges of rows are summed by k_weight_sum in their order.
struct WeightLaunch {
  SharedLaunch a;  // q, kp, sizes; lse read; splits: ranges of rows
  const float *lse, *w_in;
  float *w_out, *part;  // part: [splits][n_groups][n_kv][prefix] (null: one range)
  float decay;
  int key_tiles;
};

template <typename T, int DH, int NW>
__global__ __launch_bounds__(64 * NW) void k_weight(WeightLaunch l) {
  using TL = Tile<T, DH>;
  __shared__ __attribute__((aligned(1024))) char lds[TL::BYTES];
  __shared__ float lse2[KEYS];
  const SharedLaunch& a = l.a;
  const int item = (int)(blockIdx.x % 8) * (int)(gridDim.x / 8) + (int)(blockIdx.x / 8);
  if (item >= a.n_groups * a.n_kv * l.key_tiles * a.splits) return;
  const int kt = item % l.key_tiles, split = item / l.key_tiles % a.splits, gk = item / (l.key_tiles * a.splits);
  const int g = gk / a.n_kv, kv = gk - g * a.n_kv;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, half = lane >> 5, col = lane & 31;
  const int plen = clamp_len(a.plen, g, a.prefix);
  if (kt * KEYS * NW >= plen) return;
  const int j = (kt * NW + w) * KEYS + col;
  typename TL::chunk key[TL::KS];
  {
    const char* p = a.kp.data + g * a.kp.outer + kv * a.kp.head + (int64_t)min(j, plen - 1) * a.kp.row;
#pragma unroll
    for (int k = 0; k < TL::KS; ++k) key[k] = *reinterpret_cast<const typename TL::chunk*>(p + (2 * k + half) * 16);
  }
  const int n_rows = a.group * a.q_rows * a.per_kv, tiles = (n_rows + KEYS - 1) / KEYS;
  const int t0 = (int)((int64_t)split * tiles / a.splits), t1 = (int)((int64_t)(split + 1) * tiles / a.splits);
  float sum = 0.f;
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    for (int c = tid; c < KEYS * TL::CPR; c += 64 * NW) {
      const int r = c / TL::CPR, cc = c - r * TL::CPR;
      const Row x = row_of(a, g, kv, t * KEYS + r);
      u32x4 v = {0, 0, 0, 0};
      if (x.b >= 0)
        v = *reinterpret_cast<const u32x4*>(a.q.data + x.b * a.q.outer + x.i * a.q.row + x.h * a.q.head + cc * 16);
      *reinterpret_cast<u32x4*>(lds + (r * TL::CPR + TL::place(r, cc)) * 16) = v;
    }
    if (tid < KEYS) {
      const Row x = row_of(a, g, kv, t * KEYS + tid);
      const float v = x.b >= 0 ? l.lse[((int64_t)x.b * a.q_rows + x.i) * a.n_heads + x.h] : -INFINITY;
      lse2[tid] = v == -INFINITY ? INFINITY : v * LOG2E;  // rows that see nothing, or are none, add 2^-inf
    }
    __syncthreads();
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int k = 0; k < TL::KS; ++k) {
      const auto x = *reinterpret_cast<const typename TL::chunk*>(lds + (col * TL::CPR + TL::place(col, 2 * k + half)) * 16);
      s = mfma_chunk<T>(x, key[k], s);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
      sum += __builtin_amdgcn_exp2f(fmaf(s[r], a.qscale, -lse2[8 * (r >> 2) + 4 * half + (r & 3)]));
  }
  sum = halves_sum(sum);
  if (half || j >= plen) return;
  const int64_t at = (int64_t)gk * a.prefix + j;
  if (l.part) l.part[(int64_t)split * a.n_groups * a.n_kv * a.prefix + at] = sum;
  else l.w_out[at] = (l.w_in ? l.decay * l.w_in[at] : 0.f) + sum;
}

__global__ __launch_bounds__(256) void k_weight_sum(WeightLaunch l) {
  const SharedLaunch& a = l.a;
  const int64_t n = (int64_t)a.n_groups * a.n_kv * a.prefix, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= n) return;
  const int gk = (int)(at / a.prefix), j = (int)(at - (int64_t)gk * a.prefix);
  if (j >= clamp_len(a.plen, gk / a.n_kv, a.prefix)) return;
  float sum = 0.f;
  for (int s = 0; s < a.splits; ++s) sum += l.part[s * n + at];
  l.w_out[at] = (l.w_in ? l.decay * l.w_in[at] : 0.f) + sum;
}

// ---------------------------------------------------------------------------
// choices and launches
// ---------------------------------------------------------------------------
View view_of(const jpi_view& v, int es) {
  return View{(const char*)v.data, v.outer * es, v.row * es, v.head * es};
}

SharedLaunch launch_of(const jpi_shared_attn& a) {
  const int es = a.dtype == JPI_BF16 ? 2 : 4;
  SharedLaunch l{};
  l.q = view_of(a.q, es);
  l.kp = view_of(a.k_prefix, es);
  l.vp = view_of(a.v_prefix, es);
  l.ks = view_of(a.k_suffix, es);
  l.vs = view_of(a.v_suffix, es);
  l.out = view_of(a.out, es);
  l.plen = a.prefix_len;
  l.slen = a.suffix_len;
  l.lse = a.lse;
  l.n_groups = a.n_groups;
  l.group = a.group;
  l.q_rows = a.q_rows;
  l.n_heads = a.n_heads;
  l.n_kv = a.n_kv_heads;
  l.per_kv = a.n_heads / a.n_kv_heads;
  l.prefix = a.prefix;
  l.suffix = a.suffix;
  l.causal = a.causal != 0;
  l.qscale = a.scale * LOG2E;
  return l;
}

struct Plan {
  int waves, row_tiles, splits;
};

Plan shared_plan(const jpi_shared_attn& a) {
  const int64_t rows = (int64_t)a.group * a.q_rows * (a.n_heads / a.n_kv_heads);
  Plan p;
  p.waves = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  p.row_tiles = (int)((rows + 32 * p.waves - 1) / (32 * p.waves));
  const int64_t items = (int64_t)a.n_groups * a.n_kv_heads * p.row_tiles;
  const int64_t tiles = (a.prefix + KEYS - 1) / KEYS + (a.suffix + KEYS - 1) / KEYS;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({64, 512 / items, (tiles + 1) / 2}));
  return p;
}

Plan weight_plan(const jpi_shared_attn& a) {
  const int64_t rows = (int64_t)a.group * a.q_rows * (a.n_heads / a.n_kv_heads);
  Plan p;
  p.waves = 4;
  p.row_tiles = (int)((a.prefix + KEYS * p.waves - 1) / (KEYS * p.waves));
  const int64_t items = (int64_t)a.n_groups * a.n_kv_heads * p.row_tiles;
  p.splits = items ? (int)std::max<int64_t>(1, std::min<int64_t>({64, 512 / items, (rows + KEYS - 1) / KEYS})) : 1;
  return p;
}

unsigned grid8(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }

template <typename T, int DH>
hipError_t shared_typed(const jpi_shared_attn& a, void* ws, hipStream_t s) {
  const Plan p = shared_plan(a);
  SharedLaunch l = launch_of(a);
  l.splits = p.splits;
  l.row_tiles = p.row_tiles;
  const int64_t rows = (int64_t)a.n_groups * a.group * a.q_rows * a.n_heads;
  if (p.splits > 1) {
    l.part = (float*)ws;
    l.stats = (float2*)(l.part + p.splits * rows * DH);
  }
  const unsigned grid = grid8((int64_t)a.n_groups * a.n_kv_heads * p.row_tiles * p.splits);
  switch (p.waves) {
    case 1: k_shared<T, DH, 1><<<grid, 64, 0, s>>>(l); break;
    case 2: k_shared<T, DH, 2><<<grid, 128, 0, s>>>(l); break;
    default: k_shared<T, DH, 4><<<grid, 256, 0, s>>>(l); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  k_shared_merge<T, DH><<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(l);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t weight_typed(const jpi_shared_attn& a, const float* w_in, float decay, float* w_out, void* ws, hipStream_t s) {
  if (a.prefix == 0) return hipSuccess;
  const Plan p = weight_plan(a);
  WeightLaunch l{};
  l.a = launch_of(a);
  l.a.splits = p.splits;
  l.lse = a.lse;
  l.w_in = w_in;
  l.w_out = w_out;
  l.decay = decay;
  l.key_tiles = p.row_tiles;
  const int64_t slots = (int64_t)a.n_groups * a.n_kv_heads * a.prefix;
  if (p.splits > 1) l.part = (float*)ws;
  k_weight<T, DH, 4><<<grid8((int64_t)a.n_groups * a.n_kv_heads * p.row_tiles * p.splits), 256, 0, s>>>(l);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  k_weight_sum<<<(unsigned)((slots + 255) / 256), 256, 0, s>>>(l);
  return hipGetLastError();
}

template <typename F>
hipError_t by_type(const jpi_shared_attn& a, F f) {
  if (a.dtype == JPI_BF16) {
    if (a.head_dim == 64) return f(bf16{}, std::integral_constant<int, 64>{});
    if (a.head_dim == 128) return f(bf16{}, std::integral_constant<int, 128>{});
    return f(bf16{}, std::integral_constant<int, 256>{});
  }
  if (a.head_dim == 64) return f(float{}, std::integral_constant<int, 64>{});
  if (a.head_dim == 128) return f(float{}, std::integral_constant<int, 128>{});
  return f(float{}, std::integral_constant<int, 256>{});
}

}  // namespace

size_t shared_attention_bytes(const jpi_shared_attn& a) {
  const Plan p = shared_plan(a);
  if (p.splits == 1) return 0;
  return (size_t)p.splits * a.n_groups * a.group * a.q_rows * a.n_heads * (a.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_shared_attention(const jpi_shared_attn& a, void* ws, hipStream_t s) {
  return by_type(a, [&](auto t, auto dh) { return shared_typed<decltype(t), dh.value>(a, ws, s); });
}

size_t prefix_weight_bytes(const jpi_shared_attn& a) {
  const Plan p = weight_plan(a);
  return p.splits == 1 ? 0 : (size_t)p.splits * a.n_groups * a.n_kv_heads * a.prefix * sizeof(float);
}

hipError_t launch_prefix_weight(const jpi_shared_attn& a, const float* w_in, float decay, float* w_out, void* ws,
                                hipStream_t s) {
  return by_type(a, [&](auto t, auto dh) { return weight_typed<decltype(t), dh.value>(a, w_in, decay, w_out, ws, s); });
}

}  // namespace jpi
