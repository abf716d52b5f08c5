// Attention over a paged cache in 8 bits (jpi_cache_attention, include/jpi_cache.h).
//
// The query rows of a sequence that read one KV head (tokens x the heads on it)
// form one matrix.  Products use matrix instructions in bf16 with the operands
// swapped, S^T = K q^T and O^T = V^T P^T, so that a lane has one query row, and
// the lanes of a row (two or four groups) 16 keys of it each.  Codes are exact in
// bf16 (eight significant bits hold -128 .. 127 and every e4m3 number), so a page's
// scale can wait: that of K goes into the score, that of V into the probability.
// fp32 queries and probabilities are taken in three bf16 parts, whose 24 bits lose
// nothing: three products each at 16 times the fp32 instructions' rate.
//
// The pages' layout gives a lane its operands in pieces of 16 bytes, and what a
// wave asks for lies in runs of 64 bytes and more: 16 dims of a key, 16 keys of a
// dim.  Rows of S^T take the tile's keys in such an order (Tile::key) that a lane's
// 16 scores are of 16 neighbouring keys: one piece of V, one page, one scale.
//
// Few rows (k_cache_attn): tiles of 16 rows; a workgroup's four or eight waves share
// out the keys of one, 64 at a time from memory to registers, and join their sums in
// LDS; where there are few row tiles the keys are cut into ranges as well, by the
// sequence's own length, and joined by a second launch.  Bound by memory where keys
// are many: sixty-four sequences of up to 8192 slots, 8 KV heads of 128 dims, 547 MB,
// 115 us, 4.7 TB/s (a copy reaches 4.8).  Where rows are more, by a SIMD's
// instructions, 4000 cycles a tile of 256 dims, 1500 of them products: eight chunks of
// 50 rows of 8 heads before 866 slots 12.8 us, 2.5 of them before the first tile is
// there and 1.5 for the join.  One row tile before 817 slots of 256 dims takes 11 us in
// eight waves of two tiles each, a chain of counts, table, pages and products (in four
// waves and three ranges 8, and their join 3 more in a launch of its own).
//
// Many rows (k_cache_rows): tiles of 32 rows, four of them sharing the keys that
// direct-to-LDS loads bring, 64 a step, up to three steps ahead.  Bound by the
// instructions between the products: of a step's 310, 1740 cycles of a wave and as
// many of the SIMD's other one in 3700, 128 widen codes, 33 scale, 32 are powers at a
// quarter of the rate, 30 add up and 28 look for the maximum; products take 1024.
// 4096 rows of 32 heads on 8 of 128 before 4096 keys 0.97 PFLOP/s, a window of 1024
// over 4099 tokens 89 us, 0.68 PFLOP/s of what is seen (a library product of 8192^3
// reaches 1.2).
#include <algorithm>
#include <type_traits>

#include "jpi_cache_device.h"

namespace jpi {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int RING_WAVES = 4, GROUP_ROWS = 32 * RING_WAVES;  // rows of a workgroup of the ring
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr float HEADROOM = 16.f;  // log2 of the most that a probability may exceed its row's reference by

// n / by for 0 <= n < 2^31, by a product with 2^(31 + l) / by rounded up, 2^l >= by: a chain of thirty instructions is ahead of
// a kernel's first load for each division that it makes itself
struct Divisor {
  u32 mul;
  int shift;
};
__host__ __device__ __forceinline__ int operator/(int n, Divisor d) { return (int)(((uint64_t)(u32)n * d.mul) >> d.shift); }
Divisor divisor(int64_t by) {
  int l = 0;
  while ((int64_t)1 << l < by) ++l;
  return {(u32)((((uint64_t)1 << (31 + l)) + by - 1) / by), 31 + l};
}

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
  int splits, waves, pairs, per_tile;  // pairs: sequences times KV heads; per_tile: rows of a tile, as far as there are
  Divisor by_splits, by_pairs, by_kv, by_group, by_per_tile;
  float* part;    // [workgroup][rows of a tile][head_dim]
  float2* stats;  // [workgroup][rows of a tile]: reference, sum
};

// What some rows see, in tiles of keys: the first `sink_tiles` and those from lo_tile on, `count` in all; but for the first
// `sinks` slots those from lo up to hi
struct Span {
  int len, nq, rows, i0, i1, pos0, lo, hi, sink_tiles, lo_tile, count;
  __device__ __forceinline__ int tile(int n) const { return n < sink_tiles ? n : n - sink_tiles + lo_tile; }
};

// of rows nth * ROWS and the next ROWS - 1 of a (sequence, KV head)
template <int ROWS, int KEYS>
__device__ __forceinline__ Span span_of(const CacheArgs& a, int s, int nth) {
  Span x;
  x.len = clamp_len(a.len[s], a.cap);
  x.nq = a.q_len ? clamp_len(a.q_len[s], a.q_rows) : a.q_rows;
  x.rows = x.nq * a.group;
  x.i0 = nth * ROWS / a.by_group;
  x.i1 = min(x.nq - 1, (nth * ROWS + ROWS - 1) / a.by_group);
  x.pos0 = x.len - x.nq;
  x.hi = a.causal ? min(max(x.pos0 + x.i1 + 1, 0), x.len) : x.len;
  x.lo = a.window ? (int)max((int64_t)x.pos0 + x.i0 - a.window + 1, (int64_t)0) : 0;
  const int hi_tile = (x.hi + KEYS - 1) / KEYS;
  x.lo_tile = min(x.lo / KEYS, hi_tile);
  x.sink_tiles = a.window ? min((min(a.sinks, x.hi) + KEYS - 1) / KEYS, x.lo_tile) : 0;
  x.count = x.sink_tiles + hi_tile - x.lo_tile;
  return x;
}

// Tiles of a range, and how many ranges have any (one at least): a wave gets a tile each where there are as many
__device__ __forceinline__ int per_range(const CacheArgs& a, int count) { return max((count + a.splits - 1) / a.by_splits, a.waves); }
__device__ __forceinline__ int ranges_of(int count, int per) { return max(1, (count + per - 1) / per); }

// One matrix instruction of R rows (queries) and R keys or dims
template <int R>
struct Tile;
template <>
struct Tile<32> {
  typedef f32x16 acc;
  static __device__ __forceinline__ acc mfma(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // the tile's key that row i of a product takes, and the dim of register 4 quad of O^T in lane group g
  static __device__ __forceinline__ int key(int i, int) { return ((i >> 2) & 1) * 16 + (i >> 3) * 4 + (i & 3); }
  static __device__ __forceinline__ int dim(int quad, int g) { return 8 * quad + 4 * g; }
};
template <>
struct Tile<16> {
  typedef f32x4 acc;
  static __device__ __forceinline__ acc mfma(bf16x8 a, bf16x8 b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ int key(int i, int set) { return (i >> 2) * 16 + set * 4 + (i & 3); }
  static __device__ __forceinline__ int dim(int quad, int g) { return 16 * quad + 4 * g; }
};

// this lane's value and that of the lane 16 away
__device__ __forceinline__ void quarters(float v, float& a, float& b) {
  const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(u32, v), __builtin_bit_cast(u32, v), false, false);
  const u32 x = p[0], y = p[1];
  a = __builtin_bit_cast(float, x), b = __builtin_bit_cast(float, y);
}
// over the lane groups of a row
template <int R>
__device__ __forceinline__ float groups_max(float v) {
  v = halves_max(v);
  if (R == 32) return v;
  float a, b;
  quarters(v, a, b);
  return fmaxf(a, b);
}
template <int R>
__device__ __forceinline__ float groups_sum(float v) {
  v = halves_sum(v);
  if (R == 32) return v;
  float a, b;
  quarters(v, a, b);
  return a + b;
}

// x in PARTS parts of bf16: the largest first
template <int PARTS>
__device__ __forceinline__ void split8(const float* x, bf16x8 (&part)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float a = x[e], b = x[e + 1];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const bf16x2 both = {(__bf16)a, (__bf16)b};  // one instruction, whose halves are taken as bits
      part[p][e] = both[0], part[p][e + 1] = both[1];
      const u32 bits = __builtin_bit_cast(u32, both);
      a -= __builtin_bit_cast(float, bits << 16), b -= __builtin_bit_cast(float, bits & 0xffff0000u);
    }
  }
}

// bits 0 .. n - 1 of 16
__device__ __forceinline__ u32 below(int n) { return (1u << min(max(n, 0), 16)) - 1; }

// What a step needs of the scales of 16 keys.  Probabilities times V's scale: with a power of two, all that append writes, that
// is a whole number in the exponent, and a factor of the sum of the 16.
struct Scales {
  float f;        // scores to powers of two: K's scale * scale / ln 2
  float e;        // V's scale is 2^e, or 0
  float unscale;  // 2^-e; 0: V's scale is no power of two, or could take a probability out of fp32
  float vs;       // V's scale
};
__device__ __forceinline__ Scales scales_of(float qscale, float ks, float vs) {
  const u32 bits = __builtin_bit_cast(u32, vs);
  const bool power = (bits & 0x807fffffu) == 0 && (bits >> 23) - (127 - 64) <= 128;
  return {qscale * ks, power ? (float)((int)(bits >> 23) - 127) : 0.f, power ? __builtin_bit_cast(float, (254u << 23) - bits) : 0.f, vs};
}

// A wave's row tile: the lane's row, its queries, and the running maximum, sum and O^T of its softmax.  A step takes NT times
// 16 keys of each lane group, one page and one scale each.  Q_LDS: the queries are in LDS, where all waves of a workgroup have the
// same row tile.
template <int DH, bool E4M3, typename T, int R, int NT, bool Q_LDS = false>
struct Rows {
  typedef Code<E4M3> C;
  typedef Tile<R> M;
  // bf16 parts of a query and of a probability.  One part of a probability adds 1.5e-3 to the 1.6e-3 of a bf16 result's own
  // rounding (2.2e-3 of both); two, which add nothing that shows, are taken where memory bounds the kernel, not where products
  // do.  us of the ring, one part and two: a window of 1024 over 4099 tokens 88 and 114, 4096 rows before 4096 keys 281 and 370,
  // 816 rows of 256 dims for eight sequences 46 and 51: a remainder is two instructions of 310 for each of 32 probabilities, and
  // its product half as many matrix instructions again.  fp16 in place of bf16, 93, 288 and 47, holds codes and 11 bits (1.7e-3
  // of both), but no probability below 2^-32 of a row's largest: elements where larger ones meet codes of 0 came out wrong.
  static constexpr int PARTS = sizeof(T) == 2 ? 1 : 3, P_PARTS = sizeof(T) == 4 ? 3 : R == 16 ? 2 : 1;
  static constexpr int G = 64 / R, KEYS = 16 * G * NT;             // lane groups, keys of a step
  static constexpr int SETS = KEYS / R, REGS = R * R / 64;         // products of a step's keys, their registers
  static constexpr int KK = DH / (16 * G), DT = DH / R;            // pieces of a lane's keys and values
  static constexpr int QUADS = DH * R / 256;                       // groups of four dims of a lane
  static constexpr int CHAINS = R == 16 ? 4 : 1;                   // sums whose products take turns: one after the other they wait

  int grp, token, head, see_lo, see_hi, full_lo, full_hi, len, sinks;
  float qscale, m_ref, sum;
  bf16x8 q[PARTS][Q_LDS ? 1 : KK][2];
  const bf16x8* q_lds;  // the lane's first piece
  typename M::acc o[DT];

  // Asks for the queries, before the sequence's counts are there: lanes past its rows have others of the array, or the last.
  // Q_LDS: each of eight waves brings a piece to `lds`, and all may read them after a barrier.
  __device__ __forceinline__ void ask(const CacheArgs& a, int s, int h, int rt, bf16x8* lds = nullptr) {
    const int lane = threadIdx.x & 63, col = lane % R;
    grp = lane / R;
    const int r = min(rt * R + col, a.q_rows * a.group - 1);
    token = r / a.by_group, head = h * a.group + (r - token * a.group);
    const T* p = reinterpret_cast<const T*>(a.q) + s * a.q_outer + token * a.q_row + head * a.q_head + 16 * grp;
    if constexpr (Q_LDS) {
      static_assert(2 * KK == 8 && PARTS == 1, "a wave's piece");
      const int wave = threadIdx.x >> 6;
      lds[wave * 64 + lane] = *reinterpret_cast<const bf16x8*>(p + (wave >> 1) * 16 * G + 8 * (wave & 1));
      q_lds = lds + lane;
      return;
    }
#pragma unroll
    for (int kk = 0; kk < (Q_LDS ? 0 : KK); ++kk)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const T* at = p + kk * 16 * G + 8 * m;
        if constexpr (PARTS == 1) {
          q[0][kk][m] = *reinterpret_cast<const bf16x8*>(at);
        } else {
          float f[8];
          const f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = lo[e], f[4 + e] = hi[e];
          bf16x8 part[PARTS];
          split8<PARTS>(f, part);
#pragma unroll
          for (int i = 0; i < PARTS; ++i) q[i][kk][m] = part[i];
        }
      }
  }

  __device__ __forceinline__ void begin(const CacheArgs& a, const Span& x) {
    len = x.len, sinks = a.sinks, qscale = a.qscale;
    see_hi = a.causal ? min(x.pos0 + token + 1, x.len) : x.len;
    see_lo = a.window ? (int)max((int64_t)x.pos0 + token - a.window + 1, (int64_t)0) : 0;
    // tiles from slot full_lo up to slot full_hi are seen whole by all rows
    full_hi = a.causal ? min(x.pos0 + x.i0 + 1, x.len) : x.len;
    full_lo = a.window ? (int)max((int64_t)x.pos0 + x.i1 - a.window + 1, (int64_t)0) : 0;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < REGS; ++e) o[d][e] = 0.f;
    m_ref = -INFINITY, sum = 0.f;
  }

  // O of 256 dims is in the accumulation registers, which the products take as they are.  Left to itself the compiler had it in
  // the others around the branch that brings it to another reference, and copied it there and back in each step.
  __device__ __forceinline__ void hold() {
    if constexpr (DH == 256 && !Q_LDS) {
#pragma unroll
      for (int d = 0; d < DT; ++d) asm volatile("" : "+a"(o[d]));
    }
  }

  // One step's keys from slot0 on, with the scales of the lane's pieces, in parts that a loop may order as it likes.
  struct Step {
    int slot0;
    bool whole, fast;  // all its keys are seen by all rows; its probabilities carry V's scale in their exponent
    u32 seen[NT];
    Scales sc[NT];
    float p[16 * NT];  // scores, then probabilities times V's scale
    float sum;         // of the probabilities, if fast
  };

  // q k^T of the codes; keys(j, kk) are the pieces
  template <typename KF>
  __device__ __forceinline__ void scores(float (&sc)[16 * NT], KF keys) const {
    typename M::acc c[SETS];
#pragma unroll
    for (int j = 0; j < SETS; ++j)
#pragma unroll
      for (int e = 0; e < REGS; ++e) c[j][e] = 0.f;
    // all sets take a piece before the next: products of one sum have to wait for each other
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j0 = 0; j0 < SETS; j0 += CHAINS) {
          bf16x8 codes[CHAINS];
#pragma unroll
          for (int j = 0; j < CHAINS; ++j) {
            const u32x4 w = keys(j0 + j, kk);
            codes[j] = C::widen8(w[2 * m], w[2 * m + 1]);
          }
#pragma unroll
          for (int i = PARTS - 1; i >= 0; --i)
#pragma unroll
            for (int j = 0; j < CHAINS; ++j) c[j0 + j] = M::mfma(codes[j], Q_LDS ? q_lds[(2 * kk + m) * 64] : q[i][Q_LDS ? 0 : kk][m], c[j0 + j]);
        }
#pragma unroll
    for (int j = 0; j < SETS; ++j)
#pragma unroll
      for (int e = 0; e < REGS; ++e) sc[j * REGS + e] = c[j][e];
  }

  // Masks, and the row's reference.  One path for all steps, with masks aside: with one path for those that are seen whole and
  // one for others, or steps left out, O was copied from register to register in each.
  __device__ __forceinline__ void refer(Step& x) {
    x.whole = x.slot0 + KEYS <= full_hi && (x.slot0 >= full_lo || x.slot0 + KEYS <= sinks);
#pragma unroll
    for (int t = 0; t < NT; ++t) x.seen[t] = 0xffffu;
    if (!x.whole) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int slot = x.slot0 + 16 * (G * t + grp);
        x.seen[t] = below(see_hi - slot) & (~below(see_lo - slot) | below(sinks - slot));
        u32 seen = x.seen[t];
        asm volatile("" : "+v"(seen));
#pragma unroll
        for (int e = 0; e < 16; ++e) x.p[16 * t + e] = seen >> e & 1 ? x.p[16 * t + e] : -INFINITY;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float* y = x.p + 16 * t;
      float t0 = fmaxf(fmaxf(y[0], y[1]), y[2]), t1 = fmaxf(fmaxf(y[3], y[4]), y[5]);
      t0 = fmaxf(fmaxf(t0, y[6]), y[7]), t1 = fmaxf(fmaxf(t1, y[8]), y[9]);
      t0 = fmaxf(fmaxf(t0, y[10]), y[11]), t1 = fmaxf(fmaxf(t1, y[12]), y[13]);
      t0 = fmaxf(fmaxf(t0, t1), fmaxf(y[14], y[15])) * x.sc[t].f;
      t0 = x.seen[t] == 0 ? -INFINITY : t0;  // -inf * 0
      top = fmaxf(top, t0);
    }
    top = groups_max<R>(top);
    const bool low = top > m_ref + HEADROOM || (m_ref == -INFINITY && top > -INFINITY);
    hold();
    if (__any(low)) {
      // A whole number: sums are brought to another reference by a power of two, and differences with it are exact.  Not where
      // probabilities are rounded to one part: the maximum itself makes that of a row's only key 1.
      // Rows whose own is not too low keep it: what is in a row changes no other's bits.
      const float now = !low ? m_ref : P_PARTS == 1 ? top : ceilf(top);
      const float g = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref - now);  // with -inf O and the sum are 0
      sum *= g;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < REGS; ++e) o[d][e] *= g;
      hold();
      m_ref = now;
    }
    // Other scales of V, and masks where K's scale makes no -inf of -inf, are seen to one by one
    int fast = 1;  // no && and ||, which would be branches
#pragma unroll
    for (int t = 0; t < NT; ++t)
      fast &= (int)(x.sc[t].unscale != 0.f) & ((int)x.whole | (int)(x.sc[t].f > 0.f) | (int)(x.seen[t] == 0xffffu));
    x.fast = __all(fast);
  }

  __device__ __forceinline__ void probabilities(Step& x) const {
    const float ref = m_ref == -INFINITY ? 0.f : m_ref;
    x.sum = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float r = x.fast ? ref - x.sc[t].e : ref;
      float part[4];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float& p = x.p[16 * t + e];
        p = __builtin_amdgcn_exp2f(fmaf(p, x.sc[t].f, -r));
        part[e & 3] = e < 4 ? p : part[e & 3] + p;
      }
      x.sum = fmaf((part[0] + part[1]) + (part[2] + part[3]), x.sc[t].unscale, x.sum);
    }
  }

  // The row's sum, and what probabilities() could not do
  __device__ __forceinline__ void settle(Step& x) {
    if (!x.fast) {
      x.sum = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        u32 seen = x.seen[t];
        asm volatile("" : "+v"(seen));  // its tests stay here: 32 of them were made in every step
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float& p = x.p[16 * t + e];
          p = seen >> e & 1 ? p : 0.f;
          x.sum += p;
          p = seen >> e & 1 ? p * x.sc[t].vs : 0.f;  // 0 * NaN
        }
      }
    }
    sum += x.sum;
  }

  // the bytes of a piece of V whose slots, from `slot` on, lie before the length: codes past it may be anything
  __device__ __forceinline__ u32x4 valid(int slot) const {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bytes = min(max(len - slot - 4 * e, 0), 4);
      v[e] = bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1;
    }
    return v;
  }

  // All bits of a piece of V that is there, none where its scale is NaN: in place of a number that names no page another one is
  // read, whose codes may be NaN, and rows that do not see it have probabilities of 0.
  static __device__ __forceinline__ u32 known(const Scales& x) { return x.vs == x.vs ? ~0u : 0u; }

  // O += P V; values(t, d) are V's pieces, without what lies past the length
  template <typename VF>
  __device__ __forceinline__ void add(const Step& x, VF values) {
    bf16x8 pp[NT][2][P_PARTS];
#pragma unroll
    for (int t = 0; t < NT; ++t) split8<P_PARTS>(x.p + 16 * t, pp[t][0]), split8<P_PARTS>(x.p + 16 * t + 8, pp[t][1]);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int d0 = 0; d0 < DT; d0 += CHAINS)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          bf16x8 codes[CHAINS];
#pragma unroll
          for (int d = 0; d < CHAINS; ++d) {
            const u32x4 w = values(t, d0 + d);
            codes[d] = C::widen8(w[2 * m], w[2 * m + 1]);
          }
#pragma unroll
          for (int i = P_PARTS - 1; i >= 0; --i)
#pragma unroll
            for (int d = 0; d < CHAINS; ++d) o[d0 + d] = M::mfma(codes[d], pp[t][m][i], o[d0 + d]);
        }
    hold();
  }

  __device__ __forceinline__ f32x4 quad(int i) const {
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = o[i * 4 / REGS][i * 4 % REGS + e];
    return y;
  }
};

__device__ __forceinline__ float lse_of(float ref, float total) {
  return total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * LN2;
}

template <typename T>
__device__ __forceinline__ void put4(T* out, f32x4 y) {
  if constexpr (sizeof(T) == 2) {
    typedef bf16 b4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<b4*>(out) = b4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
  } else {
    *reinterpret_cast<f32x4*>(out) = y;
  }
}

constexpr int NO_PAGE = -1;  // of slots past the length
// A number that names no page, of slots that are there: they are NaN.  Past the length nothing is seen.
__device__ __forceinline__ float scale_at(const CacheArgs& a, const float* scale, int id, int h, bool there) {
  return (u32)id < (u32)a.n_pages ? scale[(int64_t)id * a.kv + h] : there ? __builtin_nanf("") : 0.f;
}
__device__ __forceinline__ int64_t page_of(const CacheArgs& a, int id, int h) {
  return (int64_t)((u32)id < (u32)a.n_pages ? id : 0) * a.kv + h;
}

// Few rows: the waves of a workgroup share out the keys of one row tile, each from memory to its own registers.
// Two waves of a SIMD leave 256 registers each: with three and 168 the loads of a tile (64 registers of 128 dims) spilled.  Of 256
// dims one wave has 330, or two of them, in a workgroup of eight, 256 each: the queries are then in LDS, and values and half of the
// next keys are asked for when what came before is done with.
template <int DH, bool E4M3, typename T, int R, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DH == 256 && WAVES == 4 ? 1 : 2) void k_cache_attn(CacheArgs a) {
  constexpr bool LATE = DH == 256 && WAVES == 8;
  typedef Rows<DH, E4M3, T, R, 1, LATE> W;
  constexpr int EARLY = LATE ? W::KK / 2 : W::KK;
  typedef typename W::M M;
  constexpr int KEYS = W::KEYS, QUADS = W::QUADS;
  static_assert(QUADS % WAVES == 0 || QUADS < WAVES, "quads of a wave");
  __shared__ __align__(16) f32x4 join[WAVES][QUADS][64];
  __shared__ float2 wave_stats[WAVES][R];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = lane / R, col = lane % R;
  const int rest = (int)blockIdx.x / a.by_pairs, pair = blockIdx.x - rest * a.pairs;
  const int rt = rest / a.by_splits, split = rest - rt * a.splits;
  const int s = pair / a.by_kv, h = pair - s * a.kv;
  W w;
  w.ask(a, s, h, rt, reinterpret_cast<bf16x8*>(join));
  const Span x = span_of<R, 1024 / R>(a, s, rt);
  if (rt * R >= x.rows) return;
  const int per = per_range(a, x.count);
  if (split > 0 && split * per >= x.count) return;
  const int first = split * per + wave, last = min(x.count, (split + 1) * per);
  w.begin(a, x);
  if (LATE) __syncthreads();  // the queries

  const int mask = (1 << a.lg_page) - 1;
  const u32 page_bytes = (u32)DH << a.lg_page;
  const int32_t* table = a.table + s * a.table_stride;
  const int key0 = M::key(col, 0), kpiece = key0 & ~15;  // the keys of all sets lie in one piece
  auto page_at = [&](int slot) { return slot < x.len ? table[slot >> a.lg_page] : NO_PAGE; };
  u32x4 kraw[W::SETS][W::KK], vraw[W::DT];
  auto load_k = [&](int t, int id, int from, int to) {
    const uint8_t* p = a.k + page_of(a, id, h) * page_bytes + (((grp << a.lg_page) + ((t * KEYS + key0) & mask)) << 4);
#pragma unroll
    for (int kk = from; kk < to; ++kk)
#pragma unroll
      for (int j = 0; j < W::SETS; ++j) kraw[j][kk] = *reinterpret_cast<const u32x4*>(p + ((u32)(kk * W::G) << (a.lg_page + 4)) + j * 64);
  };
  auto load_v = [&](int t, int id) {
    const uint8_t* p = a.v + page_of(a, id, h) * page_bytes + (u32)(((t * KEYS + 16 * grp) & mask) * DH + (col << 4));
#pragma unroll
    for (int d = 0; d < W::DT; ++d) vraw[d] = *reinterpret_cast<const u32x4*>(p + d * R * 16);
  };

  // pages of the lane's K and V pieces of the next tile, of V's of the present one, and the present one's scales
  int kid = NO_PAGE, vid = NO_PAGE, vid0 = NO_PAGE;
  float ks = 0.f, vs = 0.f;
  if (first < last) {
    const int t = x.tile(first);
    const int k0 = page_at(t * KEYS + kpiece), v0 = page_at(t * KEYS + 16 * grp);
    if (first + WAVES < last) {
      const int t1 = x.tile(first + WAVES);
      kid = page_at(t1 * KEYS + kpiece), vid = page_at(t1 * KEYS + 16 * grp);
    }
    const bool there = t * KEYS + 16 * grp < x.len;
    ks = scale_at(a, a.k_scale, v0, h, there), vs = scale_at(a, a.v_scale, v0, h, there);
    load_k(t, k0, 0, W::KK);
    if (!LATE) load_v(t, v0);
    vid0 = v0;
  }
  for (int n = first; n < last; n += WAVES) {
    const int t = x.tile(n), next = x.tile(min(n + WAVES, last - 1));
    const bool more = n + WAVES < last;
    const int kid1 = kid, vid1 = vid;
    // asked for before the next tile's loads, so that waiting for them does not wait for those
    if (n + 2 * WAVES < last) {
      const int t2 = x.tile(n + 2 * WAVES);
      kid = page_at(t2 * KEYS + kpiece), vid = page_at(t2 * KEYS + 16 * grp);
    }
    typename W::Step st;
    st.slot0 = t * KEYS, st.sc[0] = scales_of(a.qscale, ks, vs);
    if (LATE) asm volatile("" ::: "memory");  // the queries stay in LDS
    w.scores(st.p, [&](int j, int kk) { return kraw[j][kk]; });
    if (LATE) load_v(t, vid0);
    vid0 = vid1;
    if (more) {
      const bool there = next * KEYS + 16 * grp < x.len;
      ks = scale_at(a, a.k_scale, vid1, h, there), vs = scale_at(a, a.v_scale, vid1, h, there);
      if (!LATE) load_k(next, kid1, 0, W::KK);
    }
    w.refer(st);
    w.probabilities(st);
    w.settle(st);
    if (LATE && more) load_k(next, kid1, 0, EARLY);
    if (st.slot0 + KEYS > x.len) {
      const u32x4 valid = w.valid(st.slot0 + 16 * grp);
#pragma unroll
      for (int d = 0; d < W::DT; ++d) vraw[d] &= valid;
    }
    if (!st.fast) {
      const u32 known = W::known(st.sc[0]);
#pragma unroll
      for (int d = 0; d < W::DT; ++d) vraw[d] &= known;
    }
    w.add(st, [&](int, int d) { return vraw[d]; });
    if (more) {
      if (LATE) load_k(next, kid1, EARLY, W::KK);
      else load_v(next, vid1);
    }
  }

  if (LATE) __syncthreads();  // the queries are done with
  // the waves' sums, brought to one reference and added in their order; each adds and writes its part of the dims
  const float sum = groups_sum<R>(w.sum);
  if (grp == 0) wave_stats[wave][col] = float2{w.m_ref, sum};
#pragma unroll
  for (int i = 0; i < QUADS; ++i) join[wave][i][lane] = w.quad(i);
  __syncthreads();
  float ref = -INFINITY, total = 0.f, g[WAVES];
  float2 st[WAVES];
#pragma unroll
  for (int i = 0; i < WAVES; ++i) st[i] = wave_stats[i][col], ref = fmaxf(ref, st[i].x);
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    g[i] = st[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[i].x - ref);
    total += g[i] * st[i].y;
  }
  if (rt * R + col >= x.rows) return;
  const bool final = x.count <= per;
  if (wave == 0 && grp == 0) {
    if (!final) a.stats[(int64_t)blockIdx.x * R + col] = float2{ref, total};
    else if (a.lse) a.lse[((int64_t)s * a.q_rows + w.token) * a.n_heads + w.head] = lse_of(ref, total);
  }
  const float norm = !final ? 1.f : total == 0.f ? 0.f : 1.f / total;
  float* part = a.part + ((int64_t)blockIdx.x * R + col) * DH;
  T* out = reinterpret_cast<T*>(a.out) + s * a.o_outer + w.token * a.o_row + w.head * a.o_head;
#pragma unroll
  for (int i = 0; i < QUADS; i += WAVES) {
    if (QUADS < WAVES && wave >= QUADS) break;  // 64 dims are four quads
    f32x4 y = join[0][i + wave][lane] * g[0];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) y += join[v][i + wave][lane] * g[v];
    y *= norm;
    const int at = M::dim(i + wave, grp);
    if (!final) put4(part + at, y);
    else put4(out + at, y);
  }
}

// Many rows: each wave has a row tile of its own, and the workgroup's keys pass through a ring in LDS that direct-to-LDS
// loads fill several steps of 64 keys ahead.
template <int DH>
struct Ring {
  static constexpr int KEYS = 64, PIECES = DH / 8;  // KB of a step: K of 32 keys, of the next 32, then V so, in the order of a lane's reads
  static constexpr int LOADS = PIECES / RING_WAVES;      // of a wave for a step
  static constexpr int STAGES = 4;
};

// 16 bytes of each lane to LDS at `to` + 16 * lane.  As assembly, which has no register outputs: loads to LDS that the
// compiler knows of are waited for before any read of LDS.
__device__ __forceinline__ void load_to_lds(const void* p, u32 to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(p)
               : "memory", "m0");
}
// the same from a base that all lanes share
__device__ __forceinline__ void load_to_lds(const void* base, u32 offset, u32 to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(base)
               : "memory", "m0");
}

// What a ring's steps are made of, in LDS: for each 16 keys of the next ones the page's place in the pool and its scales
struct Piece16 {
  Scales sc;
  u32 at;  // page * KV heads + head: 2^32 of them, of 1 KB at least, are more than a device holds
};
constexpr int AHEAD = 16;  // steps of a block of these; two blocks are held

template <int DH, bool E4M3>
__global__ __launch_bounds__(64 * RING_WAVES, DH == 256 ? 1 : 2) void k_cache_rows(CacheArgs a) {
  typedef bf16 T;
  typedef Rows<DH, E4M3, T, 32, 2> W;
  typedef Ring<DH> RG;
  constexpr int R = 32, KEYS = RG::KEYS, STAGE = RG::PIECES * 1024, HALF = RG::LOADS / 2;
  static_assert(RG::PIECES == 2 * (W::KK + W::DT) && RG::LOADS % 2 == 0, "ring shape");
  __shared__ __align__(1024) char ring[RG::STAGES * STAGE];
  __shared__ Piece16 pieces[2][AHEAD][4];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = lane / R, col = lane % R;
  // the last rows of causal ones see most: they come first
  const int nth = gridDim.x - 1 - blockIdx.x, rest = nth / a.by_pairs, pair = nth - rest * a.pairs, s = pair / a.by_kv, h = pair - s * a.kv;
  const int group = rest / a.by_splits, split = rest - group * a.splits, rt = group * RING_WAVES + wave;
  const Span all = span_of<GROUP_ROWS, KEYS>(a, s, group);
  if (group * GROUP_ROWS >= all.rows) return;
  const int per = per_range(a, all.count), first = split * per;
  if (split > 0 && first >= all.count) return;
  const int count = min(per, all.count - first);  // of steps, from `first` on
  // a wave without rows computes others' again; steps left out would have O copied from register to register in each
  const int own = min(rt, (all.rows - 1) / R);
  const Span x = span_of<R, KEYS>(a, s, own);
  W w;
  w.ask(a, s, h, own);
  w.begin(a, x);

  const int32_t* table = a.table + s * a.table_stride;
  auto look_up = [&](int block) {  // by one wave: the pieces of a block of steps
    const int n = block * AHEAD + (lane >> 2);
    if (n >= count) return;
    const int slot = all.tile(first + n) * KEYS + 16 * (lane & 3);
    const bool there = slot < all.len;
    const int id = there ? table[slot >> a.lg_page] : NO_PAGE;
    pieces[block & 1][lane >> 2][lane & 3].sc =
        scales_of(a.qscale, scale_at(a, a.k_scale, id, h, there), scale_at(a, a.v_scale, id, h, there));
    pieces[block & 1][lane >> 2][lane & 3].at = (u32)page_of(a, id, h);
  };
  if (wave == 0) look_up(0);
  if (wave == 1) look_up(1);
  __syncthreads();
  wait_vm<0>();  // the queries are there too: waited for in the loop, they would have it wait for the ring's loads

  const int mask = (1 << a.lg_page) - 1;
  const u32 page_bytes = (u32)DH << a.lg_page;
  const int key0 = W::M::key(col, 0);
  const u32 lds = (u32)(uintptr_t)(__attribute__((address_space(3))) char*)ring + wave * 1024;
  // Load i of a wave is piece wave + 4 i of a step: of K, 32 keys after the other in units of 32 dims, then of V
  u32 tile[RG::LOADS], unit[RG::LOADS];
#pragma unroll
  for (int i = 0; i < RG::LOADS; ++i) {
    const int piece = wave + RING_WAVES * (i % HALF);
    tile[i] = piece / W::KK, unit[i] = piece % W::KK;  // as many units of K as of V
  }
  const bool one_page = a.lg_page >= 6;
  // places of the pieces of the next step to be asked for: read a step before, since what depends on them waits for LDS
  u32 place[RG::LOADS];
  auto look = [&](int n) {
    const Piece16* at = pieces[n / AHEAD & 1][n % AHEAD];
#pragma unroll
    for (int i = 0; i < RG::LOADS; ++i)
      if (i == 0 || !one_page) place[i] = at[one_page ? 0 : 2 * tile[i] + (i < HALF ? key0 >> 4 : grp)].at;
  };
  auto issue = [&](int n, int stage) {
    const int t0 = all.tile(first + n) * KEYS;
    const u32 to = lds + stage * STAGE;
    if (one_page) {  // of all 64 keys: its place is the same for all lanes
      const uint64_t base = (uint64_t)(u32)__builtin_amdgcn_readfirstlane((int)place[0]) * page_bytes;
      const uint8_t *kp = a.k + base + (u32)(t0 & mask) * 16, *vp = a.v + base + (u32)(t0 & mask) * DH;
#pragma unroll
      for (int i = 0; i < RG::LOADS; ++i) {
        if (i < HALF) load_to_lds(kp + ((unit[i] << (a.lg_page + 5)) + tile[i] * 512), (((u32)grp << a.lg_page) + key0) * 16, to + i * RING_WAVES * 1024);
        else load_to_lds(vp + (tile[i] * 32 * DH + unit[i] * 512), grp * 16 * DH + col * 16, to + i * RING_WAVES * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < RG::LOADS; ++i) {
        const int slot = t0 + tile[i] * 32 + (i < HALF ? key0 : 16 * grp);
        const uint64_t base = (uint64_t)place[i] * page_bytes;
        const u32 in = i < HALF ? (((2 * unit[i] + grp) << a.lg_page) + (slot & mask)) * 16 : (slot & mask) * DH + unit[i] * 512 + col * 16;
        load_to_lds((i < HALF ? a.k : a.v) + base + in, to + i * RING_WAVES * 1024);
      }
    }
  };

  constexpr int S = RG::STAGES;
#pragma unroll
  for (int n = 0; n < S - 1; ++n)
    if (n < count) look(n), issue(n, n);
  look(min(S - 1, max(count - 1, 0)));
  // Step n's softmax is between the products of the keys after it and of its own values: those of one fill the time of the other.
  auto arrived = [&](int later) {  // everybody's loads but those of the `later` latest steps are there, and all are done with before
    wait_later<RG::LOADS, S - 2>(later);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto keys_of = [&](int stage) {
    const char* at = ring + stage * STAGE + lane * 16;
    return [at](int j, int kk) { return *reinterpret_cast<const u32x4*>(at + (j * W::KK + kk) * 1024); };
  };
  typename W::Step st;
  arrived(min(S - 2, max(count - 1, 0)));
  if (count > 0) w.scores(st.p, keys_of(0));
  for (int n = 0; n < count; ++n) {
    const int stage = n % S, next = (n + 1) % S;
    arrived(min(S - 3, max(count - 2 - n, 0)));
    if (n % AHEAD == 0 && n > 0 && wave == 0) {  // the block before is done with; seen at the next barrier, used after it
      look_up(n / AHEAD + 1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    if (n + S - 1 < count) issue(n + S - 1, (n + S - 1) % S);
    look(min(n + S, count - 1));
    u32x4 k[2][W::KK];  // asked for before they are needed
    const char* keys = ring + next * STAGE + lane * 16;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int kk = 0; kk < W::KK; ++kk) k[j][kk] = *reinterpret_cast<const u32x4*>(keys + (j * W::KK + kk) * 1024);
    const Piece16* mine = pieces[n / AHEAD & 1][n % AHEAD];
    char* values = ring + stage * STAGE + (2 * W::KK) * 1024 + lane * 16;
    st.slot0 = all.tile(first + n) * KEYS;
    st.sc[0] = mine[grp].sc, st.sc[1] = mine[2 + grp].sc;
    if (st.slot0 + KEYS > all.len) {  // the sequence's last step
#pragma unroll
      for (int i = 0; i < HALF; ++i) {
        u32x4* at = reinterpret_cast<u32x4*>(values + (wave + RING_WAVES * i) * 1024);
        *at &= w.valid(st.slot0 + 32 * tile[i] + 16 * grp);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
    w.refer(st);
    float after[32];
    w.probabilities(st);
    w.scores(after, [&](int j, int kk) { return k[j][kk]; });  // behind the last step of what lies there; not used
    u32x4 v[2][W::DT];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int d = 0; d < W::DT; ++d) v[t][d] = *reinterpret_cast<const u32x4*>(values + (t * W::DT + d) * 1024);
    w.settle(st);
    if (!st.fast) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32 known = W::known(st.sc[t]);
#pragma unroll
        for (int d = 0; d < W::DT; ++d) v[t][d] &= known;
      }
    }
    w.add(st, [&](int t, int d) { return v[t][d]; });
#pragma unroll
    for (int e = 0; e < 32; ++e) st.p[e] = after[e];
  }

  const float total = groups_sum<R>(w.sum), norm = total == 0.f ? 0.f : 1.f / total;
  if (rt * R + col >= x.rows) return;
  if (all.count > per) {
    const int64_t at = (int64_t)((group * a.splits + split) * a.pairs + pair) * GROUP_ROWS + wave * R + col;
    if (grp == 0) a.stats[at] = float2{w.m_ref, total};
#pragma unroll
    for (int i = 0; i < W::QUADS; ++i) put4(a.part + at * DH + W::M::dim(i, grp), w.quad(i));
    return;
  }
  T* out = reinterpret_cast<T*>(a.out) + s * a.o_outer + w.token * a.o_row + w.head * a.o_head;
  if (grp == 0 && a.lse) a.lse[((int64_t)s * a.q_rows + w.token) * a.n_heads + w.head] = lse_of(w.m_ref, total);
#pragma unroll
  for (int i = 0; i < W::QUADS; ++i) put4(out + W::M::dim(i, grp), w.quad(i) * norm);
}

// A row whose keys were cut into ranges, and where range i of it is: that of workgroup (rt * splits + i) * pairs + pair
struct CutRow {
  int s, token, head, ranges;  // ranges 1: nothing to join, 0: no such row
  int64_t at, step;
};
template <int R>
__device__ __forceinline__ CutRow cut_row(const CacheArgs& a, int nth) {
  const int rest = nth / a.by_pairs, pair = nth - rest * a.pairs, rt = rest / a.by_per_tile, col = rest - rt * a.per_tile;
  const int s = pair / a.by_kv, h = pair - s * a.kv;
  const Span x = span_of<R, 64>(a, s, rt);
  const int r = rt * R + col, token = r / a.by_group;
  return {s, token, h * a.group + (r - token * a.group), r < x.rows ? ranges_of(x.count, per_range(a, x.count)) : 0,
          ((int64_t)rt * a.splits * a.pairs + pair) * R + col, (int64_t)a.pairs * R};
}
template <typename T>
__device__ __forceinline__ T* out_of(const CacheArgs& a, const CutRow& x) {
  return reinterpret_cast<T*>(a.out) + x.s * a.o_outer + x.token * a.o_row + x.head * a.o_head;
}

// Few rows: a workgroup takes one, groups of DH / 4 lanes, of four dims each, its ranges in turn, and the groups' sums are
// added in their order.
template <int DH, typename T, int R>
__global__ __launch_bounds__(256) void k_cache_join(CacheArgs a) {
  constexpr int LANES = DH / 4, GROUPS = 256 / LANES;
  __shared__ __align__(16) f32x4 sums[GROUPS][LANES];
  const CutRow x = cut_row<R>(a, blockIdx.x);
  if (x.ranges <= 1) return;
  float ref = -INFINITY, total = 0.f;
  for (int i = threadIdx.x & 63; i < x.ranges; i += 64) ref = fmaxf(ref, a.stats[x.at + i * x.step].x);
  ref = wave_max(ref);
  for (int i = threadIdx.x & 63; i < x.ranges; i += 64) {
    const float2 st = a.stats[x.at + i * x.step];
    total += (st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - ref)) * st.y;
  }
  total = wave_sum(total);
  const int d4 = threadIdx.x % LANES, group = threadIdx.x / LANES;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = group; i < x.ranges; i += GROUPS) {
    const float m = a.stats[x.at + i * x.step].x;
    const float g = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - ref);
    y += g * *reinterpret_cast<const f32x4*>(a.part + (x.at + i * x.step) * DH + 4 * d4);
  }
  sums[group][d4] = y;
  __syncthreads();
  if (group != 0) return;
#pragma unroll
  for (int g = 1; g < GROUPS; ++g) y += sums[g][d4];
  y *= total == 0.f ? 0.f : 1.f / total;
  put4(out_of<T>(a, x) + 4 * d4, y);
  if (threadIdx.x == 0 && a.lse) a.lse[((int64_t)x.s * a.q_rows + x.token) * a.n_heads + x.head] = lse_of(ref, total);
}

// Many rows: DH / 4 lanes take a row, all its ranges.  16384 rows of 128 dims in four ranges: the call 109 us with a workgroup
// for each row, 90 so; 1024 rows in sixteen 39 and 69.
template <int DH, typename T, int R>
__global__ __launch_bounds__(256) void k_cache_join_rows(CacheArgs a, int rows) {
  constexpr int LANES = DH / 4;
  const int d4 = threadIdx.x % LANES;
  const int nth = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (nth >= rows) return;
  const CutRow x = cut_row<R>(a, nth);
  if (x.ranges <= 1) return;
  float ref = -INFINITY, total = 0.f;
  for (int i = 0; i < x.ranges; ++i) ref = fmaxf(ref, a.stats[x.at + i * x.step].x);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < x.ranges; ++i) {
    const float2 st = a.stats[x.at + i * x.step];
    const float g = st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - ref);
    total += g * st.y;
    y += g * *reinterpret_cast<const f32x4*>(a.part + (x.at + i * x.step) * DH + 4 * d4);
  }
  y *= total == 0.f ? 0.f : 1.f / total;
  put4(out_of<T>(a, x) + 4 * d4, y);
  if (d4 == 0 && a.lse) a.lse[((int64_t)x.s * a.q_rows + x.token) * a.n_heads + x.head] = lse_of(ref, total);
}

// the row tiles' R rows in ranges
template <int DH, typename T, int R>
void launch_join(CacheArgs& a, int tiles, hipStream_t s) {
  a.per_tile = std::min(R, a.q_rows * a.group), a.by_per_tile = divisor(a.per_tile);
  const int rows = a.pairs * tiles * a.per_tile;  // below 2^24: cache_attention_fits
  if constexpr (R == GROUP_ROWS) {
    if (rows >= 8192) {
      k_cache_join_rows<DH, T, R><<<(unsigned)(((int64_t)rows * DH / 4 + 255) / 256), 256, 0, s>>>(a, rows);
      return;
    }
  }
  k_cache_join<DH, T, R><<<(unsigned)rows, 256, 0, s>>>(a);
}

template <int DH, bool E4M3, typename T>
void launch_typed(CacheArgs& a, const CachePlan& plan, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (plan.groups) {
      k_cache_rows<DH, E4M3><<<(unsigned)(a.pairs * plan.groups * plan.splits), 64 * RING_WAVES, 0, s>>>(a);
      if (plan.splits > 1) launch_join<DH, T, GROUP_ROWS>(a, plan.groups, s);
      return;
    }
  }
  const unsigned grid = (unsigned)(a.pairs * plan.tiles * plan.splits);
  if constexpr (sizeof(T) == 2) {
    if (plan.waves == 8) k_cache_attn<DH, E4M3, T, 16, 8><<<grid, 512, 0, s>>>(a);
  }
  if (plan.waves == 4) k_cache_attn<DH, E4M3, T, 16, 4><<<grid, 256, 0, s>>>(a);
  if (plan.splits > 1) launch_join<DH, T, 16>(a, plan.tiles, s);
}

template <int DH>
void launch_dim(CacheArgs& a, int code, bool f32, const CachePlan& plan, hipStream_t s) {
  if (code == JPI_E4M3) {
    if (f32) launch_typed<DH, true, float>(a, plan, s);
    else launch_typed<DH, true, bf16>(a, plan, s);
  } else {
    if (f32) launch_typed<DH, false, float>(a, plan, s);
    else launch_typed<DH, false, bf16>(a, plan, s);
  }
}

}  // namespace

CachePlan cache_plan(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  const int group = a.n_heads / p.n_kv_heads;
  const int64_t all = (int64_t)a.q_rows * group, pairs = (int64_t)q.n_seqs * p.n_kv_heads;
  int64_t keys = (int64_t)q.max_pages * p.page;
  if (a.window) keys = std::min<int64_t>(keys, (int64_t)a.window + a.sinks + GROUP_ROWS / group + 2 * 64);
  CachePlan plan{0, 0, 1, 4};
  // The ring from a workgroup for each compute unit on (of 256 dims, which it holds one wave of a SIMD at a time for, from half
  // of that), or where there are so many products that it is worth joining ranges of their keys.  us, ring and other: 1024 rows
  // of 32 heads on 8 of 128, 256 workgroups, 27 and 30; 2048 rows 54 and 86; 512 rows 20 and 13, but before 8192 slots 87 and
  // 130; 256 before 4096 41 and 38; 48, 32 and 16 chunks of 50 rows, 8 heads of 256, 866 slots 43, 42 and 33, 57, 45 and 24; 12,
  // 10 and 4 before 4096, 4096 and 8192 slots 50, 45 and 40, 66, 37 and 39.  fp32 has three times the products and none of its
  // time in what the ring saves: 1024 rows 60 and 43.
  const int64_t groups = (all + GROUP_ROWS - 1) / GROUP_ROWS, steps = (keys + 63) / 64, wgs = groups * pairs;
  const bool enough = wgs >= (p.head_dim == 256 ? 128 : 256);
  if (a.dtype == JPI_BF16 && all >= 64 && (enough || all * pairs / GROUP_ROWS * steps >= (p.head_dim == 256 ? 2400 : 8192))) {
    plan.groups = (int)groups;
    plan.splits = enough ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({16, (p.head_dim == 256 ? 256 : 512) / wgs, steps / 4}));
    return plan;
  }
  // Ranges until there is a workgroup for each unit; two, if they are resident together, where there is enough for both to
  // compute.  us, one and two: 64 rows of 32 heads on 8 of 128 before 8192 slots 32 and 27, 128 rows before 2048 15 and 20; one
  // row of 32 sequences, memory alone, before 4096 51 and 55.
  const int64_t slots = p.head_dim < 256 && all >= 64 && steps >= 64 ? 512 : 256;
  plan.tiles = (int)((all + 15) / 16);
  // Eight waves of 256 dims where a sequence's rows have them compute.  us, four and eight: 16, 8, 5 and one chunk of 50 rows of 8
  // heads 27, 14.6, 16.6 and 12.7, 24, 12.8, 13.7 and 12.3; one of 8 rows 11.7 and 12.1; decoding 32 sequences of 4096 slots 96
  // and 101.  And of all dims where they spare the launch that joins ranges, with two tiles a wave at most: a row before 817 slots
  // of 256 dims 11.3 and 11.5 of the GPU, before 600 and 1024 of 128 8.9 and 7.6, 6.7 and 7.9, in int8 8.0 and 9.5 before 1024,
  // 50 rows before 1024 10.6 and 8.5, and 11 us of the host instead of 15, which a captured graph has no use for.  Not int8 of
  // 256 dims, 12.7 and 15.2 of the GPU, nor fp32, of 128 dims 8.3 and 9.9.
  // All of this goes by the slots that the table has room for: the lengths are on the device.  The row before 817 slots in a table
  // for 1088 and more: four ranges, 9.6 of the GPU and 16 with the host.  Eight chunks of 50 rows of 8 heads before 866 slots: 12.9
  // in tables for up to 6080, 32 in wider ones, which go to the ring.
  const bool bf = a.dtype == JPI_BF16, wide = p.head_dim == 256;
  const bool spares = bf && (!wide || p.code == JPI_E4M3) && steps >= 8 && steps <= 16 && pairs * plan.tiles <= slots / 2;
  if (spares || (bf && wide && all >= 128)) plan.waves = 8;
  plan.splits = spares ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({256, slots / (pairs * plan.tiles), steps / plan.waves}));
  return plan;
}

bool cache_attention_fits(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  const CachePlan plan = cache_plan(a, p, q);
  const int64_t pairs = (int64_t)q.n_seqs * p.n_kv_heads, most = 1 << 24;  // 2^32 threads
  return pairs * (plan.groups + plan.tiles) * plan.splits < most &&
         (plan.splits == 1 || pairs * (plan.groups * GROUP_ROWS + plan.tiles * 16) < most);
}

// rows of all ranges
static int64_t part_rows(const CachePlan& plan, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  return plan.splits == 1 ? 0 : (int64_t)q.n_seqs * p.n_kv_heads * (plan.groups * GROUP_ROWS + plan.tiles * 16) * plan.splits;
}

size_t cache_attention_bytes(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q) {
  return (size_t)part_rows(cache_plan(a, p, q), p, q) * (p.head_dim * sizeof(float) + sizeof(float2));
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
  a.splits = plan.splits, a.waves = plan.waves, a.pairs = q.n_seqs * p.n_kv_heads;
  a.by_splits = divisor(a.splits), a.by_pairs = divisor(a.pairs), a.by_kv = divisor(a.kv), a.by_group = divisor(a.group);
  a.part = (float*)ws;
  a.stats = (float2*)((float*)ws + part_rows(plan, p, q) * p.head_dim);
  const bool f32 = c.dtype == JPI_F32;
  switch (p.head_dim) {
    case 64: launch_dim<64>(a, p.code, f32, plan, s); break;
    case 128: launch_dim<128>(a, p.code, f32, plan, s); break;
    default: launch_dim<256>(a, p.code, f32, plan, s);
  }
  return hipGetLastError();
}

}  // namespace jpi
