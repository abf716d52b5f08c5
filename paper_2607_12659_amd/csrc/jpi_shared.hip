// Attention of a batch that shares a prefix, and the weight of its slots
// (jpi_shared_attention, jpi_prefix_weight, include/jpi_prefix.h).
//
// All query rows of a group that read one KV head (rollouts x query rows x the
// heads on that KV head) form one matrix against one key sequence: the prefix,
// which every row sees, and behind it the tails of the rollouts, each seen by
// its own rows only.  A workgroup takes 32 rows per wave and a range of tiles of
// that sequence (64 keys in bf16, 32 in fp32), so each prefix tile that it loads
// serves all its rows, whichever rollouts they belong to.  A running maximum and
// sum per row give the softmax in one pass; ranges of one row tile are joined by
// k_shared_merge.
//
// Products use 32 x 32 matrix instructions with the operands swapped:
// S^T = K q^T puts one query row in each lane (lane % 32) and 16 of the tile's
// keys in its registers, register r <-> key 8 (r / 4) + 4 (lane / 32) + r % 4, so
// the row maximum and sum are in-lane but for one lane swap, and P^T is the B
// operand of O^T = V^T P^T without leaving its registers.
//
// What bounds it.  With many rows the products: a tile of 64 keys x 128 rows of
// 256 dims takes a workgroup 1.4 us, 1.5 PFLOP/s if all 256 units had one.  Four
// prefixes of up to 1600 slots against 6400 rows each, 58 us: the workgroups of
// the longest prefix are the call's time, since lengths are on the device when
// ranges are chosen.  With few rows memory: 65536 slots x 8 KV heads of 128 dims
// and 64 tails of up to 512, 107 us, 3.2 TB/s.  A launch of one tile takes 14 us
// whatever its range, 9 of them inside its workgroup (32 rows of 256 dims: 2.9
// until the first tile is there, 1.7 for its scores, 1.4 for the product with V,
// 2.8 for the rows' way out), and the join 4 to 9.
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

// Keys of a tile.  Two 32-key halves in bf16 share the waits, the first reads from LDS and the bookkeeping of a tile, and
// the products of one half fill the latency of the other's; 64 fp32 keys of 256 dims would not leave room for two stages.
template <typename T>
constexpr int KEYS = sizeof(T) == 2 ? 64 : 32;
// Share of a range that a tile of a tail counts for, in prefix tiles.  us with 1, 2 and 3 (and their plans), tails of up to 512
// slots: eight waves (64 samples, 32 heads on 8 of 128 dims, 65536 slots) 126, 111 and 128; four (8 chunks of 50 rows, 8 heads
// of 256, 3200 slots) 46, 37 and 37; two (16 samples, 32 heads on 8 of 128, 16384 slots) 40, 31 and 30; one (32 samples, 8 heads
// on 8 of 64, 8192 slots) 30, 26 and 26, in fp32 65, 80 and 106: there a tail's tile costs what a prefix tile does.
constexpr int TAIL_COST = 2;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr float HEADROOM = 16.f;  // log2 of the most that a probability may exceed its row's reference by

// A tile of R rows (keys, or queries) of DH elements in LDS, in 1 KB pieces of 8 rows x 128 bytes.  A load instruction
// fills a piece lane after lane, and it is fast only where neighbouring lanes ask for neighbouring memory, so rows stay
// whole in a piece and their eight 16-byte chunks are permuted, row by row, such that the lanes of one LDS read share
// out the 64 banks evenly.  A read's address is one of a few bases of its lane plus a constant.
template <typename T, int DH, int R>
struct Tile {
  static constexpr int CE = 16 / sizeof(T);      // elements of a chunk
  static constexpr int CPR = DH / CE;            // chunks of a row
  static constexpr int KS = CPR / 2;             // k-steps: a chunk for each lane half
  static constexpr int NT = DH / 32;             // 32-wide output tiles
  static constexpr int BYTES = R * DH * (int)sizeof(T);
  static constexpr int GROUPS = R / 8;           // of rows
  static constexpr int PIECES = BYTES / 1024;    // piece f: chunks 8 (f / GROUPS) .. + 7 of rows 8 (f % GROUPS) .. + 7
  typedef T chunk __attribute__((ext_vector_type(CE)));
  // Rows of a product over DH (K, or queries) are read 32 at a time at one chunk: chunk c of row r lies at c ^ swz(r).
  static __device__ __forceinline__ int swz(int r) { return (r & 7) ^ (r >> 3 & 1); }
  // V in bf16 is read transposed, 16 lanes addressing 4 keys x 16 dims: keys 4 .. 7, 2 keys apart, change 64-byte halves.
  static __device__ __forceinline__ int swz_v(int r) { return sizeof(T) == 2 ? (r & 2) << 1 : 0; }
  // what chunk `at` of a piece (of row group g) holds: a row of its eight, and a chunk of the row's eight
  static __device__ __forceinline__ int row(int at) { return at >> 3; }
  static __device__ __forceinline__ int col(int g, int at) { return (at & 7) ^ swz(8 * g + (at >> 3)); }
  static __device__ __forceinline__ int col_v(int at) { return (at & 7) ^ swz_v(at >> 3); }
  // the chunk of k-step k that a lane (row 32 hh + lane % 32, half lane / 32) reads: base(lane, k % 4) + step(k, hh)
  static __device__ __forceinline__ int base(int lane, int j) {
    const int r = lane & 31, h = lane >> 5;
    return r * 128 + ((2 * j + h) ^ swz(r)) * 16;
  }
  static constexpr int step(int k, int hh) { return (k >> 2) * GROUPS * 1024 + hh * 4096; }
  // V, bf16: the 8 bytes that a lane addresses for 16-key step u, output tile t and keys 8 z .. of it:
  // base_v(lane, t % 2) + step_v(t, u, z)
  static __device__ __forceinline__ int base_v(int lane, int tp) {
    const int key = 4 * (lane >> 5) + (lane >> 2 & 3);
    return key * 128 + ((tp ^ (key >> 1 & 1)) * 64) + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
  }
  static constexpr int step_v(int t, int u, int z) { return (t >> 1) * GROUPS * 1024 + (2 * u + z) * 1024; }
};

template <typename T>
__device__ __forceinline__ f32x16 mfma_chunk(const typename Tile<T, 64, 32>::chunk& a, const typename Tile<T, 64, 32>::chunk& b,
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

__device__ __forceinline__ u32 uniform(u32 v) { return __builtin_amdgcn_readfirstlane(v); }

struct View {
  const char* data;
  int64_t outer, row, head;  // bytes
};

// n / d for n < 2^31 by a product (round-up method: m = floor(2^32 (2^s - d) / d) + 1 with 2^s >= d)
struct Divisor {
  u32 d, m, s;
  __device__ __forceinline__ u32 of(u32 n) const { return (__umulhi(n, m) + n) >> s; }
};

struct SharedLaunch {
  View q, kp, vp, ks, vs, out;
  const int32_t *plen, *slen;
  float* lse;
  float* part;    // [splits][rows in all][DH]: a range's sum of p v (null: the output is written directly)
  float2* stats;  // [splits][rows in all]: its reference and sum of p
  int n_groups, group, q_rows, n_heads, n_kv, per_kv, prefix, suffix;
  int causal, splits, row_tiles;
  Divisor by_kv_heads, by_rows, by_splits, by_tiles, by_rollout;  // per_kv, q_rows, splits, row_tiles, q_rows * per_kv
  float qscale;  // scale * log2(e): scores in powers of two
};

// Rows of a (group, KV head): r = (rollout of the group * q_rows + query) * per_kv + head of the KV head.
struct Row {
  int b, i, h;  // rollout in the batch, query, head; b < 0: past the last row
};
__device__ __forceinline__ Row row_of(const SharedLaunch& l, int g, int kv, int r) {
  if (r >= l.group * l.q_rows * l.per_kv) return Row{-1, 0, 0};
  const int qi = (int)l.by_kv_heads.of(r), bl = (int)l.by_rows.of(qi);
  return Row{g * l.group + bl, qi - bl * l.q_rows, kv * l.per_kv + r - qi * l.per_kv};
}

__device__ __forceinline__ int clamp_len(const int32_t* len, int i, int most) {
  return len ? max(0, min(len[i], most)) : most;
}

// Rows that do not see a key have probability 0 for it, and 0 * V of the matrix product would carry NaN or infinity of
// its V into them.  In a tile of a tail that not all rows see, such values are therefore taken out of LDS, by each wave in
// the pieces that it loaded, and their keys noted; the rows that see one add its kind to all their elements at the end.
// kinds[3 i ..]: those of keys 32 i .. + 31 with +inf, -inf, NaN.
template <typename T, int DH, int NW>
__device__ __forceinline__ void take_out(char* vt, u32* kinds) {
  using TL = Tile<T, DH, KEYS<T>>;
  constexpr u32 ones = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u, step = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
  constexpr u32 carry = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
  u32x4 x[TL::PIECES / NW];
  u32 hit = 0;
#pragma unroll
  for (int i = 0; i < TL::PIECES / NW; ++i) x[i] = *reinterpret_cast<const u32x4*>(vt + i * NW * 1024);
#pragma unroll
  for (int i = 0; i < TL::PIECES / NW; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) hit |= (x[i][e] & ones) + step;
  if (__all((hit & carry) == 0)) return;
#pragma unroll 1
  for (int i = 0; i < TL::PIECES / NW; ++i) {
    T* v = reinterpret_cast<T*>(vt + i * NW * 1024);
    const int f = (threadIdx.x >> 6) + i * NW, key = 8 * (f % TL::GROUPS) + TL::row(threadIdx.x & 63);
#pragma unroll 1
    for (int e = 0; e < TL::CE; ++e) {
      const float y = (float)v[e];
      if (__builtin_isfinite(y)) continue;
      atomicOr(&kinds[3 * (key >> 5) + (y == INFINITY ? 0 : y == -INFINITY ? 1 : 2)], 1u << (key & 31));
      v[e] = (T)0.f;
    }
  }
}

// what the keys below `lim` among those add to a row
template <int N>
__device__ __forceinline__ float taint_of(const u32* kinds, int lim) {
  bool pos = false, neg = false, nan = false;
#pragma unroll
  for (int i = 0; i < N / 32; ++i) {
    const int rest = lim - 32 * i;
    const u32 seen = rest >= 32 ? ~0u : (1u << max(rest, 0)) - 1;
    pos |= (kinds[3 * i] & seen) != 0, neg |= (kinds[3 * i + 1] & seen) != 0, nan |= (kinds[3 * i + 2] & seen) != 0;
  }
  return nan || (pos && neg) ? __builtin_nanf("") : pos ? INFINITY : neg ? -INFINITY : 0.f;
}

constexpr int SCHED_MFMA = 0x008, SCHED_DS_READ = 0x100;

// V^T operands of one 16-key step and output tile (bf16)
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
__device__ __forceinline__ bf16x8 read_vt(const char* p) {
  typedef short i16x8 __attribute__((ext_vector_type(8)));
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
  const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 1024));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The work of a wave's 32 rows on a tile: S^T = K q^T, the softmax, O^T += V^T P^T.
template <typename T, int DH>
struct Steps {
  static constexpr int N = KEYS<T>, HT = N / 32;  // keys of a tile, 32-key halves
  using TL = Tile<T, DH, N>;
  typedef typename TL::chunk chunk;
  static constexpr bool HALF = sizeof(T) == 2;
  static constexpr int KS = TL::KS, NT = TL::NT;
  static constexpr int QK = KS * HT, PV = NT * 2 * HT;      // products of a tile (bf16)
  // Operands of K, of V (bf16), that are read ahead: a read takes longer than a product.
  static constexpr int AHEAD = QK < 8 ? QK : 8, VA = 4;

  struct State {  // a row in each lane, its keys and dims shared by the lane halves
    f32x16 o[NT];   // sum of p v
    float m_ref;    // reference of the row's probabilities: 2^(s - m_ref)
    float l_run;    // sum of p over this half's keys
  };

  static __device__ __forceinline__ void k_bases(const char* kt, const char* (&kl)[4]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 4; ++j) kl[j] = kt + TL::base(lane, j);
  }
  static __device__ __forceinline__ chunk k_operand(const char* const (&kl)[4], int f) {  // k-step f / HT, half f % HT
    return *reinterpret_cast<const chunk*>(kl[f / HT & 3] + TL::step(f / HT, f % HT));
  }
  static __device__ __forceinline__ void scores(const char* kt, const chunk (&q)[KS], f32x16 (&s)[HT]) {
    const char* kl[4];
    k_bases(kt, kl);
#pragma unroll
    for (int h = 0; h < HT; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[h][r] = 0.f;
#pragma unroll
    for (int f = 0; f < QK; ++f) s[f % HT] = mfma_chunk<T>(k_operand(kl, f), q[f / HT], s[f % HT]);
    if constexpr (HALF) {
      __builtin_amdgcn_sched_group_barrier(SCHED_DS_READ, AHEAD, 0);
#pragma unroll
      for (int f = 0; f < QK; ++f) {
        __builtin_amdgcn_sched_group_barrier(SCHED_MFMA, 1, 0);
        if (f < QK - AHEAD) __builtin_amdgcn_sched_group_barrier(SCHED_DS_READ, 1, 0);
      }
    }
  }
  // Keys from `lim` on are not visible to the row.  Returns the row's largest score in powers of two.
  static __device__ __forceinline__ float mask_max(f32x16 (&s)[HT], int lim, float qscale) {
    const int rest = lim - 4 * ((threadIdx.x & 63) >> 5);
    float m = -INFINITY;
#pragma unroll
    for (int h = 0; h < HT; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[h][r] = 32 * h + 8 * (r >> 2) + (r & 3) < rest ? s[h][r] : -INFINITY;
        m = fmaxf(m, s[h][r]);
      }
    return halves_max(m) * qscale;
  }
  // The row's reference is the maximum of its first tile with a visible key; it moves up, and the row's sums are
  // rescaled, only when a later score exceeds it by more than 2^HEADROOM.
  static __device__ __forceinline__ void settle(State& x, float m) {
    const bool over = m > x.m_ref + HEADROOM || (x.m_ref == -INFINITY && m > -INFINITY);
    if (__any(over)) {
      const float f = over ? __builtin_amdgcn_exp2f(x.m_ref - m) : 1.f;
      x.l_run *= f;
#pragma unroll
      for (int t = 0; t < NT; ++t) x.o[t] *= f;
      x.m_ref = over ? m : x.m_ref;
    }
  }
  static __device__ __forceinline__ void probabilities(State& x, f32x16 (&s)[HT], float qscale) {
    const float ref = x.m_ref == -INFINITY ? 0.f : x.m_ref;  // nothing seen yet: every probability is 2^-inf
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int h = 0; h < HT; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[h][r] = __builtin_amdgcn_exp2f(fmaf(s[h][r], qscale, -ref));
        sum[r & 1] += s[h][r];
      }
    x.l_run += sum[0] + sum[1];
  }
  // 16 keys each: registers 8 (u % 2) .. + 7 of half u / 2 of S^T.  Rounded to bf16, as V is, for the bf16 matrix instructions;
  // half a step of each probability, which leaves outputs 2.0e-3 to 2.3e-3 from 64 bits where fp32 probabilities leave 1.7e-3
  // (the output's own rounding).  Row sums and lse take them in fp32.
  static __device__ __forceinline__ void round_p(const f32x16 (&s)[HT], bf16x8 (&p)[2 * HT]) {
#pragma unroll
    for (int u = 0; u < 2 * HT; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) p[u][e] = static_cast<bf16>(s[u >> 1][8 * (u & 1) + e]);
  }
  // product i with V: output tile, 16-key step; two output tiles take turns, so that no product waits for the last one's sum
  static constexpr int out_tile(int i) { return i / (4 * HT) * 2 + (i & 1); }
  static constexpr int key_step(int i) { return i / 2 % (2 * HT); }
  static __device__ __forceinline__ bf16x8 v_operand(const char* const (&vl)[2], int i) {
    return read_vt(vl[out_tile(i) & 1] + TL::step_v(out_tile(i), key_step(i), 0));
  }
  // O^T += V^T P^T of one tile, P^T in the registers of S^T
  static __device__ __forceinline__ void weigh(State& x, const char* vt, f32x16 (&s)[HT], float qscale) {
    const int lane = threadIdx.x & 63;
    probabilities(x, s, qscale);
    if constexpr (HALF) {
      const char* const vl[2] = {vt + TL::base_v(lane, 0), vt + TL::base_v(lane, 1)};
      bf16x8 p[2 * HT];
      round_p(s, p);
#pragma unroll
      for (int i = 0; i < PV; ++i)
        x.o[out_tile(i)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(vl, i), p[key_step(i)], x.o[out_tile(i)], 0, 0, 0);
      __builtin_amdgcn_sched_group_barrier(SCHED_DS_READ, 2 * VA, 0);
#pragma unroll
      for (int i = 0; i < PV; ++i) {
        __builtin_amdgcn_sched_group_barrier(SCHED_MFMA, 1, 0);
        if (i < PV - VA) __builtin_amdgcn_sched_group_barrier(SCHED_DS_READ, 2, 0);
      }
    } else {
      const char* const vl = vt + (lane >> 5) * 512 + (lane & 31) * 4;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float v = *reinterpret_cast<const float*>(vl + t * 4096 + (r >> 2) * 1024 + (r & 3) * 128);
          x.o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[0][r], x.o[t], 0, 0, 0);
        }
    }
  }
  // One tile's probabilities and product with V, and the scores of the next, a full tile that all rows see (bf16).  A wave
  // has the matrix unit to itself or shares it with one other, so the work is laid out by hand, a product and what fits
  // beside it at a time: while the unit works on the next scores, the probabilities are formed; while it works on V, the
  // maximum of the next scores is found and the ring's loads are issued (`load(i)`, i < PV).  Operands are read from LDS
  // AHEAD and VA products before they are used.
  template <typename F>
  static __device__ __forceinline__ void both(State& x, const char* vt, const char* kt, const chunk (&q)[KS], f32x16 (&s)[HT],
                                              float qscale, F load) {
    const int lane = threadIdx.x & 63;
    const char* kl[4];
    k_bases(kt, kl);
    const char* const vl[2] = {vt + TL::base_v(lane, 0), vt + TL::base_v(lane, 1)};
    const float ref = x.m_ref == -INFINITY ? 0.f : x.m_ref;
    constexpr int E = 16 * HT, PRE = 4;  // probabilities; of them formed while the first operands are on their way
    constexpr int WAIT = 2;              // products with V before the scores are looked at
    chunk kf[AHEAD];
    bf16x8 vf[VA];
    float sum[2] = {0.f, 0.f};
    auto probability = [&](int e) __attribute__((always_inline)) {
      float& y = reinterpret_cast<float*>(&s[e >> 4])[e & 15];
      y = __builtin_amdgcn_exp2f(fmaf(y, qscale, -ref));
      sum[e & 1] += y;
    };
#pragma unroll
    for (int f = 0; f < AHEAD; ++f) kf[f] = k_operand(kl, f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < PRE; ++e) probability(e);
    f32x16 n[HT];
#pragma unroll
    for (int h = 0; h < HT; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) n[h][r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < QK; ++f) {
      n[f % HT] = mfma_chunk<T>(kf[f % AHEAD], q[f / HT], n[f % HT]);
      if (f + AHEAD < QK) kf[f % AHEAD] = k_operand(kl, f + AHEAD);
      if (f >= QK - VA) vf[f - (QK - VA)] = v_operand(vl, f - (QK - VA));
#pragma unroll
      for (int e = PRE + f * (E - PRE) / QK; e < PRE + (f + 1) * (E - PRE) / QK; ++e) probability(e);
      __builtin_amdgcn_sched_barrier(0);
    }
    x.l_run += sum[0] + sum[1];
    bf16x8 p[2 * HT];
    round_p(s, p);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < PV; ++i) {
      x.o[out_tile(i)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % VA], p[key_step(i)], x.o[out_tile(i)], 0, 0, 0);
      if (i + VA < PV) vf[i % VA] = v_operand(vl, i + VA);
      load(i);
      if (i >= WAIT) {
#pragma unroll
        for (int e = (i - WAIT) * (E / 2) / (PV - WAIT) * 2; e < (i + 1 - WAIT) * (E / 2) / (PV - WAIT) * 2; e += 2)
          m = fmaxf(fmaxf(m, n[e >> 4][e & 15]), n[e >> 4][(e & 15) + 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int h = 0; h < HT; ++h) s[h] = n[h];
    if (__any(m * qscale > x.m_ref + HEADROOM)) settle(x, halves_max(m) * qscale);
  }
};

// Loads of a ring stage, K of a tile and V of the tile before it (whose probabilities are formed while the scores of the
// next are), piece f of the two by wave f % NW, as direct-to-LDS loads (16 bytes of
// each lane, written lane after lane; the order inside a piece is made by what each lane asks for).  Every stage has the
// same number of loads, so that waits can count them.
template <typename T, int DH, int NW>
struct Ring {
  using TL = Tile<T, DH, KEYS<T>>;
  static constexpr int PIECES = TL::PIECES;                  // of one operand
  static constexpr int LOADS = 2 * PIECES / NW;              // of one wave and stage
  static constexpr int STAGE = 2 * TL::BYTES;
  static constexpr int FIT = 128 * 1024 / STAGE;
  static constexpr int MOST = 2 + 63 / LOADS;                // the loads of all stages but two are counted in six bits
  static constexpr int NS = FIT < MOST ? (FIT < 8 ? FIT : 8) : (MOST < 8 ? MOST : 8);  // stages
  static_assert(PIECES % NW == 0 && NS >= 2 && (NS - 2) * LOADS < 64, "ring shape");
  // Buffer resource over the valid rows: what lies past row n - 1 is read as zero.
  static __device__ __forceinline__ u32x4 rows(const char* p, u32 stride, int n) {
    const u32 bytes = n > 0 ? (n - 1) * stride + DH * (u32)sizeof(T) : 0;
    return u32x4{uniform((u32)(uintptr_t)p), uniform((u32)((uintptr_t)p >> 32) & 0xffffu), uniform(bytes), 0x00020000u};
  }
  // 16 bytes per lane to LDS at `to` + 16 * lane.  Written as assembly, which has no register outputs, because the compiler
  // makes the transposed LDS reads wait for every direct-to-LDS load that it knows of, the later stages' too.
  static __device__ __forceinline__ void load(u32x4 rsrc, u32 offset, u32 to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform(to)), "v"(offset), "s"(rsrc) : "memory", "m0");
  }
  // What the loads of one stage share, and load u of them.  Load u fills piece w + NW u: its rows are one of ROWS groups
  // of eight, its chunks 128 bytes further on with each piece of the same rows.
  static constexpr int GROUPS = TL::GROUPS, ROWS = NW < GROUPS ? GROUPS / NW : 1;
  struct Issue {
    u32x4 k, v;
    u32 at_k[ROWS], at_v[ROWS];  // byte of the lane's chunk from the tile's first row on
    u32 to;                      // LDS address of the wave's first piece
  };
  static __device__ __forceinline__ Issue prepare(u32 stage, const char* kb, u32 kr, int kn, const char* vb, u32 vr, int vn) {
    int lane = threadIdx.x & 63;
    const int w = uniform(threadIdx.x >> 6);
    asm volatile("" : "+v"(lane));  // the lane's offsets are formed anew for each stage: kept, they cost spills
    Issue x;
    x.k = rows(kb, kr, kn), x.v = rows(vb, vr, vn);
    x.to = uniform(stage + w * 1024);
    u32 k0 = TL::row(lane) * kr + w / GROUPS * 128, v0 = TL::row(lane) * vr + TL::col_v(lane) * 16 + w / GROUPS * 128;
    asm volatile("" : "+v"(k0), "+v"(v0));
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int g = (w + NW * i) % GROUPS;
      x.at_k[i] = k0 + TL::col(g, lane) * 16 + 8 * g * kr;
      x.at_v[i] = v0 + 8 * g * vr;
    }
    return x;
  }
  static __device__ __forceinline__ void forward(u32x4& rsrc, u32 by) {
    const uint64_t p = ((uint64_t)rsrc[1] << 32 | rsrc[0]) + by;
    rsrc[0] = (u32)p, rsrc[1] = (u32)(p >> 32);
  }
  static __device__ __forceinline__ void one(const Issue& x, int u) {
    // with half of the loads each for K and V, whether load u is one of K does not depend on the wave
    const bool is_k = u < LOADS / 2;
    const int i = is_k ? u : u - LOADS / 2;
    const u32 off = (NW > GROUPS ? i * (NW / GROUPS) : i / ROWS) * 128;
    load(is_k ? x.k : x.v, (is_k ? x.at_k[i % ROWS] : x.at_v[i % ROWS]) + off, x.to + u * NW * 1024);
  }
};

// A place in a row tile's key sequence: the prefix's tiles, then those of the rollouts' tails one after another.
// Kept such that a step inside a prefix or tail is a few scalar additions.
struct Walk {
  int seg;  // rollout of the row tile whose tail this is (-1: prefix)
  int n;    // valid keys from the tile's first on; <= 0: past the end
};
struct Source {
  Walk at;
  int tile;       // its number in the sequence
  const char* p;  // its first row of K or V
  u32 stride;     // bytes from row to row
};

template <typename T, int DH, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 8 ? 2 : 1))) void k_shared(SharedLaunch l) {
  using TL = Tile<T, DH, KEYS<T>>;
  using RG = Ring<T, DH, NW>;
  using ST = Steps<T, DH>;
  constexpr int ROWS = 32 * NW, NS = RG::NS, KT = KEYS<T>, KINDS = 3 * (KT / 32);
  __shared__ __attribute__((aligned(1024))) char lds[NS * RG::STAGE + 4 * (2 * ROWS + 1 + NW + 3 * KINDS)];
  int* const cum = reinterpret_cast<int*>(lds + NS * RG::STAGE);  // tail tiles of the rollouts of this row tile, summed up
  int* const wave_sum = cum + ROWS + 1;
  u32* const kinds = reinterpret_cast<u32*>(wave_sum + NW);  // of this tile and the two next (take_out)
  int* const lens = wave_sum + NW + 3 * KINDS;               // of those tails

  // items (group, KV head, range, row tile): row tiles of one range are neighbours, and neighbours share an XCD's L2
  const int item = (int)(blockIdx.x % 8) * (int)(gridDim.x / 8) + (int)(blockIdx.x / 8);
  if (item >= l.n_groups * l.n_kv * l.splits * l.row_tiles) return;
  const int by_tile = (int)l.by_tiles.of(item), rt = item - by_tile * l.row_tiles;
  const int gk = (int)l.by_splits.of(by_tile), split = by_tile - gk * l.splits;
  const int g = gk / l.n_kv, kv = gk - g * l.n_kv;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, half = lane >> 5;
  const int n_rows = l.group * l.q_rows * l.per_kv, r0 = rt * ROWS;

  // lengths and queries are asked for together
  const int first = (int)l.by_rollout.of(r0), b0 = g * l.group + first;
  const int nb = l.suffix ? (int)l.by_rollout.of(min(r0 + ROWS, n_rows) - 1) - first + 1 : 0;
  const int prefix_len = clamp_len(l.plen, g, l.prefix);
  const int some_len = tid < nb ? clamp_len(l.slen, b0 + tid, l.suffix) : 0;
  typename TL::chunk q[TL::KS];
  {
    const Row any = row_of(l, g, kv, min(r0 + w * 32 + (lane & 31), n_rows - 1));  // rows past the last one repeat it
    const char* p = l.q.data + any.b * l.q.outer + any.i * l.q.row + any.h * l.q.head + half * 16;
#pragma unroll
    for (int k = 0; k < TL::KS; ++k) q[k] = *reinterpret_cast<const typename TL::chunk*>(p + k * 32);
  }

  // the key sequence
  const int plen = uniform(prefix_len), np = (plen + KT - 1) / KT;
  if (l.suffix) {
    int c = (some_len + KT - 1) / KT;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int x = __shfl_up(c, d, 64);
      c += lane >= d ? x : 0;
    }
    if (lane == 63) wave_sum[w] = c;
    __syncthreads();
    for (int v = 0; v < w; ++v) c += wave_sum[v];
    if (tid < nb) cum[tid + 1] = c, lens[tid] = some_len;
    if (tid == 0) cum[0] = 0;
    if (tid < 3 * KINDS) kinds[tid] = 0;
    __syncthreads();
  }
  const int total = np + (l.suffix ? __builtin_amdgcn_readfirstlane(cum[nb]) : 0);
  // Ranges of equal time: a tile of a tail takes TAIL_COST times a prefix tile's (it is one wave's or few waves' work).
  const int64_t units = np + (int64_t)TAIL_COST * (total - np);
  auto first_of = [&](int r) {
    const int64_t u = r * units / l.splits;
    return (int)(u <= np ? u : np + (u - np + TAIL_COST - 1) / TAIL_COST);
  };
  const int t0 = first_of(split), t1 = first_of(split + 1);

  typename ST::State x;
#pragma unroll
  for (int t = 0; t < TL::NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) x.o[t][r] = 0.f;
  x.m_ref = -INFINITY, x.l_run = 0.f;
  float taint = 0.f;
  int own_b, own_lim = 0;  // the lane's rollout, and how many keys of its tail its row sees, less the tail's length
  {
    const Row me = row_of(l, g, kv, r0 + w * 32 + (lane & 31));
    own_b = me.b;
    if (me.b >= 0 && l.causal) own_lim = min(0, me.i + 1 - l.q_rows);
  }

  auto tail_len = [&](int seg) { return (int)uniform(lens[seg]); };
  auto seek = [&](int t) {  // tile t
    if (t < np) return Walk{-1, plen - t * KT};
    int lo = 0, hi = nb;  // the tail with cum[lo] <= t - np < cum[lo + 1]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if ((int)uniform(cum[mid]) <= t - np) lo = mid;
      else hi = mid;
    }
    return Walk{lo, tail_len(lo) - (t - np - (int)uniform(cum[lo])) * KT};
  };
  auto step = [&](Walk& y) __attribute__((always_inline)) {  // one tile on; true: into another tail
    y.n -= KT;
    if (y.n > 0) return false;
    while (y.n <= 0 && y.seg + 1 < nb) y.n = tail_len(++y.seg);
    return true;
  };
  auto open = [&](Source& y, bool keys) __attribute__((always_inline)) {  // where its tile lies
    const bool tail = y.at.seg >= 0;
    const View& v = keys ? (tail ? l.ks : l.kp) : (tail ? l.vs : l.vp);
    const int64_t o_at = tail ? b0 + y.at.seg : g, j = (tail ? tail_len(y.at.seg) : plen) - y.at.n;
    y.p = v.data + o_at * v.outer + kv * v.head + j * v.row;
    y.stride = (u32)v.row;
  };
  auto advance = [&](Source& y, bool keys) __attribute__((always_inline)) {
    if (++y.tile <= t0 || y.tile >= t1) return;
    if (step(y.at)) open(y, keys);
    else y.p += KT * y.stride;
  };

  wait_vm<0>();  // the queries are there: waited for in the loop, they would have it wait for the ring's loads too
  if (t0 < t1) {
    Walk cur = seek(t0);
    Source ks{cur, t0}, vs{cur, t0 - 1};
    open(ks, true);
    open(vs, false);
    // One stage more, as long as V of some tile is to come: K of nothing past the last tile, V of nothing before the first.
    auto load = [&](int stage) __attribute__((always_inline)) {
      if (vs.tile >= t1) return;
      const auto y = RG::prepare((u32)(uintptr_t)(dma_lds_t*)lds + stage * RG::STAGE, ks.p, ks.stride,
                                 ks.tile < t1 ? min(ks.at.n, KT) : 0, vs.p, vs.stride, vs.tile >= t0 ? min(vs.at.n, KT) : 0);
#pragma unroll
      for (int u = 0; u < RG::LOADS; ++u) RG::one(y, u);
      advance(ks, true);
      advance(vs, false);
    };
    for (int u = 0; u < NS - 1; ++u) load(u);
    int stage = 0, taken = 0;
    const bool partly = nb > 1 || l.causal;  // rows may not see all of a tail's tile
    auto next_stage = [&](auto full_ring, u32* here) __attribute__((always_inline)) -> char* {
      // of the stages asked for, vs.tile - (t0 - 1), those after the next one may still be on their way
      if constexpr (decltype(full_ring)::value) wait_vm<(NS - 2) * RG::LOADS>();
      else wait_later<RG::LOADS, NS - 2>(vs.tile - t0 - taken);
      if (here) {
        take_out<T, DH, NW>(lds + stage * RG::STAGE + TL::BYTES + tid * 16, here);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      // every wave's loads of this stage have landed, and every wave is done with the stage before it, which is free
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      char* const at = lds + stage * RG::STAGE;
      stage = stage == NS - 1 ? 0 : stage + 1;
      ++taken;
      return at;
    };
    const std::false_type some{};
    auto freed = [&]() { return stage < 2 ? stage + NS - 2 : stage - 2; };  // the stage before the one just taken
    auto limit = [&](const Walk& y) { return y.seg < 0 ? y.n : own_b == b0 + y.seg ? y.n + own_lim : 0; };

    f32x16 s[ST::HT];
    int lim = limit(cur);
    bool have = __any(lim > 0);  // whether some row sees a key of the tile: its scores are in s
    {
      const char* const at = next_stage(some, nullptr);
      load(freed());
      if (have) {
        ST::scores(at, q, s);
        x.m_ref = ST::mask_max(s, lim, l.qscale);
      }
    }
    int t = t0;
    if constexpr (ST::HALF) {
      // full tiles of the prefix
      const int full = min(plen / KT, t1), start = t;
      if (t + 1 < full && ks.tile < full) {  // so are the tiles loaded next: their loads differ by a step of the addresses
        auto is = RG::prepare(0, ks.p, ks.stride, KT, vs.p, vs.stride, KT);
        const u32 first = is.to, k_step = KT * ks.stride, v_step = KT * vs.stride;
        const int run = full - ks.tile;  // t + run < full: a tile of K is loaded before its scores are wanted
        for (int r = 0; r < run; ++r) {
          const char* const at = next_stage(std::true_type{}, nullptr);
          is.to = first + freed() * RG::STAGE;
          ST::both(x, at + TL::BYTES, at, q, s, l.qscale, [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int u = i * RG::LOADS / ST::PV; u < (i + 1) * RG::LOADS / ST::PV; ++u) RG::one(is, u);
          });
          RG::forward(is.k, k_step);
          RG::forward(is.v, v_step);
        }
        t += run;
        ks.p += (int64_t)run * k_step, vs.p += (int64_t)run * v_step;
        ks.at.n -= run * KT, vs.at.n -= run * KT;
        ks.tile += run, vs.tile += run;
        if (ks.at.n <= 0 && ks.tile < t1) {  // the prefix ended with a full tile
          ks.at.n += KT;
          step(ks.at);
          open(ks, true);
        }
      }
      for (; t + 1 < full; ++t) {
        const char* const at = next_stage(some, nullptr);
        load(freed());
        ST::both(x, at + TL::BYTES, at, q, s, l.qscale, [](int) {});
      }
      cur.n -= (t - start) * KT;
      lim = limit(cur);
    }
    for (; t < t1; ++t) {
      const bool check = cur.seg >= 0 && partly;
      u32* const here = kinds + KINDS * (t % 3);
      const char* const at = next_stage(some, check ? here : nullptr);
      load(freed());
      if (check) {
        u32 any = 0;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) any |= here[i];
        if (any) taint += taint_of<KT>(here, lim);
        // read last before this tile's barrier, noted in first after the next one's
        if (tid < KINDS) kinds[KINDS * ((t + 2) % 3) + tid] = 0;
      }
      if (have) ST::weigh(x, at + TL::BYTES, s, l.qscale);
      if (t + 1 < t1) {
        step(cur);
        lim = limit(cur);
        have = __any(lim > 0);
        if (have) {
          ST::scores(at, q, s);
          ST::settle(x, ST::mask_max(s, lim, l.qscale));
        }
      }
    }
    wait_vm<0>();  // no load is in flight into LDS when the workgroup ends
  }

  // The rows leave through the ring's memory, 32 x DH fp32 of each wave, so that stores are whole rows: chunk c (4 dims)
  // of row r at c ^ r % 16.  With several ranges that is the sum of p v, else the output.
  const float l_run = halves_sum(x.l_run);
  const Row me = row_of(l, g, kv, r0 + w * 32 + (lane & 31));
  const int64_t row = ((int64_t)me.b * l.q_rows + me.i) * l.n_heads + me.h;
  const int64_t at = (int64_t)split * l.n_groups * l.group * l.q_rows * l.n_heads + row;
  const float ref = x.m_ref == -INFINITY ? 0.f : x.m_ref;
  const float inv = l.part ? 1.f : l_run == 0.f ? 0.f : 1.f / l_run;
  if (half == 0 && me.b >= 0) {
    if (l.part) l.stats[at] = l_run == 0.f ? float2{-INFINITY, 0.f} : float2{ref, l_run};
    else if (l.lse) l.lse[row] = l_run == 0.f ? -INFINITY : (ref + log2f(l_run)) * LN2;
  }
  static_assert(NS * RG::STAGE >= NW * 32 * DH * 4, "room for the rows");
  constexpr int CH = DH / 4;  // chunks of a row
  __syncthreads();
  f32x4* const mine = reinterpret_cast<f32x4*>(lds + w * 32 * DH * 4);
#pragma unroll
  for (int t = 0; t < TL::NT; ++t)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x4 y = {x.o[t][4 * k], x.o[t][4 * k + 1], x.o[t][4 * k + 2], x.o[t][4 * k + 3]};
      const int r = lane & 31;
      mine[r * CH + ((8 * t + 2 * k + half) ^ (r & 15))] = y * inv + taint;
    }
  typedef T quad __attribute__((ext_vector_type(4)));
  int64_t base = l.part ? (int64_t)(uintptr_t)(l.part + at * DH)
                        : (int64_t)(uintptr_t)l.out.data + me.b * l.out.outer + me.i * l.out.row + me.h * l.out.head;
  if (me.b < 0) base = 0;
  constexpr int RW = 64 / CH;       // rows of one store
  const int c = lane % CH, sub = lane / CH;
  auto leave = [&](auto part) __attribute__((always_inline)) {
    constexpr int U = 8;
#pragma unroll 1
    for (int r0 = 0; r0 < 32; r0 += U * RW) {
      f32x4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * RW + sub;
        y[u] = mine[r * CH + (c ^ (r & 15))];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int64_t to = 0;
#pragma unroll
        for (int j = 0; j < RW; ++j) {
          const int r = r0 + u * RW + j;
          const u32 lo = __builtin_amdgcn_readlane((u32)base, r), hi = __builtin_amdgcn_readlane((u32)((uint64_t)base >> 32), r);
          if (sub == j) to = (int64_t)((uint64_t)hi << 32 | lo);
        }
        if (to == 0) continue;
        if constexpr (decltype(part)::value) *reinterpret_cast<f32x4*>(to + c * 16) = y[u];
        else *reinterpret_cast<quad*>(to + c * 4 * sizeof(T)) = quad{from_f32<T>(y[u][0]), from_f32<T>(y[u][1]), from_f32<T>(y[u][2]), from_f32<T>(y[u][3])};
      }
    }
  };
  if (l.part) leave(std::true_type{});
  else leave(std::false_type{});
}

// Join of a row's ranges: the ranges' sums brought to their largest reference.  WPR waves a row, each for a part of the
// ranges (at most 64): with one, 64 ranges of few rows would be sixteen trips to memory one after another, with four, four.
template <typename T, int DH, int WPR>
__global__ __launch_bounds__(WPR > 4 ? 64 * WPR : 256) void k_shared_merge(SharedLaunch l) {
  constexpr int N = DH / 64, RPW = WPR < 4 ? 4 / WPR : 1;  // rows of a workgroup
  typedef float vec __attribute__((ext_vector_type(N)));
  typedef T tvec __attribute__((ext_vector_type(N)));
  __shared__ vec parts[WPR > 1 ? WPR : 1][64];
  __shared__ float2 stats[WPR];
  const int64_t rows = (int64_t)l.n_groups * l.group * l.q_rows * l.n_heads;
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), share = w % WPR;
  const int64_t row = (int64_t)blockIdx.x * RPW + w / WPR;
  if (row >= rows) return;  // WPR > 1: all of the workgroup
  const int s0 = share * l.splits / WPR, n = (share + 1) * l.splits / WPR - s0;
  const float2 st = lane < n ? l.stats[(s0 + lane) * rows + row] : float2{-INFINITY, 0.f};
  float m = wave_max(st.x);
  const float f = st.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.x - m);
  float sum = wave_sum(st.x == -INFINITY ? 0.f : st.y * f);
  const unsigned long long there = __ballot(st.x != -INFINITY);  // a range without a visible key wrote nothing
  vec o;
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = 0.f;
  constexpr int U = 4;  // loads in flight; where fewer ranges are left, the last one again
  const float* const at = l.part + (s0 * rows + row) * DH + lane * N;
  for (int s = 0; s < n; s += U) {
    vec v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const vec*>(at + min(s + u, n - 1) * rows * DH);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = s + u < n && (there >> (s + u) & 1);
      const float g = on ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), min(s + u, 63))) : 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) o[e] = fmaf(g, on ? v[u][e] : 0.f, o[e]);
    }
  }
  if constexpr (WPR > 1) {
    parts[share][lane] = o;
    if (lane == 0) stats[share] = float2{m, sum};
    __syncthreads();
    if (share) return;
#pragma unroll
    for (int i = 1; i < WPR; ++i) m = fmaxf(m, stats[i].x);
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      const float g = stats[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stats[i].x - m);
      sum = fmaf(g, stats[i].y, sum);
      if (g != 0.f) o += parts[i][lane] * g;
    }
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
// A wave keeps 64 keys (fp32 heads of 256: 32) in registers and takes the rows, 32 at a time, from LDS: S = q K^T puts one
// key in each lane and 16 rows in its registers, so the sum over rows stays in a register, and a read of a row from LDS
// serves two products.  65536 slots x 8 KV heads of 128 dims against 256 rows take 52 us: 28 to read the keys, which only
// partly overlap the 33 of products and exponentials (the loop's slope over more rows).  A workgroup's range of rows has
// its lse in LDS from the start, as the exponent's summand; ranges are summed by k_weight_sum in their order.
struct WeightLaunch {
  SharedLaunch a;  // q, kp, sizes; splits: ranges of rows
  const float *lse, *w_in;
  float *w_out, *part;  // part: [splits][n_groups][n_kv][prefix] (null: one range)
  float decay;
  int key_tiles;
};

constexpr int WEIGHT_WAVES = 4;
constexpr int WEIGHT_ROWS = 2048;  // rows of a range at most

template <typename T, int DH>
struct WeightShape {
  using TL = Tile<T, DH, 32>;
  static constexpr int KT = sizeof(T) == 4 && DH == 256 ? 1 : 2;  // 32-key tiles of a wave
  static constexpr int KEYS_WG = 32 * KT * WEIGHT_WAVES;
  static constexpr int NS = 4;                                    // stages of rows; the same memory first takes the keys
  static constexpr int LOADS = TL::PIECES / WEIGHT_WAVES;         // of one wave and stage
};

template <typename T, int DH>
__global__ __launch_bounds__(64 * WEIGHT_WAVES) __attribute__((amdgpu_waves_per_eu(2))) void k_weight(WeightLaunch l) {
  using TL = Tile<T, DH, 32>;
  using WS = WeightShape<T, DH>;
  constexpr int NW = WEIGHT_WAVES, NS = WS::NS, KT = WS::KT;
  static_assert(NW == 4 && NS >= NW, "a wave's pieces are eight rows of all chunks; each wave stages its keys");
  __shared__ __attribute__((aligned(1024))) char lds[NS * TL::BYTES];
  __shared__ float lse2[WEIGHT_ROWS];
  const SharedLaunch& a = l.a;
  const int item = (int)(blockIdx.x % 8) * (int)(gridDim.x / 8) + (int)(blockIdx.x / 8);
  if (item >= a.n_groups * a.n_kv * l.key_tiles * a.splits) return;
  const int kt = item % l.key_tiles, split = item / l.key_tiles % a.splits, gk = item / (l.key_tiles * a.splits);
  const int g = gk / a.n_kv, kv = gk - g * a.n_kv;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), half = lane >> 5, col = lane & 31;
  const int plen = uniform(clamp_len(a.plen, g, a.prefix));
  if (kt * WS::KEYS_WG >= plen) return;
  const u32 ring = (u32)(uintptr_t)(dma_lds_t*)lds;
  auto load = [&](const char* p, u32 to) __attribute__((always_inline)) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(uniform(to)), "v"(p) : "memory", "m0");
  };

  // keys into registers, by way of LDS so that whole lines are asked for
  const int key0 = kt * WS::KEYS_WG + w * 32 * KT;
  typename TL::chunk key[KT][TL::KS];
#pragma unroll
  for (int u = 0; u < KT; ++u) {
#pragma unroll
    for (int f = 0; f < TL::PIECES; ++f) {
      const int r = min(key0 + u * 32 + 8 * (f & 3) + TL::row(lane), plen - 1);
      load(a.kp.data + g * a.kp.outer + kv * a.kp.head + (int64_t)r * a.kp.row + (8 * (f >> 2) + TL::col(f & 3, lane)) * 16,
           ring + w * TL::BYTES + f * 1024);
    }
    wait_vm<0>();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int k = 0; k < TL::KS; ++k)
      key[u][k] = *reinterpret_cast<const typename TL::chunk*>(lds + w * TL::BYTES + TL::base(lane, k & 3) + TL::step(k, 0));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  const int n_rows = a.group * a.q_rows * a.per_kv, tiles = (n_rows + 32 - 1) / 32;
  const int t0 = (int)((int64_t)split * tiles / a.splits), t1 = (int)((int64_t)(split + 1) * tiles / a.splits);
  bool silent = false;  // a row that adds nothing, whatever its queries hold
  for (int r = tid; r < (t1 - t0) * 32; r += 64 * NW) {
    const Row x = row_of(a, g, kv, t0 * 32 + r);
    const float v = x.b >= 0 ? l.lse[((int64_t)x.b * a.q_rows + x.i) * a.n_heads + x.h] : -INFINITY;
    // rows that see nothing, or are none, add 2^-inf.  The product's rounding is 2^-24 of the summand (about 15 for a long
    // prefix), 6e-7 of a weight at most; sums of 3200 rows come out 9.0e-8 from 64 bits, 7.3e-8 where lse is subtracted first
    lse2[r] = v == -INFINITY ? -INFINITY : -v * LOG2E;
    silent = silent || (x.b >= 0 && v == -INFINITY);
  }
  const bool some_silent = __syncthreads_or(silent);

  auto rows = [&](int t, int stage) __attribute__((always_inline)) {  // past the last tile: the last row again
    const Row x = row_of(a, g, kv, min(t * 32 + 8 * w + TL::row(lane), n_rows - 1));
    const char* p = a.q.data + x.b * a.q.outer + x.i * a.q.row + x.h * a.q.head + TL::col(w, lane) * 16;
#pragma unroll
    for (int i = 0; i < WS::LOADS; ++i) load(p + i * 128, ring + stage * TL::BYTES + (w + NW * i) * 1024);
  };
#pragma unroll
  for (int u = 0; u < NS - 1; ++u) rows(t0 + u, u);
  float sum[KT][2] = {};
  int stage = 0;
  for (int t = t0; t < t1; ++t) {
    wait_vm<(NS - 2) * WS::LOADS>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    rows(t + NS - 1, stage == 0 ? NS - 1 : stage - 1);
    const char* const at = lds + stage * TL::BYTES;
    stage = stage == NS - 1 ? 0 : stage + 1;
    f32x16 s[KT];
#pragma unroll
    for (int u = 0; u < KT; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
#pragma unroll
    for (int k = 0; k < TL::KS; ++k) {
      const auto x = *reinterpret_cast<const typename TL::chunk*>(at + TL::base(lane, k & 3) + TL::step(k, 0));
#pragma unroll
      for (int u = 0; u < KT; ++u) s[u] = mfma_chunk<T>(x, key[u][k], s[u]);
    }
    f32x4 e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = *reinterpret_cast<const f32x4*>(&lse2[(t - t0) * 32 + 8 * j + 4 * half]);
    if (some_silent) {  // their scores may be NaN or infinite
#pragma unroll
      for (int u = 0; u < KT; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = e[r >> 2][r & 3] == -INFINITY ? 0.f : s[u][r];
    }
#pragma unroll
    for (int u = 0; u < KT; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[u][r & 1] += __builtin_amdgcn_exp2f(fmaf(s[u][r], a.qscale, e[r >> 2][r & 3]));
  }
  wait_vm<0>();  // no load is in flight into LDS when the workgroup ends
#pragma unroll
  for (int u = 0; u < KT; ++u) {
    const float x = halves_sum(sum[u][0] + sum[u][1]);
    const int j = key0 + u * 32 + col;
    if (half || j >= plen) continue;
    const int64_t at = (int64_t)gk * a.prefix + j;
    if (l.part) l.part[(int64_t)split * a.n_groups * a.n_kv * a.prefix + at] = x;
    else l.w_out[at] = (l.w_in ? l.decay * l.w_in[at] : 0.f) + x;
  }
}

// 64 slots a workgroup; each wave sums every fourth range, the four sums are added in order
__global__ __launch_bounds__(256) void k_weight_sum(WeightLaunch l) {
  __shared__ float sums[4][64];
  const SharedLaunch& a = l.a;
  const int64_t n = (int64_t)a.n_groups * a.n_kv * a.prefix, at = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int w = threadIdx.x >> 6, gk = (int)(at / a.prefix), j = (int)(at - (int64_t)gk * a.prefix);
  const bool on = at < n && j < clamp_len(a.plen, gk / a.n_kv, a.prefix);
  float sum = 0.f;
  if (on) {
#pragma unroll 8
    for (int s = w; s < a.splits; s += 4) sum += l.part[s * n + at];
  }
  sums[w][threadIdx.x & 63] = sum;
  __syncthreads();
  if (w || !on) return;
  const int c = threadIdx.x;
  l.w_out[at] = (l.w_in ? l.decay * l.w_in[at] : 0.f) + (((sums[0][c] + sums[1][c]) + sums[2][c]) + sums[3][c]);
}

// ---------------------------------------------------------------------------
// choices and launches
// ---------------------------------------------------------------------------
View view_of(const jpi_view& v, int es) {
  return View{(const char*)v.data, v.outer * es, v.row * es, v.head * es};
}

Divisor divisor(int64_t d) {
  u32 s = 0;
  while (((int64_t)1 << s) < d) ++s;
  return Divisor{(u32)d, (u32)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - d)) / d + 1), s};
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
  l.by_kv_heads = divisor(l.per_kv);
  l.by_rows = divisor(l.q_rows);
  l.by_rollout = divisor((int64_t)l.q_rows * l.per_kv);
  return l;
}

}  // namespace

// Waves (32 rows each) of a workgroup and ranges of the key sequence, by estimated time.  A workgroup fills a compute
// unit's LDS, so workgroups beyond one per unit wait for another round.  Microseconds, fitted to heads of 64 to 256 on 256
// units (estimates within a fifth of what was measured): a tile takes 0.9 + 0.002 of head_dim in bf16, four tenths more
// where waves share matrix cores, and 0.4 + 0.022 of head_dim in fp32; the rest of a workgroup 12; joining ranges a launch,
// 4, and their sums, written and read, 6.6 TB/s.  Lengths are on the device: the slots count, and all tails as full.
// Few rows over a long prefix want as many ranges as units: 32 rows of 256 dims over 65536 slots took 47 us with 64 ranges at
// most and take 30 with 256.
PrefixPlan shared_plan(const jpi_shared_attn& a) {
  const double n_cu = 256;
  const bool half = a.dtype == JPI_BF16;
  const int64_t per_rollout = (int64_t)a.q_rows * (a.n_heads / a.n_kv_heads), rows = a.group * per_rollout;
  const int keys = half ? KEYS<bf16> : KEYS<float>;
  const int64_t prefix = (a.prefix + keys - 1) / keys, tail = (a.suffix + keys - 1) / keys;
  const double all_mb = (double)a.n_groups * rows * a.n_kv_heads * a.head_dim * 4e-6;
  const int most = a.head_dim == 256 ? 4 : 8;  // eight waves share a unit's matrix cores and registers two by two
  PrefixPlan best{};
  double best_us = 1e30;
  for (int w = 1; w <= most; w *= 2) {
    if (w > 1 && 32 * (w / 2) >= rows) break;
    const int64_t row_tiles = (rows + 32 * w - 1) / (32 * w), items = (int64_t)a.n_groups * a.n_kv_heads * row_tiles;
    const int64_t rollouts = std::min<int64_t>(a.group, (32 * w + per_rollout - 1) / per_rollout);
    const double tiles = (double)prefix + (double)TAIL_COST * tail * rollouts;
    const double tile_us = (half ? 0.9 + 0.002 * a.head_dim : 0.4 + 0.022 * a.head_dim) * (w == 8 ? 1.4 : 1.0);
    for (const int s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64, 96, 128, 192, 256}) {
      if (s > 1 && s > prefix + tail) break;
      const double us = ceil(items * s / n_cu) * (ceil(tiles / s) * tile_us + 12) + (s > 1 ? 4 + all_mb * s / 3.3 : 0);
      if (us < best_us) best_us = us, best = PrefixPlan{w, (int)row_tiles, s};
    }
  }
  return best;
}

// Key blocks of a workgroup, and ranges of rows: 512 workgroups where there are as many pieces, ranges of at most WEIGHT_ROWS.
// A unit holds three in bf16 with heads of 64 and 128 and in fp32 with 64, two with bf16 256 and fp32 128, one with fp32 256.
PrefixPlan weight_plan(const jpi_shared_attn& a) {
  const int64_t rows = (int64_t)a.group * a.q_rows * (a.n_heads / a.n_kv_heads), tiles = (rows + 32 - 1) / 32;
  const int keys = 32 * (a.dtype == JPI_F32 && a.head_dim == 256 ? 1 : 2) * WEIGHT_WAVES;
  PrefixPlan p{};
  p.waves = WEIGHT_WAVES;
  p.tiles = (a.prefix + keys - 1) / keys;
  const int64_t items = (int64_t)a.n_groups * a.n_kv_heads * p.tiles;
  const int64_t least = (tiles + WEIGHT_ROWS / 32 - 1) / (WEIGHT_ROWS / 32);
  p.splits = items ? (int)std::max(least, std::min<int64_t>({64, 512 / items, tiles})) : 1;
  if (p.splits < 1) p.splits = 1;
  return p;
}

namespace {

unsigned grid8(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }
bool fits(int64_t groups, int threads) { return groups * threads < (int64_t)1 << 32; }  // a launch's threads are counted in 32 bits

int merge_waves(int splits) { return splits > 64 ? 16 : splits > 8 ? 4 : 1; }  // of a row

template <typename T, int DH>
hipError_t shared_typed(const jpi_shared_attn& a, void* ws, hipStream_t s) {
  const PrefixPlan p = shared_plan(a);
  SharedLaunch l = launch_of(a);
  l.splits = p.splits;
  l.row_tiles = p.tiles;
  l.by_splits = divisor(p.splits);
  l.by_tiles = divisor(p.tiles);
  const int64_t rows = (int64_t)a.n_groups * a.group * a.q_rows * a.n_heads;
  if (p.splits > 1) {
    l.part = (float*)ws;
    l.stats = (float2*)(l.part + p.splits * rows * DH);
  }
  const unsigned grid = grid8((int64_t)a.n_groups * a.n_kv_heads * p.tiles * p.splits);
  switch (p.waves) {
    case 1: k_shared<T, DH, 1><<<grid, 64, 0, s>>>(l); break;
    case 2: k_shared<T, DH, 2><<<grid, 128, 0, s>>>(l); break;
    case 4: k_shared<T, DH, 4><<<grid, 256, 0, s>>>(l); break;
    default:
      if constexpr (DH < 256) k_shared<T, DH, 8><<<grid, 512, 0, s>>>(l);
      break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const int waves = merge_waves(p.splits);
  if (waves == 16) k_shared_merge<T, DH, 16><<<(unsigned)rows, 1024, 0, s>>>(l);
  else if (waves == 4) k_shared_merge<T, DH, 4><<<(unsigned)rows, 256, 0, s>>>(l);
  else k_shared_merge<T, DH, 1><<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(l);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t weight_typed(const jpi_shared_attn& a, const float* w_in, float decay, float* w_out, void* ws, hipStream_t s) {
  if (a.prefix == 0) return hipSuccess;
  const PrefixPlan p = weight_plan(a);
  WeightLaunch l{};
  l.a = launch_of(a);
  l.a.splits = p.splits;
  l.lse = a.lse;
  l.w_in = w_in;
  l.w_out = w_out;
  l.decay = decay;
  l.key_tiles = p.tiles;
  const int64_t slots = (int64_t)a.n_groups * a.n_kv_heads * a.prefix;
  if (p.splits > 1) l.part = (float*)ws;
  k_weight<T, DH><<<grid8((int64_t)a.n_groups * a.n_kv_heads * p.tiles * p.splits), 64 * WEIGHT_WAVES, 0, s>>>(l);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  k_weight_sum<<<(unsigned)((slots + 63) / 64), 256, 0, s>>>(l);
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

bool shared_attention_fits(const jpi_shared_attn& a) {
  const int64_t rows = (int64_t)a.n_groups * a.group * a.q_rows * a.n_heads;
  // whatever the plan: at most 2 threads a row and 512 a (group, KV head) in each of 256 ranges, and 1024 a row of the join
  if (rows <= 1 << 21 && (int64_t)a.n_groups * a.n_kv_heads <= 1 << 13) return true;
  const PrefixPlan p = shared_plan(a);
  return fits((int64_t)a.n_groups * a.n_kv_heads * p.tiles * p.splits + 7, 64 * p.waves) &&
         (p.splits == 1 || fits(rows + 3, 64 * merge_waves(p.splits)));
}

bool prefix_weight_fits(const jpi_shared_attn& a) {
  const PrefixPlan p = weight_plan(a);
  const int64_t kv = (int64_t)a.n_groups * a.n_kv_heads;
  return fits(kv * p.tiles * p.splits + 7, 64 * WEIGHT_WAVES) && (p.splits == 1 || fits(kv * a.prefix / 64 + 1, 256));
}

size_t shared_attention_bytes(const jpi_shared_attn& a) {
  const PrefixPlan p = shared_plan(a);
  if (p.splits == 1) return 0;
  return (size_t)p.splits * a.n_groups * a.group * a.q_rows * a.n_heads * (a.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_shared_attention(const jpi_shared_attn& a, void* ws, hipStream_t s) {
  return by_type(a, [&](auto t, auto dh) { return shared_typed<decltype(t), dh.value>(a, ws, s); });
}

size_t prefix_weight_bytes(const jpi_shared_attn& a) {
  const PrefixPlan p = weight_plan(a);
  return p.splits == 1 ? 0 : (size_t)p.splits * a.n_groups * a.n_kv_heads * a.prefix * sizeof(float);
}

hipError_t launch_prefix_weight(const jpi_shared_attn& a, const float* w_in, float decay, float* w_out, void* ws,
                                hipStream_t s) {
  return by_type(a, [&](auto t, auto dh) { return weight_typed<decltype(t), dh.value>(a, w_in, decay, w_out, ws, s); });
}

}  // namespace jpi
