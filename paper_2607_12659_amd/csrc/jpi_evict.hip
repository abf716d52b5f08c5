// Eviction of the lightest slots of a prefix cache (jpi_evict, include/jpi_prefix.h).
//
// Two launches.  k_evict_select, one workgroup per sequence, finds the weight of
// the last slot that stays (a search over the bits of an order-preserving integer
// image of the weights, counting with ballots: no sort, no order of atomics that
// could show), marks what stays and writes the old slot of each new one.
// k_evict_copy or, where the cache is compacted in place, k_evict_shift then
// moves the rows of K and V.  Both are bound by memory: the kept rows are read
// and written once.
#include <algorithm>

#include "jpi_device.h"
#include "jpi_prefix_internal.h"

namespace jpi {
namespace {

typedef unsigned int u32;
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

constexpr int SEL = 1024;         // threads of the selection
constexpr int SEL_WAVES = SEL / 64;

// Order-preserving image of a weight: larger weight, larger integer; NaN as -inf, -0 as 0; never 0.
__device__ __forceinline__ u32 weight_key(float w) {
  if (__builtin_isnan(w)) w = -INFINITY;
  const u32 u = __builtin_bit_cast(u32, w + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int evict_len(const jpi_evict_args& a, int o) {
  return a.len ? max(0, min(a.len[o], a.slots)) : a.slots;
}

// N: weights that a thread keeps in registers (sequences of up to N * SEL slots); 0: they are read anew in each pass.
template <int N>
__global__ __launch_bounds__(SEL) void k_evict_select(jpi_evict_args a) {
  __shared__ int count[16][3];
  __shared__ int tie_of[SEL_WAVES], kept_of[SEL_WAVES];
  const int seq = blockIdx.x, o = seq / a.n_heads, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = evict_len(a, o), m = min(n, a.keep);
  const float* wt = a.weight + (int64_t)seq * a.weight_stride;
  float* wo = a.weight_out ? a.weight_out + (int64_t)seq * a.weight_out_stride : nullptr;
  int32_t* index = a.index + (int64_t)seq * a.keep;
  if (n <= a.keep) {
    for (int j = tid; j < m; j += SEL) {
      index[j] = j;
      if (wo && wo != wt) wo[j] = wt[j];
    }
    return;
  }
  const int lo = a.n_first, hi = n - a.n_last;  // the slots that compete
  const int need = a.keep - a.n_first - a.n_last;
  const int chunks = (n + SEL - 1) / SEL;
  auto load = [&](int c) -> u32 {
    const int j = c * SEL + tid;
    return j >= lo && j < hi ? weight_key(wt[j]) : 0u;
  };
  u32 key[N ? N : 1];
  if constexpr (N != 0) {
#pragma unroll
    for (int c = 0; c < N; ++c) key[c] = load(c);
  }
  if (tid < 48) (&count[0][0])[tid] = 0;
  __syncthreads();

  // the need-th largest key, two bits at a time
  u32 last = 0;
  for (int it = 0; it < 16; ++it) {
    const int sh = 30 - 2 * it;
    int c1 = 0, c2 = 0, c3 = 0;
    auto tally = [&](u32 k) {
      c1 += __builtin_popcountll(__ballot(k >= (last | 1u << sh)));
      c2 += __builtin_popcountll(__ballot(k >= (last | 2u << sh)));
      c3 += __builtin_popcountll(__ballot(k >= (last | 3u << sh)));
    };
    if constexpr (N != 0) {
#pragma unroll
      for (int c = 0; c < N; ++c) tally(key[c]);
    } else {
      for (int c = 0; c < chunks; ++c) tally(load(c));
    }
    if (lane == 0) {
      atomicAdd(&count[it][0], c1);
      atomicAdd(&count[it][1], c2);
      atomicAdd(&count[it][2], c3);
    }
    __syncthreads();
    last |= (count[it][2] >= need ? 3u : count[it][1] >= need ? 2u : count[it][0] >= need ? 1u : 0u) << sh;
  }
  // slots above it, and so how many equal ones stay
  __syncthreads();
  if (tid == 0) count[0][0] = 0;
  __syncthreads();
  {
    int c1 = 0;
    if constexpr (N != 0) {
#pragma unroll
      for (int c = 0; c < N; ++c) c1 += __builtin_popcountll(__ballot(key[c] > last));
    } else {
      for (int c = 0; c < chunks; ++c) c1 += __builtin_popcountll(__ballot(load(c) > last));
    }
    if (lane == 0) atomicAdd(&count[0][0], c1);
  }
  __syncthreads();
  const int ties = need - count[0][0];

  // places, chunk by chunk in slot order
  int ties_before = 0, kept_before = 0;
  auto place = [&](int c, u32 k) {
    const int j = c * SEL + tid;
    const bool tie = k == last && k != 0;
    const unsigned long long tm = __ballot(tie), below = (1ull << lane) - 1;
    if (lane == 0) tie_of[w] = __builtin_popcountll(tm);
    __syncthreads();
    int tb = ties_before;
#pragma unroll
    for (int v = 0; v < SEL_WAVES; ++v) {
      const int x = tie_of[v];
      tb += v < w ? x : 0;
      ties_before += x;
    }
    const bool kept = j < n && (j < lo || j >= hi || k > last || (tie && tb + __builtin_popcountll(tm & below) < ties));
    const unsigned long long km = __ballot(kept);
    const float weight = kept && wo ? wt[j] : 0.f;
    if (lane == 0) kept_of[w] = __builtin_popcountll(km);
    // in place, a slot's weight is written where an earlier or this one's was read: all of this chunk is in registers
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int kb = kept_before;
#pragma unroll
    for (int v = 0; v < SEL_WAVES; ++v) {
      const int x = kept_of[v];
      kb += v < w ? x : 0;
      kept_before += x;
    }
    if (kept) {
      const int t = kb + __builtin_popcountll(km & below);
      index[t] = j;
      if (wo) wo[t] = weight;
    }
  };
  if constexpr (N != 0) {
#pragma unroll
    for (int c = 0; c < N; ++c)
      if (c < chunks) place(c, key[c]);
  } else {
    for (int c = 0; c < chunks; ++c) place(c, load(c));
  }
}

struct MoveTensor {
  const char* src;
  char* dst;
  int64_t so, sr, sh, d_o, dr, dh;  // bytes: outer, row, head
};

struct MoveLaunch {
  MoveTensor t[2];
  int n_t;  // tensors
  jpi_evict_args a;
  int pieces;  // of a row
  int parts;   // workgroups of one sequence and tensor: ranges of rows (copy), of pieces (shift)
  int per;     // rows (copy) or pieces (shift) of one of them
};

__device__ __forceinline__ void move_item(const MoveLaunch& l, int& seq, int& ti, int& part) {
  part = blockIdx.x % l.parts;
  ti = blockIdx.x / l.parts % l.n_t;
  seq = blockIdx.x / (l.parts * l.n_t);
}

// Kept rows into other memory.  P: a piece of a row, 16 bytes where everything is aligned, else an element.
template <typename P>
__global__ __launch_bounds__(256) void k_evict_copy(MoveLaunch l) {
  int seq, ti, part;
  move_item(l, seq, ti, part);
  const int o = seq / l.a.n_heads, h = seq - o * l.a.n_heads;
  const int m = min(evict_len(l.a, o), l.a.keep);
  const MoveTensor& x = l.t[ti];
  const char* src = x.src + o * x.so + h * x.sh;
  char* dst = x.dst + o * x.d_o + h * x.dh;
  const int32_t* index = l.a.index + (int64_t)seq * l.a.keep;
  const int t0 = part * l.per, t1 = min(m, t0 + l.per);
  for (int u = threadIdx.x; u < (t1 - t0) * l.pieces; u += 256) {
    const int r = u / l.pieces, c = u - r * l.pieces, t = t0 + r;
    *reinterpret_cast<P*>(dst + t * x.dr + c * sizeof(P)) =
        *reinterpret_cast<const P*>(src + (int64_t)index[t] * x.sr + c * sizeof(P));
  }
  if (part == 0 && ti == 0 && h == 0 && threadIdx.x == 0 && l.a.len_out) l.a.len_out[o] = m;
}

// Kept rows moved down in their own memory: a workgroup takes some pieces of every row of a sequence.  A row's new
// place is never behind its old one, so a batch of rows may be written as soon as it is read whole, and the reads of
// the next batch touch nothing that this one writes.
template <typename P>
__global__ __launch_bounds__(256) void k_evict_shift(MoveLaunch l) {
  constexpr int U = 4;
  int seq, ti, part;
  move_item(l, seq, ti, part);
  const int o = seq / l.a.n_heads, h = seq - o * l.a.n_heads;
  const int m = min(evict_len(l.a, o), l.a.keep);
  const MoveTensor& x = l.t[ti];
  char* at = x.dst + o * x.d_o + h * x.dh;
  const int32_t* index = l.a.index + (int64_t)seq * l.a.keep;
  const int rows = 256 / l.per, r = threadIdx.x / l.per, c = part * l.per + (threadIdx.x - r * l.per);
  const bool on = r < rows && c < l.pieces;
  for (int t0 = 0; t0 < m; t0 += rows * U) {
    P v[U];
    bool moves[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * rows + r;
      moves[u] = false;
      if (on && t < m) {
        const int from = index[t];
        moves[u] = from != t;
        if (moves[u]) v[u] = *reinterpret_cast<const P*>(at + (int64_t)from * x.dr + c * sizeof(P));
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this batch is in registers before any of it is written
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (moves[u]) *reinterpret_cast<P*>(at + (int64_t)(t0 + u * rows + r) * x.dr + c * sizeof(P)) = v[u];
  }
  if (part == 0 && ti == 0 && h == 0 && threadIdx.x == 0 && l.a.len_out) l.a.len_out[o] = m;
}

template <typename P>
hipError_t move_rows(MoveLaunch l, bool in_place, int row_bytes, hipStream_t s) {
  l.pieces = row_bytes / (int)sizeof(P);
  const int64_t seqs = (int64_t)l.a.n_outer * l.a.n_heads;
  const int most = std::min(l.a.keep, l.a.slots);
  if (in_place) {
    l.per = std::min(l.pieces, std::max(1, 64 / (int)sizeof(P)));
    l.parts = (l.pieces + l.per - 1) / l.per;
    k_evict_shift<P><<<(unsigned)(seqs * l.n_t * l.parts), 256, 0, s>>>(l);
  } else {
    l.per = std::max(1, 1024 / l.pieces);
    l.parts = std::max(1, (most + l.per - 1) / l.per);
    k_evict_copy<P><<<(unsigned)(seqs * l.n_t * l.parts), 256, 0, s>>>(l);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_evict(const jpi_evict_args& a, hipStream_t s) {
  const int es = a.dtype == JPI_BF16 ? 2 : 4;
  const unsigned seqs = (unsigned)(a.n_outer * a.n_heads);
  if (a.slots <= SEL) k_evict_select<1><<<seqs, SEL, 0, s>>>(a);
  else if (a.slots <= 4 * SEL) k_evict_select<4><<<seqs, SEL, 0, s>>>(a);
  else if (a.slots <= 16 * SEL) k_evict_select<16><<<seqs, SEL, 0, s>>>(a);
  else k_evict_select<0><<<seqs, SEL, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  const jpi_view* in[2] = {&a.k, &a.v};
  const jpi_view* out[2] = {&a.k_out, &a.v_out};
  MoveTensor t[2];
  bool in_place[2];
  int64_t any = a.head_dim * es;
  for (int i = 0; i < 2; ++i) {
    t[i] = MoveTensor{(const char*)in[i]->data, (char*)out[i]->data, in[i]->outer * es, in[i]->row * es, in[i]->head * es,
                      out[i]->outer * es, out[i]->row * es, out[i]->head * es};
    in_place[i] = in[i]->data == out[i]->data;
    any |= (int64_t)((uintptr_t)t[i].src | (uintptr_t)t[i].dst) | t[i].so | t[i].sr | t[i].sh | t[i].d_o | t[i].dr | t[i].dh;
  }
  const bool together = in_place[0] == in_place[1];
  for (int i = 0; i < (together ? 1 : 2) && e == hipSuccess; ++i) {
    MoveLaunch l{};
    l.a = a;
    l.n_t = together ? 2 : 1;
    l.t[0] = t[i];
    if (together) l.t[1] = t[1];
    if (any % 16 == 0) e = move_rows<u32x4>(l, in_place[i], a.head_dim * es, s);
    else if (es == 4) e = move_rows<u32>(l, in_place[i], a.head_dim * es, s);
    else e = move_rows<uint16_t>(l, in_place[i], a.head_dim * es, s);
  }
  return e;
}

}  // namespace jpi
