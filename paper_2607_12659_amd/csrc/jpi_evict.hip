// Eviction of the lightest slots of a prefix cache (jpi_evict, include/jpi_prefix.h).
//
// Bound by memory: the kept rows of K and V are read and written once.  Which rows those are is found by a radix
// selection of the last weight that stays, over an order-preserving integer image of the weights (counts only, so no
// order of atomics could show), and a prefix sum in slot order.
//   Into other memory, few rows: one launch.  Every workgroup of a sequence makes the selection for itself, in which the
//   card is otherwise idle, and moves its share of the rows: 18 sequences of 816 slots cut to 408 (15 MB) take 10.5 us, with
//   the selection in a launch of its own 13.
//   Into other memory, many rows or slots: k_evict_select, then k_evict_copy.  144 sequences of 4096 slots cut to 1024
//   (302 MB) take 75 us, 4.0 TB/s; on inputs that the last-level cache holds 12 and 48.  The selection is one workgroup's
//   work for each sequence: 65536 slots take 120 us.
//   In place: k_evict_select, then k_evict_shift, since weights and lengths change where other workgroups read them.  The
//   same 18 sequences take 18 us, the 144 105 (11 and 88): a workgroup's rows follow each other, 256 at a time, and few
//   sequences make few workgroups (one of 65536 slots cut to half: 121 and 361).
#include <algorithm>

#include "jpi_device.h"
#include "jpi_prefix_internal.h"

namespace jpi {
namespace {

typedef unsigned int u32;
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

constexpr int SEL = 1024;         // threads of a selection
constexpr int SEL_WAVES = SEL / 64;
constexpr int DIGIT = 11;         // bits of a radix digit: three passes
constexpr int BINS = 1 << DIGIT;
constexpr int TOGETHER = 8;       // chunks of SEL slots that are read, and placed, together

// Order-preserving image of a weight: larger weight, larger integer; NaN as -inf, -0 as 0; never 0.
__device__ __forceinline__ u32 weight_key(float w) {
  if (__builtin_isnan(w)) w = -INFINITY;
  const u32 u = __builtin_bit_cast(u32, w + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int evict_len(const jpi_evict_args& a, int o) {
  return a.len ? max(0, min(a.len[o], a.slots)) : a.slots;
}

struct SelectLds {
  int bins[BINS];
  int sums[SEL_WAVES];
  int found[2];
  int ties[TOGETHER * SEL_WAVES], kept[TOGETHER * SEL_WAVES];  // of each wave, chunk by chunk
};

// Sum over the threads of lower index; `all` the sum over all of them.
__device__ __forceinline__ int before_me(int v, int* sums, int& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d, 64);
    x += lane >= d ? y : 0;
  }
  __syncthreads();
  if (lane == 63) sums[w] = x;
  __syncthreads();
  int add = 0;
  all = 0;
#pragma unroll
  for (int i = 0; i < SEL_WAVES; ++i) {
    const int y = sums[i];
    add += i < w ? y : 0;
    all += y;
  }
  return add + x - v;
}

// From each wave's counts of C chunks: the sum over all that come before this wave's, for each chunk; returns the whole sum.
// Every wave makes the one scan for itself.
template <int C>
__device__ __forceinline__ int before_chunks(const int* counts, int (&before)[C]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const bool on = 2 * lane < C * SEL_WAVES;
  const int a = on ? counts[2 * lane] : 0, b = on ? counts[2 * lane + 1] : 0;
  int x = a + b;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d, 64);
    x += lane >= d ? y : 0;
  }
  const int first = x - a - b, second = x - b;
#pragma unroll
  for (int c = 0; c < C; ++c) before[c] = __shfl(w & 1 ? second : first, (c * SEL_WAVES + w) / 2, 64);
  return __builtin_amdgcn_readlane(x, 63);
}

// The slots of a sequence that stay, n > keep.  N: weights that a thread keeps in registers (up to N * SEL slots); 0: they
// are read anew in each pass.  `stays(t, j)` is called for each kept slot j with its new place t.
template <int N, typename F>
__device__ __forceinline__ void select(const jpi_evict_args& a, const float* wt, int n, SelectLds& lds, F stays) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int lo = a.n_first, hi = n - a.n_last;  // the slots that compete
  int need = a.keep - a.n_first - a.n_last;     // how many of them stay
  const int chunks = (n + SEL - 1) / SEL;
  auto load = [&](int c) __attribute__((always_inline)) -> u32 {
    const int j = c * SEL + tid;
    return j >= lo && j < hi ? weight_key(wt[j]) : 0u;
  };
  u32 key[N ? N : 1];
  if constexpr (N != 0) {
#pragma unroll
    for (int c = 0; c < N; ++c) key[c] = load(c);
  }

  // the need-th largest key, a digit at a time from the top; `need` becomes its place among the equal ones
  u32 last = 0;
  if (need > 0) {
#pragma unroll 1
    for (int sh = 32 - DIGIT; sh > -DIGIT; sh -= DIGIT) {
      const int s = max(sh, 0), bits = min(DIGIT, sh + DIGIT);
      for (int i = tid; i < BINS; i += SEL) lds.bins[i] = 0;
      __syncthreads();
      auto count = [&](u32 k) __attribute__((always_inline)) {
        const bool on = k != 0 && (sh == 32 - DIGIT || k >> (s + bits) == last >> (s + bits));
        const u32 bin = k >> s & ((1u << bits) - 1);
        // equal weights are common (zeros), and adds to one address wait for each other: the first lane's bin as one
        const unsigned long long act = __ballot(on);
        if (act == 0) return;
        const u32 first = __builtin_amdgcn_readlane(bin, __builtin_ctzll(act));
        const unsigned long long same = __ballot(on && bin == first);
        if (lane == __builtin_ctzll(act)) atomicAdd(&lds.bins[first], __builtin_popcountll(same));
        if (on && bin != first) atomicAdd(&lds.bins[bin], 1);
      };
      if constexpr (N != 0) {
#pragma unroll
        for (int c = 0; c < N; ++c)
          if (c < chunks) count(key[c]);
      } else {
        for (int c0 = 0; c0 < chunks; c0 += TOGETHER) {
          u32 k[TOGETHER];
#pragma unroll
          for (int c = 0; c < TOGETHER; ++c) k[c] = load(c0 + c);  // 0 past the last slot
#pragma unroll
          for (int c = 0; c < TOGETHER; ++c) count(k[c]);
        }
      }
      __syncthreads();
      // from the largest bin down, two a thread: the one that holds the need-th
      const int b1 = BINS - 1 - 2 * tid, b0 = b1 - 1, c1 = lds.bins[b1], c0 = lds.bins[b0];
      int all;
      const int above = before_me(c1 + c0, lds.sums, all);
      if (above < need && need <= above + c1) lds.found[0] = b1, lds.found[1] = above;
      else if (above + c1 < need && need <= above + c1 + c0) lds.found[0] = b0, lds.found[1] = above + c1;
      __syncthreads();
      last |= (u32)lds.found[0] << s;
      need -= lds.found[1];
    }
  } else {
    last = ~0u;  // no key is as large
  }

  // places in slot order
  constexpr int C = N != 0 && N < TOGETHER ? N : TOGETHER;
  int ties_before = 0, kept_before = 0;
  auto place = [&](int c0, const u32* k) __attribute__((always_inline)) {
    const int w = tid >> 6;
    int before[C];
    unsigned long long in[C];  // of this wave
#pragma unroll
    for (int c = 0; c < C; ++c) {
      in[c] = __ballot(k[c] == last);
      if (lane == 0) lds.ties[c * SEL_WAVES + w] = __builtin_popcountll(in[c]);
    }
    __syncthreads();
    const int ties = before_chunks<C>(lds.ties, before);
    const unsigned long long lower = (1ull << lane) - 1;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int j = (c0 + c) * SEL + tid, tie = ties_before + before[c] + __builtin_popcountll(in[c] & lower);
      in[c] = __ballot(j < n && (j < lo || j >= hi || k[c] > last || (k[c] == last && tie < need)));
      if (lane == 0) lds.kept[c * SEL_WAVES + w] = __builtin_popcountll(in[c]);
    }
    __syncthreads();
    const int kept = before_chunks<C>(lds.kept, before);
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (in[c] >> lane & 1) stays(kept_before + before[c] + __builtin_popcountll(in[c] & lower), (c0 + c) * SEL + tid);
    ties_before += ties, kept_before += kept;
  };
  if constexpr (N != 0) {
#pragma unroll
    for (int c0 = 0; c0 < N; c0 += C)
      if (c0 < chunks) place(c0, key + c0);
  } else {
    for (int c0 = 0; c0 < chunks; c0 += C) {
      u32 k[C];
#pragma unroll
      for (int c = 0; c < C; ++c) k[c] = load(c0 + c);
      place(c0, k);
    }
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
  int parts;   // workgroups of one sequence: ranges of rows (gather); of one tensor, too: ranges of pieces (shift)
  int per;     // rows (gather) or pieces (shift) of one of them
  int first;   // first sequence of this launch (shift)
};

constexpr int GATHER_LEAST = 32, GATHER_MOST = SEL;  // rows of a workgroup

// Selection and move into other memory.  P: a piece of a row, 16 bytes where everything is aligned, else an element.
template <int N, typename P>
__global__ __launch_bounds__(SEL) void k_evict_gather(MoveLaunch l) {
  __shared__ SelectLds lds;
  __shared__ int from[GATHER_MOST];
  const jpi_evict_args& a = l.a;
  const int part = blockIdx.x % l.parts, seq = blockIdx.x / l.parts, o = seq / a.n_heads, h = seq - o * a.n_heads;
  const int n = evict_len(a, o), m = min(n, a.keep);
  const int t0 = part * l.per, t1 = min(m, t0 + l.per);
  if (part == 0 && h == 0 && threadIdx.x == 0 && a.len_out) a.len_out[o] = m;
  if (t0 >= t1) return;
  if (n > a.keep) {
    select<N>(a, a.weight + (int64_t)seq * a.weight_stride, n, lds, [&](int t, int j) __attribute__((always_inline)) {
      if (t >= t0 && t < t1) from[t - t0] = j;
    });
  } else {
    for (int t = t0 + threadIdx.x; t < t1; t += SEL) from[t - t0] = t;
  }
  __syncthreads();
  const float* wt = a.weight + (int64_t)seq * a.weight_stride;
  for (int t = t0 + threadIdx.x; t < t1; t += SEL) {
    const int j = from[t - t0];
    a.index[(int64_t)seq * a.keep + t] = j;
    if (a.weight_out) a.weight_out[(int64_t)seq * a.weight_out_stride + t] = wt[j];
  }
  // a thread keeps its piece of the row, and its rows are a fixed number apart, where the pieces divide the threads
  constexpr int U = 4;
  const int total = (t1 - t0) * l.pieces;
  for (int u0 = threadIdx.x; u0 < total; u0 += SEL * U) {
    P v[2][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = u0 + u * SEL, r = i / l.pieces, c = i - r * l.pieces;
      if (i >= total) continue;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x < l.n_t)
          v[x][u] = *reinterpret_cast<const P*>(l.t[x].src + o * l.t[x].so + h * l.t[x].sh + from[r] * l.t[x].sr + c * sizeof(P));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = u0 + u * SEL, r = i / l.pieces, c = i - r * l.pieces;
      if (i >= total) continue;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x < l.n_t)
          *reinterpret_cast<P*>(l.t[x].dst + o * l.t[x].d_o + h * l.t[x].dh + (t0 + r) * l.t[x].dr + c * sizeof(P)) = v[x][u];
    }
  }
}

// Selection alone: old slots, and the weights moved down where they may lie.
template <int N>
__global__ __launch_bounds__(SEL) void k_evict_select(jpi_evict_args a) {
  __shared__ SelectLds lds;
  const int seq = blockIdx.x, o = seq / a.n_heads, tid = threadIdx.x;
  const int n = evict_len(a, o), m = min(n, a.keep);
  const float* wt = a.weight + (int64_t)seq * a.weight_stride;
  float* wo = a.weight_out ? a.weight_out + (int64_t)seq * a.weight_out_stride : nullptr;
  int32_t* index = a.index + (int64_t)seq * a.keep;
  if (n <= a.keep) {
    for (int j = tid; j < m; j += SEL) index[j] = j;
  } else {
    select<N>(a, wt, n, lds, [&](int t, int j) __attribute__((always_inline)) { index[t] = j; });
  }
  if (!wo || (wo == wt && n <= a.keep)) return;
  // 1024 at a time, read before written: a weight's new place is never behind its old one
  __syncthreads();
  for (int t0 = 0; t0 < m; t0 += SEL) {
    const int t = t0 + tid;
    const float v = t < m ? wt[index[t]] : 0.f;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t < m) wo[t] = v;
  }
}

// Kept rows into other memory after a selection in a launch of its own, 16 KB a workgroup.
template <typename P>
__global__ __launch_bounds__(256) void k_evict_copy(MoveLaunch l) {
  const int part = blockIdx.x % l.parts, ti = blockIdx.x / l.parts % l.n_t, seq = blockIdx.x / (l.parts * l.n_t);
  const int o = seq / l.a.n_heads, h = seq - o * l.a.n_heads;
  const int m = min(evict_len(l.a, o), l.a.keep);
  const MoveTensor& x = l.t[ti];
  const char* src = x.src + o * x.so + h * x.sh;
  char* dst = x.dst + o * x.d_o + h * x.dh;
  const int32_t* index = l.a.index + (int64_t)seq * l.a.keep;
  const int t0 = part * l.per, t1 = min(m, t0 + l.per);
#pragma unroll 2
  for (int u = threadIdx.x; u < (t1 - t0) * l.pieces; u += 256) {
    const int r = u / l.pieces, c = u - r * l.pieces, t = t0 + r;
    *reinterpret_cast<P*>(dst + t * x.dr + c * sizeof(P)) = *reinterpret_cast<const P*>(src + index[t] * x.sr + c * sizeof(P));
  }
  if (part == 0 && ti == 0 && h == 0 && threadIdx.x == 0 && l.a.len_out) l.a.len_out[o] = m;
}

// Kept rows moved down in their own memory: a workgroup takes some pieces of every row of a sequence.  A row's new
// place is never behind its old one, so a batch of rows may be written as soon as it is read whole, and the reads of
// the next batch touch nothing that this one writes.
template <typename P>
__global__ __launch_bounds__(256) void k_evict_shift(MoveLaunch l) {
  constexpr int U = 4;
  const int part = blockIdx.x % l.parts, ti = blockIdx.x / l.parts % l.n_t, seq = l.first + (int)(blockIdx.x / (l.parts * l.n_t));
  const int o = seq / l.a.n_heads, h = seq - o * l.a.n_heads;
  const int m = min(evict_len(l.a, o), l.a.keep);  // the same before and after len_out, where that is len
  const MoveTensor& x = l.t[ti];
  const char* src = x.src + o * x.so + h * x.sh;
  char* dst = x.dst + o * x.d_o + h * x.dh;
  const bool in_place = x.src == x.dst;
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
        moves[u] = !in_place || from != t;
        if (moves[u]) v[u] = *reinterpret_cast<const P*>(src + from * x.sr + c * sizeof(P));
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this batch is in registers before any of it is written
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (moves[u]) *reinterpret_cast<P*>(dst + (t0 + u * rows + r) * x.dr + c * sizeof(P)) = v[u];
  }
  if (part == 0 && ti == 0 && h == 0 && threadIdx.x == 0 && l.a.len_out) l.a.len_out[o] = m;
}

template <typename P>
hipError_t evict_pieces(MoveLaunch l, bool gather, int row_bytes, hipStream_t s) {
  const jpi_evict_args& a = l.a;
  l.pieces = row_bytes / (int)sizeof(P);
  const int64_t seqs = (int64_t)a.n_outer * a.n_heads;
  const int most = std::min(a.keep, a.slots);
  if (!gather && l.t[0].src != l.t[0].dst && l.t[1].src != l.t[1].dst) {
    // 16 KB a workgroup; more where a launch, whose threads are counted in 32 bits, would not hold them
    l.per = (int)std::max<int64_t>(std::max(1, 1024 / l.pieces), (seqs * l.n_t * most >> 23) + 1);
    l.parts = std::max(1, (most + l.per - 1) / l.per);
    k_evict_copy<P><<<(unsigned)(seqs * l.n_t * l.parts), 256, 0, s>>>(l);
    return hipGetLastError();
  }
  if (!gather) {
    // 64 bytes of a row: half of a line, so that few sequences make enough workgroups
    l.per = std::min(l.pieces, std::max(1, 64 / (int)sizeof(P)));
    l.parts = (l.pieces + l.per - 1) / l.per;
    // a launch's threads are counted in 32 bits: as many launches as the sequences need
    const int64_t each = ((1 << 24) - 1) / (l.n_t * l.parts);
    for (int64_t first = 0; first < seqs; first += each) {
      l.first = (int)first;
      k_evict_shift<P><<<(unsigned)(std::min(each, seqs - first) * l.n_t * l.parts), 256, 0, s>>>(l);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  // two workgroups for each of 256 units, but no fewer than GATHER_LEAST rows in one.  At most GATHER_MOST: up to SEL slots
  // there are no more rows, past them the rule of launch_evict leaves at most 256 times GATHER_LEAST rows in all
  const int64_t want = std::max<int64_t>(1, 512 / seqs);
  l.per = (int)std::max<int64_t>(GATHER_LEAST, (most + want - 1) / want);
  l.parts = std::max(1, (most + l.per - 1) / l.per);
  const unsigned grid = (unsigned)(seqs * l.parts);
  if (a.slots <= SEL) k_evict_gather<1, P><<<grid, SEL, 0, s>>>(l);
  else if (a.slots <= 4 * SEL) k_evict_gather<4, P><<<grid, SEL, 0, s>>>(l);
  else k_evict_gather<16, P><<<grid, SEL, 0, s>>>(l);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_evict(const jpi_evict_args& a, hipStream_t s) {
  const int es = a.dtype == JPI_BF16 ? 2 : 4;
  const jpi_view* in[2] = {&a.k, &a.v};
  const jpi_view* out[2] = {&a.k_out, &a.v_out};
  MoveLaunch l{};
  l.a = a;
  l.n_t = 2;
  // One launch where nothing that a workgroup writes is read by another, and where a thread's weights stay in registers: read
  // anew by every workgroup, the selection of one sequence of 65536 slots took 214 us against 135 in a launch of its own, of
  // 20000 slots 79 against 51.
  bool gather = a.slots <= 16 * SEL && a.weight_out != a.weight && (!a.len || a.len_out != a.len);
  int64_t any = a.head_dim * es;
  for (int i = 0; i < 2; ++i) {
    l.t[i] = MoveTensor{(const char*)in[i]->data, (char*)out[i]->data, in[i]->outer * es, in[i]->row * es, in[i]->head * es,
                        out[i]->outer * es, out[i]->row * es, out[i]->head * es};
    gather = gather && in[i]->data != out[i]->data;
    any |= (int64_t)((uintptr_t)l.t[i].src | (uintptr_t)l.t[i].dst) | l.t[i].so | l.t[i].sr | l.t[i].sh | l.t[i].d_o |
           l.t[i].dr | l.t[i].dh;
  }
  // One launch or two, in us, heads of 256 in bf16 unless said; of 211 calls timed the rule's side was the faster one or within a
  // fifth of it, and half a percent slower on average.
  //   Up to SEL slots a selection is cheap, and one launch wins until the move is long: 18 sequences, 408 of 816 slots (K 4 MB),
  //   10 and 13; 512, 408 of 816 slots of 64 (27 MB), 28 and 34; 512, 900 of 1024 slots of 64 (59 MB), 68 and 60.
  //   Past them it wins while no unit has two workgroups, whose selections take twice as long: eight sequences, 1024 of 4096
  //   slots, 14 and 16, sixteen 27 and 19; one, 8192 of 16384 slots, 28 and 32, two 56 and 38.
  const int64_t n_seqs = (int64_t)a.n_outer * a.n_heads, most = std::min(a.keep, a.slots);
  gather = gather && n_seqs * most * a.head_dim * es < (int64_t)32 << 20 &&
           (a.slots <= SEL || n_seqs * ((most + GATHER_LEAST - 1) / GATHER_LEAST) <= 256);
  if (!gather) {
    const unsigned seqs = (unsigned)n_seqs;
    if (a.slots <= SEL) k_evict_select<1><<<seqs, SEL, 0, s>>>(a);
    else if (a.slots <= 4 * SEL) k_evict_select<4><<<seqs, SEL, 0, s>>>(a);
    else if (a.slots <= 16 * SEL) k_evict_select<16><<<seqs, SEL, 0, s>>>(a);
    else k_evict_select<0><<<seqs, SEL, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (any % 16 == 0) return evict_pieces<u32x4>(l, gather, a.head_dim * es, s);
  if (es == 4) return evict_pieces<u32>(l, gather, a.head_dim * es, s);
  return evict_pieces<uint16_t>(l, gather, a.head_dim * es, s);
}

}  // namespace jpi
