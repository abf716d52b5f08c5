// Moves of the pages of a cache (jpi_cache_resize, jpi_cache_reorder, jpi_cache_compact, include/jpi_cache.h).
//
// Each call is two launches.  The first settles what happens: one workgroup runs
// prefix sums over the sequences' needs and over the pages' counts, so that every
// result is by rank and no order of threads shows (reorder: copies of what it would
// overwrite).  The second does it: some workgroups write the tables' rows and
// change counts (integer atomics, which end alike in any order), the others share
// out the list of pages that move, in chunks.  Bound by the memory that moved pages
// are (compaction of 227 MB 104 us, 4.4 TB/s, 9 of them the plan), for few of them by
// the chain of reads of the two launches: eight forks of a prefix and their growth
// 11 us, 64 that are reordered and grow 15.  In large pools by the plan, whose one
// workgroup walks the counts, 8192 pages a step: to the last free page that a growth
// needs, through all of them for a compaction or where counts go elsewhere.  One free
// page at the end of 4096, 131072 and 2^20 pages: growth and its way back 13, 78 and
// 552 us, a compaction that moves nothing 8, 99 and 891; 5 where nobody needs a page.
#include <algorithm>

#include "jpi_cache_device.h"

namespace jpi {
namespace {

constexpr int PLAN_THREADS = 1024, THREADS = 256;
constexpr int PER = 8;            // pages of a planning thread at a time
constexpr int CHUNK = 16384;      // bytes of a page that a workgroup moves at a time
constexpr int ROW_ENTRIES = 1024; // entries of a table row that a workgroup writes

struct Moves {
  const int32_t *table, *len, *refs;
  int32_t *table_out, *len_out, *refs_out;
  int64_t table_stride, table_out_stride;
  int n_seqs, max_pages, n_pages, lg_page;
  // workspace
  int32_t* count;  // [0]: pages that move
  int32_t *src, *dst;
  int32_t *a, *b, *c;  // by call
};

struct Contents {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int64_t page_bytes, layer_pages;  // of K or of V; pages from layer to layer
  int kv, layers, chunks;           // chunks: of a page of K or V
};

__device__ __forceinline__ int pages_of(int len, int lg_page) { return (int)(((int64_t)len + (1 << lg_page) - 1) >> lg_page); }
__device__ __forceinline__ bool names(int page, int n_pages) { return (unsigned)page < (unsigned)n_pages; }

// Sum of the values of the threads before this one, and of all; every thread of the workgroup calls it
__device__ __forceinline__ int scan_before(int v, int& all, int* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // red may still be read by a scan before
  if (lane == 63) red[wave] = x;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 64; ++w) {
    before += w < wave ? red[w] : 0;
    total += red[w];
  }
  all = total;
  return before + x - v;
}

// One workgroup: which pages each sequence gets.  a: the place of its first page in `src`'s list of free pages, b: its length
// before the call, c: the page that is copied, or -1.  Free pages go to dst, as many as are needed.
__global__ __launch_bounds__(PLAN_THREADS) void k_resize_plan(Moves m, const int32_t* new_len, int32_t* short_out) {
  __shared__ int red[PLAN_THREADS / 64];
  __shared__ int copies;
  const int cap = m.max_pages << m.lg_page, page = 1 << m.lg_page;
  if (threadIdx.x == 0) copies = 0;

  // what the sequences need, and where each one's part begins
  int needed = 0;
  for (int s0 = 0; s0 < m.n_seqs; s0 += PLAN_THREADS) {
    const int s = s0 + threadIdx.x;
    int need = 0, copied = -1, old = 0;
    if (s < m.n_seqs) {
      old = clamp_len(m.len[s], cap);
      const int want = new_len[s], now = want < 0 ? old : min(want, cap);
      if (now > old) {
        const int had = pages_of(old, m.lg_page);
        need = pages_of(now, m.lg_page) - had;
        if (old & (page - 1)) {
          const int last = m.table[s * m.table_stride + had - 1];
          if (names(last, m.n_pages) && m.refs[last] > 1) copied = last, ++need;
        }
      }
    }
    int all;
    const int before = scan_before(need, all, red);
    if (s < m.n_seqs) m.a[s] = needed + before, m.b[s] = old, m.c[s] = copied;
    needed += all;
  }

  // free pages in ascending order, as many as are needed
  int found = 0;
  const bool other = m.refs_out != m.refs;
  for (int p0 = 0; p0 < m.n_pages && (other || found < needed); p0 += PLAN_THREADS * PER) {
    int r[PER], mine = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int p = p0 + (int)threadIdx.x * PER + e;
      r[e] = p < m.n_pages ? m.refs[p] : 1;
      if (other && p < m.n_pages) m.refs_out[p] = r[e];
      mine += r[e] <= 0;
    }
    int all;
    int at = found + scan_before(mine, all, red);
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (r[e] <= 0 && at < needed) m.dst[at++] = p0 + (int)threadIdx.x * PER + e;
    found += all;
  }
  if (threadIdx.x == 0 && short_out) *short_out = max(0, needed - found);
  __syncthreads();  // dst and a are read by other threads than wrote them

  // lengths, and the list of copies: sources to src, their places in dst stay with the sequences
  for (int s = threadIdx.x; s < m.n_seqs; s += PLAN_THREADS) {
    const int old = m.b[s], want = new_len[s], now = want < 0 ? old : min(want, cap), first = m.a[s];
    const int had = pages_of(old, m.lg_page), copied = m.c[s];
    const int need = now > old ? pages_of(now, m.lg_page) - had + (copied >= 0) : 0;
    const bool served = need == 0 || first + need <= found;
    m.len_out[s] = served ? now : old;
    if (!served) m.a[s] = -1;
    if (served && copied >= 0) {
      const int at = atomicAdd(&copies, 1);  // the list's order is that of no result
      m.src[2 * at] = copied;
      m.src[2 * at + 1] = m.dst[first];
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) m.count[0] = copies;
}

// Chunk c of a moving page: K and V of each layer in pieces, the scales with each layer's first.  PASSING: through no cache, for
// many pages whose old places nobody reads again: 227 MB of them 104 us, through the caches 115; the few copies of growing forks,
// whose sources and copies are read next, took 16 us instead of 15 so.
template <bool PASSING>
__device__ __forceinline__ void move_chunk(const Contents& x, int src, int dst, int item) {
  const int per_layer = 2 * x.chunks, layer = item / per_layer, c = item - layer * per_layer;
  const bool values = c >= x.chunks;
  const int64_t base = (int64_t)layer * x.layer_pages, at = (int64_t)(values ? c - x.chunks : c) * CHUNK;
  uint8_t* data = values ? x.v : x.k;
  const u32x4* from = reinterpret_cast<const u32x4*>(data + (base + src) * x.page_bytes + at);
  u32x4* to = reinterpret_cast<u32x4*>(data + (base + dst) * x.page_bytes + at);
  const int pieces = (int)(min((int64_t)CHUNK, x.page_bytes - at) / 16);
#pragma unroll 4
  for (int i = threadIdx.x; i < pieces; i += THREADS) {
    if constexpr (PASSING) __builtin_nontemporal_store(__builtin_nontemporal_load(from + i), to + i);
    else to[i] = from[i];
  }
  if (at == 0) {
    float* scale = values ? x.v_scale : x.k_scale;
    for (int i = threadIdx.x; i < x.kv; i += THREADS) scale[(base + dst) * x.kv + i] = scale[(base + src) * x.kv + i];
  }
}

template <bool PASSING>
__device__ __forceinline__ void move_pages(const Moves& m, const Contents& x, int first, int workgroups) {
  const int moves = m.count[0], items = x.layers * 2 * x.chunks;
  for (int64_t i = first; i < (int64_t)moves * items; i += workgroups) {
    const int n = (int)(i / items);
    move_chunk<PASSING>(x, m.src[2 * n], m.src[2 * n + 1], (int)(i - (int64_t)n * items));
  }
}

__global__ __launch_bounds__(THREADS) void k_resize(Moves m, Contents x, int row_groups, int per_row) {
  if ((int)blockIdx.x >= row_groups) return move_pages<false>(m, x, blockIdx.x - row_groups, gridDim.x - row_groups);
  const int s = blockIdx.x / per_row, e0 = (blockIdx.x - s * per_row) * ROW_ENTRIES;
  const int old = m.b[s], now = m.len_out[s], first = m.a[s], copied = first >= 0 ? m.c[s] : -1;
  const int had = pages_of(old, m.lg_page), has = pages_of(now, m.lg_page);
  for (int e = e0 + threadIdx.x; e < min(e0 + ROW_ENTRIES, m.max_pages); e += THREADS) {
    const int32_t was = e < had ? m.table[s * m.table_stride + e] : -1;
    int32_t is = was;
    if (e >= has) {
      is = -1;
      if (e < had && names(was, m.n_pages)) atomicSub(&m.refs_out[was], 1);
    } else if (e >= had || (copied >= 0 && e == had - 1)) {
      is = m.dst[first + (e >= had ? e - had + (copied >= 0) : 0)];
      m.refs_out[is] = 1;  // it was free, and nobody else has it
      if (e < had) atomicSub(&m.refs_out[was], 1);
    }
    m.table_out[s * m.table_out_stride + e] = is;
  }
}

// What reorder overwrites: the table where it is its own output (to a), the lengths (to b); counts that go elsewhere
__global__ __launch_bounds__(THREADS) void k_reorder_keep(Moves m, bool table) {
  const int64_t n = (int64_t)m.n_seqs * m.max_pages, stride = (int64_t)gridDim.x * THREADS;
  const int64_t i0 = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (table)
    for (int64_t i = i0; i < n; i += stride) m.a[i] = m.table[i / m.max_pages * m.table_stride + i % m.max_pages];
  for (int64_t i = i0; i < m.n_seqs; i += stride) m.b[i] = m.len[i];
  if (m.refs_out != m.refs)
    for (int64_t i = i0; i < m.n_pages; i += stride) m.refs_out[i] = m.refs[i];
}

__global__ __launch_bounds__(THREADS) void k_reorder(Moves m, const int32_t* parents, int per_row) {
  const int s = blockIdx.x / per_row, e0 = (blockIdx.x - s * per_row) * ROW_ENTRIES;
  const int cap = m.max_pages << m.lg_page, parent = parents[s];
  const bool some = (unsigned)parent < (unsigned)m.n_seqs;
  const int old = clamp_len(m.b[s], cap), now = some ? clamp_len(m.b[parent], cap) : 0;
  const int had = pages_of(old, m.lg_page), has = pages_of(now, m.lg_page);
  for (int e = e0 + threadIdx.x; e < min(e0 + ROW_ENTRIES, m.max_pages); e += THREADS) {
    const int32_t was = e < had ? m.table[s * m.table_stride + e] : -1;
    const int32_t is = e < has ? m.table[parent * m.table_stride + e] : -1;
    if (parent != s) {
      if (names(was, m.n_pages)) atomicSub(&m.refs_out[was], 1);
      if (names(is, m.n_pages)) atomicAdd(&m.refs_out[is], 1);
    }
    m.table_out[s * m.table_out_stride + e] = is;
  }
  if (e0 == 0 && threadIdx.x == 0) m.len_out[s] = now;
}

// Both in one launch by one workgroup, which reads all that it overwrites first: for tables of up to ONE_ENTRIES entries and
// pools of up to ONE_PAGES pages, whose counts it copies where they go elsewhere.  With its growth behind it, 8 x 15 entries
// 13.0 -> 11.4 us on the GPU and three launches for the host instead of four; 64 x 64 entries 15.2 -> 22.7.
constexpr int ONE_ENTRIES = 2 * PLAN_THREADS, ONE_PAGES = 64 * PLAN_THREADS;
__global__ __launch_bounds__(PLAN_THREADS) void k_reorder_one(Moves m, const int32_t* parents) {
  constexpr int MOST = ONE_ENTRIES / PLAN_THREADS;
  const int cap = m.max_pages << m.lg_page, entries = m.n_seqs * m.max_pages;
  int32_t was[MOST], is[MOST], now[MOST];
  bool other[MOST];
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    const int i = threadIdx.x + k * PLAN_THREADS;
    if (i >= entries) continue;
    const int s = i / m.max_pages, e = i - s * m.max_pages, parent = parents[s];
    const bool some = (unsigned)parent < (unsigned)m.n_seqs;
    now[k] = some ? clamp_len(m.len[parent], cap) : 0;
    was[k] = e < pages_of(clamp_len(m.len[s], cap), m.lg_page) ? m.table[s * m.table_stride + e] : -1;
    is[k] = e < pages_of(now[k], m.lg_page) ? m.table[parent * m.table_stride + e] : -1;
    other[k] = parent != s;
  }
  if (m.refs_out != m.refs)
    for (int p = threadIdx.x; p < m.n_pages; p += PLAN_THREADS) m.refs_out[p] = m.refs[p];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    const int i = threadIdx.x + k * PLAN_THREADS;
    if (i >= entries) continue;
    const int s = i / m.max_pages, e = i - s * m.max_pages;
    if (other[k]) {
      if (names(was[k], m.n_pages)) atomicSub(&m.refs_out[was[k]], 1);
      if (names(is[k], m.n_pages)) atomicAdd(&m.refs_out[is[k]], 1);
    }
    m.table_out[s * m.table_out_stride + e] = is[k];
    if (e == 0) m.len_out[s] = now[k];
  }
}

// One workgroup: counts pages in use, then pairs those behind them with the free ones before.  a: the new number of each page
// from n_live on; count[1]: n_live.
__global__ __launch_bounds__(PLAN_THREADS) void k_compact_plan(Moves m, int32_t* n_live_out) {
  __shared__ int red[PLAN_THREADS / 64];
  int mine = 0, n_live;
#pragma unroll 8
  for (int p = threadIdx.x; p < m.n_pages; p += PLAN_THREADS) mine += m.refs[p] > 0;
  scan_before(mine, n_live, red);

  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < m.n_pages; p0 += PLAN_THREADS * PER) {
    int r[PER], hole = 0, mover = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int p = p0 + (int)threadIdx.x * PER + e;
      r[e] = p < m.n_pages ? m.refs[p] : 0;
      hole += p < n_live && r[e] <= 0;
      mover += p >= n_live && r[e] > 0;
    }
    // both counts in one sum: there are 2^13 of either at most
    int all;
    const int before = scan_before(mover << 16 | hole, all, red), all_holes = all & 0xffff, all_movers = all >> 16;
    int at_hole = holes + (before & 0xffff), at_mover = movers + (before >> 16);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int p = p0 + (int)threadIdx.x * PER + e;
      if (p >= m.n_pages) break;
      if (p < n_live) {
        if (r[e] <= 0) m.src[2 * at_hole++ + 1] = p;
      } else {
        if (r[e] > 0) m.src[2 * at_mover++] = p;
        else m.a[p] = p;
      }
    }
    holes += all_holes, movers += all_movers;
  }
  __syncthreads();
  // the same number of either: n_live pages are in use, n_live - holes of them below n_live
  for (int i = threadIdx.x; i < movers; i += PLAN_THREADS) m.a[m.src[2 * i]] = m.src[2 * i + 1];
  if (m.refs_out != m.refs)
    for (int p = threadIdx.x; p < m.n_pages; p += PLAN_THREADS) m.refs_out[p] = m.refs[p];
  __syncthreads();
  for (int i = threadIdx.x; i < movers; i += PLAN_THREADS) {
    const int from = m.src[2 * i], to = m.src[2 * i + 1], n = m.refs[from];
    m.refs_out[to] = n;
    m.refs_out[from] = 0;
  }
  if (threadIdx.x == 0) {
    m.count[0] = movers, m.count[1] = n_live;
    if (n_live_out) *n_live_out = n_live;
  }
}

__global__ __launch_bounds__(THREADS) void k_compact(Moves m, Contents x, int row_groups, int per_row) {
  if ((int)blockIdx.x >= row_groups) return move_pages<true>(m, x, blockIdx.x - row_groups, gridDim.x - row_groups);
  const int s = blockIdx.x / per_row, e0 = (blockIdx.x - s * per_row) * ROW_ENTRIES, n_live = m.count[1];
  for (int e = e0 + threadIdx.x; e < min(e0 + ROW_ENTRIES, m.max_pages); e += THREADS) {
    const int32_t was = m.table[s * m.table_stride + e];
    m.table_out[s * m.table_out_stride + e] = names(was, m.n_pages) && was >= n_live ? m.a[was] : was;
  }
}

int64_t rounded(int64_t ints) { return (ints + 3) / 4 * 4; }

Moves moves_of(const jpi_cache_moves& m, void* ws) {
  Moves x{};
  x.table = m.seqs.table, x.len = m.seqs.len, x.refs = m.refs;
  x.table_out = m.table_out, x.len_out = m.len_out, x.refs_out = m.refs_out;
  x.table_stride = m.seqs.table_stride, x.table_out_stride = m.table_out_stride;
  x.n_seqs = m.seqs.n_seqs, x.max_pages = m.seqs.max_pages, x.n_pages = m.n_pages, x.lg_page = __builtin_ctz(m.page);
  x.count = (int32_t*)ws;
  return x;
}

Contents contents_of(const jpi_cache_pool* pool, int layers) {
  Contents x{};
  if (!pool) return x;
  const jpi_cache_pool& p = *pool;
  x.k = (uint8_t*)p.k, x.v = (uint8_t*)p.v, x.k_scale = p.k_scale, x.v_scale = p.v_scale;
  x.page_bytes = (int64_t)p.n_kv_heads * p.page * p.head_dim;
  x.layer_pages = p.n_pages, x.kv = p.n_kv_heads, x.layers = layers;
  x.chunks = (int)((x.page_bytes + CHUNK - 1) / CHUNK);
  return x;
}

int per_row(const jpi_cache_moves& m) { return (m.seqs.max_pages + ROW_ENTRIES - 1) / ROW_ENTRIES; }

// workgroups that move pages: as many as there can be chunks, up to eight a unit
int movers(const Contents& x, int64_t most) {
  return x.layers ? (int)std::min<int64_t>(2048, most * x.layers * 2 * x.chunks) : 0;
}

}  // namespace

bool moves_fit(const jpi_cache_moves& m) { return (int64_t)m.seqs.n_seqs * per_row(m) < (1 << 24) - 4096; }

// count; then resize: a, b, c and pairs of the sequences, free pages; reorder: table and lengths; compact: pairs and numbers
size_t moves_bytes(const jpi_cache_moves& m) {
  const int64_t seqs = rounded(m.seqs.n_seqs), pages = rounded(m.n_pages);
  const int64_t resize = 5 * seqs + pages, reorder = rounded((int64_t)m.seqs.n_seqs * m.seqs.max_pages) + seqs, compact = 2 * pages + pages;
  return (size_t)(4 + std::max({resize, reorder, compact})) * sizeof(int32_t);
}

hipError_t launch_resize(const jpi_cache_moves& m, const jpi_cache_pool* pool, int layers, const int32_t* new_len,
                         int32_t* short_out, void* ws, hipStream_t s) {
  Moves x = moves_of(m, ws);
  const Contents c = contents_of(pool, layers);
  const int64_t seqs = rounded(m.seqs.n_seqs);
  x.a = x.count + 4, x.b = x.a + seqs, x.c = x.b + seqs, x.src = x.c + seqs, x.dst = x.src + 2 * seqs;
  k_resize_plan<<<1, PLAN_THREADS, 0, s>>>(x, new_len, short_out);
  const int rows = m.seqs.n_seqs * per_row(m);
  k_resize<<<rows + movers(c, m.seqs.n_seqs), THREADS, 0, s>>>(x, c, rows, per_row(m));
  return hipGetLastError();
}

hipError_t launch_reorder(const jpi_cache_moves& m, const int32_t* parents, void* ws, hipStream_t s) {
  Moves x = moves_of(m, ws);
  if ((int64_t)m.seqs.n_seqs * m.seqs.max_pages <= ONE_ENTRIES && m.n_pages <= ONE_PAGES) {
    k_reorder_one<<<1, PLAN_THREADS, 0, s>>>(x, parents);
    return hipGetLastError();
  }
  const bool in_place = m.table_out == m.seqs.table;
  x.b = x.count + 4, x.a = x.b + rounded(m.seqs.n_seqs);
  const int64_t most = std::max<int64_t>(m.n_pages, in_place ? (int64_t)m.seqs.n_seqs * m.seqs.max_pages : m.seqs.n_seqs);
  k_reorder_keep<<<(unsigned)std::min<int64_t>(1024, (most + THREADS - 1) / THREADS), THREADS, 0, s>>>(x, in_place);
  if (in_place) x.table = x.a, x.table_stride = m.seqs.max_pages;
  k_reorder<<<m.seqs.n_seqs * per_row(m), THREADS, 0, s>>>(x, parents, per_row(m));
  return hipGetLastError();
}

hipError_t launch_compact(const jpi_cache_moves& m, const jpi_cache_pool* pool, int layers, int32_t* n_live_out, void* ws,
                          hipStream_t s) {
  Moves x = moves_of(m, ws);
  const Contents c = contents_of(pool, layers);
  const int64_t pages = rounded(m.n_pages);
  x.src = x.count + 4, x.a = x.src + 2 * pages;
  k_compact_plan<<<1, PLAN_THREADS, 0, s>>>(x, n_live_out);
  const int rows = m.seqs.n_seqs * per_row(m);
  k_compact<<<rows + movers(c, m.n_pages / 2), THREADS, 0, s>>>(x, c, rows, per_row(m));
  return hipGetLastError();
}

}  // namespace jpi
