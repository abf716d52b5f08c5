// Launches of the operators of a paged 8-bit cache (include/jpi_cache.h), which checks their arguments first.
#pragma once

#include "../../include/jpi_cache.h"
#include "jpi_prefix_internal.h"

namespace jpi {

struct NormWeights {
  const void* w[2];  // queries, keys; NULL: the norm alone
  int64_t stride;    // elements from head to head
  float offset, eps;
};
hipError_t launch_norm_rope(jpi_dtype dt, jpi_dtype weight_dt, const RopeLaunch& l, const NormWeights& nw, hipStream_t s);

bool append_fits(const jpi_cache_pool& p, const jpi_cache_seqs& q, int tokens);
hipError_t launch_append(const jpi_cache_pool& p, const jpi_cache_seqs& q, jpi_dtype dt, int tokens, const jpi_view& k,
                         const jpi_view& v, const int32_t* n_new, hipStream_t s);

// how a call is cut, for each (sequence, KV head): into workgroups of 128 rows that pass the keys through a ring, or (groups 0)
// into tiles of 16 rows and ranges of their keys, shared out among 4 or 8 waves
struct CachePlan {
  int groups, tiles, splits, waves;
};
CachePlan cache_plan(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q);
bool cache_attention_fits(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q);
size_t cache_attention_bytes(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q);
hipError_t launch_cache_attention(const jpi_cache_attn& a, const jpi_cache_pool& p, const jpi_cache_seqs& q, void* ws,
                                  hipStream_t s);

bool moves_fit(const jpi_cache_moves& m);  // whether every launch holds its workgroups
size_t moves_bytes(const jpi_cache_moves& m);
hipError_t launch_resize(const jpi_cache_moves& m, const jpi_cache_pool* pool, int layers, const int32_t* new_len,
                         int32_t* short_out, void* ws, hipStream_t s);
hipError_t launch_reorder(const jpi_cache_moves& m, const int32_t* parents, void* ws, hipStream_t s);
hipError_t launch_compact(const jpi_cache_moves& m, const jpi_cache_pool* pool, int layers, int32_t* n_live_out, void* ws,
                          hipStream_t s);

}  // namespace jpi
