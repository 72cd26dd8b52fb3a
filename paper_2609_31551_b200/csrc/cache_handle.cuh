// What the sources of the language-model operators share: the cache handle and the checks of a call that gets one.
#pragma once
#include "../../include/eas_language.h"

#include "host.cuh"
#include "kv_cache.cuh"

struct eas_cache {
  eas_cache_desc d;
  int device = 0, sm_count = 0, bs_log2 = 0;
  CUtensorMap map_k, map_v;
};

namespace eas {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
constexpr double kLog2e = 1.4426950408889634;

inline eas_status check_cache_call(const eas_cache* c, const eas_cache_seqs* s, bool rows, int32_t dtype, const uint32_t* status_dev, int32_t sm_budget,
                                   int* budget) {
  if (c == nullptr || s == nullptr || status_dev == nullptr) return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
  if (dtype != EAS_DTYPE_BF16 && dtype != EAS_DTYPE_FP16) return fail(EAS_ERR_UNSUPPORTED, "dtype %d", dtype);
  if (s->n_seqs < 0 || s->max_blocks < 0) return fail(EAS_ERR_INVALID_ARG, "n_seqs %d, max_blocks %d", s->n_seqs, s->max_blocks);
  if (s->n_seqs > 0) {
    if ((s->max_blocks > 0 && s->block_table == nullptr) || (rows ? s->cu_seqlens == nullptr || s->start == nullptr : s->seq_lens == nullptr))
      return fail(EAS_ERR_INVALID_ARG, "a required pointer is null");
    if (s->ld_table < s->max_blocks) return fail(EAS_ERR_INVALID_ARG, "ld_table %lld below max_blocks", static_cast<long long>(s->ld_table));
  }
  EAS_TRY(resolve_budget(sm_budget, budget));
  int dev = -1;
  CUDA_TRY(cudaGetDevice(&dev));
  if (dev != c->device) return fail(EAS_ERR_INVALID_ARG, "the cache was created on device %d but device %d is current", c->device, dev);
  return EAS_OK;
}

inline CacheView view_of(const eas_cache* c) {
  return CacheView{c->d.k, c->d.v, c->d.k_scale, c->d.v_scale, c->d.n_blocks, c->d.n_kv_heads, c->bs_log2};
}

}  // namespace eas
