// Shared parts of the calls over the paged 16-bit cache (include/eas_paged.h).
#pragma once

#include "../../include/eas_paged.h"
#include "attention_ops.h"

namespace eas {

inline eas_status check_cache16(const eas_kv16_cache* c) {
  if (!c) return EAS_ERR_INVALID_ARG;
  const eas_status st = check_dtype(c->dtype);
  if (st != EAS_OK) return st;
  if (c->kv_heads <= 0 || c->kv_heads > 1024 || c->head_dim <= 0 || c->page_tokens <= 0 || c->n_pages <= 0)
    return EAS_ERR_INVALID_ARG;
  if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return EAS_ERR_INVALID_ARG;
  const int p = c->page_tokens;
  if ((c->head_dim != 64 && c->head_dim != 128) || (p != 16 && p != 32 && p != 64 && p != 128))
    return EAS_ERR_UNSUPPORTED;
  return EAS_OK;
}

// The page table: at most 2^30 tokens of a sequence.
inline eas_status check_table16(const eas_kv16_cache* c, const int32_t* pages, int32_t max_pages, int32_t n_seqs) {
  if ((!pages && n_seqs > 0) || max_pages <= 0 || n_seqs < 0 || (uintptr_t)pages % 4) return EAS_ERR_INVALID_ARG;
  return (int64_t)max_pages * c->page_tokens > (1 << 30) ? EAS_ERR_UNSUPPORTED : EAS_OK;
}

// The cache as the attention kernels get it.
struct Kv16Args {
  const void* k;
  const void* v;
  int kv_heads, n_pages, page_shift;   // page_tokens = 1 << page_shift
};

inline Kv16Args kv16_args(const eas_kv16_cache* c) {
  return {c->k, c->v, c->kv_heads, c->n_pages, __builtin_ctz((unsigned)c->page_tokens)};
}

}  // namespace eas
