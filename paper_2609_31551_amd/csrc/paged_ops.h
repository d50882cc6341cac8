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

struct Kv16AttnArgs {
  Kv16Args c;
  const void* q;
  void* out;
  float* lse;
  eas_strides qs, os;
  const int* cu_q;
  const int* lens;
  const int* pages;
  float* part;          // results of runs [slots, head_dim]
  float* part_lse;      // and their softmax's log2 sums [slots]
  float scale_log2;     // scale * log2(e)
  int heads, causal, n_rows, max_len, max_pages, n_seqs;
  int max_q, most_q;    // the caller's, and a bound of the queries of a sequence that are computed
  long slots;           // of a sequence; 0: most_runs for each row and head instead
  int most_runs;        // of any sequence within the bounds
  int items;            // of the launch: row tiles and runs of all sequences with many rows
};

// ---- which kernel takes a sequence, and in how many runs of its tokens: by the sequence's own sizes alone, as runs
// are joined with other roundings than one walk's, and a result must not depend on the batch ------------------------

// A sequence's rows of a key / value head, its queries times the group's heads: up to this many are taken 16 at a time
// by waves that share the tokens, more 32 to a wave, all tokens each.
constexpr int FEW_ROWS = 32;
__host__ __device__ inline bool few_rows(int lq, int group) { return (long)lq * group <= FEW_ROWS; }

// Few rows: runs of 1,024 tokens at least
constexpr int FEW_STEP = 128;    // tokens that a run's length is a multiple of
__host__ __device__ inline int few_runs(int len, int nq, int heads, int kv_heads) {
  const int by_len = (int)(((unsigned)len + 1023) / 1024);   // len <= 2^30: 32 bits hold all sums here
  const int most = kv_heads >= 512 ? 1 : 512 / kv_heads < 64 ? 512 / kv_heads : 64;
  return by_len < 1 ? 1 : by_len < most ? by_len : most;
}
__host__ __device__ inline int few_run_tokens(int len, int runs) {
  const unsigned all = (unsigned)runs * FEW_STEP;
  return (int)(((unsigned)len + all - 1) / all) * FEW_STEP;
}

// Many: where the sequence alone leaves CUs without a workgroup
constexpr int MANY_ALONE = 256, MANY_RUNS = 16;
__host__ __device__ inline int many_runs(int len, long rows, int kv_heads) {
  const long alone = (rows + 127) / 128 * kv_heads;   // workgroups of one run
  if (alone > MANY_ALONE) return 1;
  const int shortest = alone <= 32 ? 1024 : alone >= 128 ? 4096 : 32 * (int)alone;
  const int runs = len / shortest;
  return runs < 1 ? 1 : runs < MANY_RUNS ? runs : MANY_RUNS;
}
__host__ __device__ inline int many_run_tiles(int len, int runs) { return ((len + 63) / 64 + runs - 1) / runs; }

// Whether a sequence has few rows, its queries cut to the call's bounds
__device__ __forceinline__ bool takes_few(const Kv16AttnArgs& a, const Seq& s) {
  return few_rows(min(s.lq, a.most_q), a.heads / a.c.kv_heads);
}
// Runs of a sequence, whichever kernel takes it
__device__ __forceinline__ int runs_of(const Kv16AttnArgs& a, const Seq& s) {
  const int group = a.heads / a.c.kv_heads;
  return takes_few(a, s) ? few_runs(s.len, s.nq, a.heads, a.c.kv_heads)
                               : many_runs(s.len, (long)s.nq * group, a.c.kv_heads);
}
// First of a sequence's slots in the workspace: [run, key / value head, row]
__device__ __forceinline__ long first_slot(const Kv16AttnArgs& a, const Seq& s, int r) {
  return a.slots ? r * a.slots : s.row0 * a.heads * a.most_runs;
}
__device__ __forceinline__ bool held_page(const Kv16AttnArgs& a, int page) { return page >= 0 && page < a.c.n_pages; }
// Offset of token t of a key / value head in the cache, `page` its page's number (one that is not held: page 0's)
__device__ __forceinline__ long token_offset(const Kv16AttnArgs& a, int page, int kvh, int t, int dim) {
  const long block = (long)(held_page(a, page) ? page : 0) * a.c.kv_heads + kvh;
  return ((block << a.c.page_shift) + (t & ((1 << a.c.page_shift) - 1))) * dim;
}

// Launches the kernel of the sequences with many rows.
eas_status launch_kv16_many(const Kv16AttnArgs& a, int32_t dtype, int dim, hipStream_t s);

}  // namespace eas
