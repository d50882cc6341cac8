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
  int items, few_blocks;   // of the launch: row tiles and runs of sequences with many rows, or rows joined of each
                           // sequence; workgroups for those with few, which come first
};

// ---- which kernel takes a sequence, and in how many runs of its tokens: by the sequence's own sizes alone, as runs
// are joined with other roundings than one walk's, and a result must not depend on the batch ------------------------

// A sequence's rows of a key / value head, its queries times the group's heads: up to this many are taken whole by each
// wave, which share the tokens out; more are taken 32 to a wave, all tokens each.  (Up to 64 as two workgroups that read the
// same tokens: four sequences of 4,096, five queries of 28 heads over 4 22 us and 23, sixteen 53 and 42.)
constexpr int FEW_ROWS = 32;
__host__ __device__ inline bool few_rows(int lq, int group) { return (long)lq * group <= FEW_ROWS; }

// Few rows: beyond 1,024 tokens, runs of 1,024 or, up to 128 workgroups of a sequence, of 512.  A run costs its first loads
// and its share of the join, and one alone draws no more than one CU's loads: one sequence of 4,096 tokens, 8 heads, 14 us
// in runs of 512 and 18 in runs of 1,024; 32 of them 103 and 99; 64 of 1,024 51 whole and 57 in two.
constexpr int FEW_STEP = 128;    // tokens that a run's length is a multiple of
__host__ __device__ inline int few_runs(int len, int kv_heads) {
  if (len <= 1024) return 1;
  const int whole = (len + 1023) / 1024, halves = (len + 511) / 512, fill = (128 + kv_heads - 1) / kv_heads;
  const int by_len = halves < fill ? halves : whole > fill ? whole : fill;
  const int most = kv_heads >= 512 ? 1 : 512 / kv_heads < 64 ? 512 / kv_heads : 64;
  return by_len < most ? by_len : most;
}
__host__ __device__ inline int few_run_tokens(int len, int runs) {
  const unsigned all = (unsigned)runs * FEW_STEP;
  return (int)(((unsigned)len + all - 1) / all) * FEW_STEP;
}

// Many: where the sequence alone leaves CUs without a workgroup, runs of 2,048 tokens, down to 512 where it has few
// workgroups without, up to 512 workgroups.  A call waits for its longest walk, and a batch that fills the chip anyway
// pays for the runs' sums: 512 queries of 28 heads over 4 over 8,192 tokens 79 us, in runs of 4,096 111, eight of them 542
// and 543; 512 of 32 over 8 over 4,096 56 and, whole, 96; 64 over 4,096 31 and, in runs of 512, 25, sixteen 99 and 126.
constexpr int MANY_ALONE = 256, MANY_FILL = 512;
__host__ __device__ inline int many_runs(int len, long rows, int kv_heads) {
  const long alone = (rows + 127) / 128 * kv_heads;   // workgroups of one run
  if (len <= 1024 || alone > MANY_ALONE) return 1;
  const int by_len = len / (alone <= 8 ? 512 : alone <= 64 ? 1024 : 2048), fill = MANY_FILL / (int)alone;
  const int runs = by_len < fill ? by_len : fill;
  return runs < 1 ? 1 : runs < 64 ? runs : 64;
}
__host__ __device__ inline int many_run_tiles(int len, int runs) { return ((len + 63) / 64 + runs - 1) / runs; }

// Whether a sequence has few rows, its queries cut to the call's bounds
__device__ __forceinline__ bool takes_few(const Kv16AttnArgs& a, const Seq& s) {
  return few_rows(min(s.lq, a.most_q), a.heads / a.c.kv_heads);
}
// Runs of a sequence, whichever kernel takes it
__device__ __forceinline__ int runs_of(const Kv16AttnArgs& a, const Seq& s) {
  const int group = a.heads / a.c.kv_heads;
  return takes_few(a, s) ? few_runs(s.len, a.c.kv_heads)
                               : many_runs(s.len, (long)s.nq * group, a.c.kv_heads);
}
// First of a sequence's slots in the workspace: [run, key / value head, row]
__device__ __forceinline__ long first_slot(const Kv16AttnArgs& a, const Seq& s, int r) {
  return a.slots ? r * a.slots : s.row0 * a.heads * a.most_runs;
}
// 16 tokens of a page that is not held
__device__ const uint4 absent_tokens[16 * 128 * 2 / 16] = {};
__device__ __forceinline__ bool held_page(const Kv16AttnArgs& a, int page) { return page >= 0 && page < a.c.n_pages; }
// Offset of token t of a key / value head in the cache, `page` its page's number (one that is not held: page 0's)
__device__ __forceinline__ long token_offset(const Kv16AttnArgs& a, int page, int kvh, int t, int dim) {
  const long block = (long)(held_page(a, page) ? page : 0) * a.c.kv_heads + kvh;
  return ((block << a.c.page_shift) + (t & ((1 << a.c.page_shift) - 1))) * dim;
}

// Sum of v over the lanes up to and with this one, by DPP: within rows of 16 lanes, then of the rows before.
__device__ __forceinline__ int sum_upto(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15, to the odd rows
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31, to the upper two
  return v;
}

// Pieces of work of a launch that sequence r has count(its Seq) of, in an order of the sequences: lane i of a wave goes
// over i, i + 64, .. one after the other, and, to find one, the wave over a lane's.  Of more than 64 sequences the waves
// of the workgroup, all of which come here together, take a share each (1,024 of 2,048 tokens, 4 heads, 4,096 allowed:
// 914 us, each wave over all 1,060; 4,096 of them 4.3 and 7.4 ms; a chunk of 512 beside 255 single tokens 159 and 197 us).
// Prefix sums that decrease would let rows, and pieces, be counted again and again: a lane counts MOST at most, more than a
// launch has workgroups for, so that no sum wraps and a piece that is found is one of its sequence's.
template <class Count>
struct Items {
  const Kv16AttnArgs& a;
  const Count count;
  int each;         // sequences of a lane
  Seq seq;          // of the last one that the lane looked at: its only one where there are 64 at most
  int own, upto;    // the lane's pieces, and those of it and of the lanes before
  static constexpr int MOST = (1 << 25) - 1;   // a sequence has 2^24 at most

  __device__ __forceinline__ Items(const Kv16AttnArgs& a_, const Count& count_) : a(a_), count(count_) {
    each = (unsigned)(a.n_seqs + 63) / 64;
    if (each == 1) {
      own = look(threadIdx.x & 63);
    } else {
      __shared__ int shares[8][64];   // a later one's are written behind a barrier of the caller's
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
      own = 0;
#pragma unroll 2
      for (int i = wave; i < each; i += waves) own = min(own + look(i * 64 + lane), MOST);
      shares[wave][lane] = own;
      __syncthreads();
      own = 0;
      for (int w = 0; w < waves; ++w) own = min(own + shares[w][lane], MOST);
    }
    upto = sum_upto(own);
  }
  __device__ __forceinline__ int look(int r) {
    seq = find_seq(a, min(r, a.n_seqs - 1));
    return r < a.n_seqs ? count(seq) : 0;
  }
  __device__ __forceinline__ int all() const { return __builtin_amdgcn_readlane(upto, 63); }
  // The sequence of the `*item`th piece, below all(), which becomes its number among the sequence's own.
  __device__ __forceinline__ int find(int* item, Seq* s) {
    int at = first_above(upto, *item), r = at, left = *item - __builtin_amdgcn_readlane(upto - own, at);
    if (each > 1) {
      const int first = at, lane = threadIdx.x & 63;
      for (int i = 0;; i += 64) {
        const int mine = i + lane < each ? look((i + lane) * 64 + first) : 0, so_far = sum_upto(mine);
        if (left < __builtin_amdgcn_readlane(so_far, 63)) {
          at = first_above(so_far, left);
          left -= __builtin_amdgcn_readlane(so_far - mine, at);
          r = (i + at) * 64 + first;
          break;
        }
        left -= __builtin_amdgcn_readlane(so_far, 63);
      }
    }
    const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
    *item = __builtin_amdgcn_readfirstlane(left);
    *s = {(long)((uint64_t)(uint32_t)of((int)seq.row0) | (uint64_t)of((int)(seq.row0 >> 32)) << 32), of(seq.before),
          of(seq.nq), of(seq.len), of(seq.lq)};
    return __builtin_amdgcn_readfirstlane(r);
  }
  // The first lane whose v is above x, where some lane's is
  __device__ __forceinline__ static int first_above(int v, int x) {
    return __builtin_amdgcn_readfirstlane(__ffsll(__ballot(v > x)) - 1);
  }
};

}  // namespace eas
