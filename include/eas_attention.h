/*
 * eas_attention.h -- C ABI of the language side's attention: packed prompts,
 * and a key / value cache held in 8 bits (libeas.so).
 *
 * The embedding rows that leave the encode worker (paper Section 3.3) are
 * consumed by a prefill worker, which may share the encode worker's GPU
 * (Section 3.4), and then by decoding steps (Section 2.1).  These calls are
 * the attention operators of those two stages:
 *   eas_prompt_attention  attention over whole packed prompts, causal or full,
 *                         with grouped heads;
 *   eas_kv8_append        new keys and values into the 8-bit cache;
 *   eas_kv8_rows          cached tokens back as 16-bit rows (a cached prefix
 *                         that the next chunk of a prompt attends to);
 *   eas_kv8_attention     attention of new tokens over the cache.
 *
 * Conventions as in eas_encoder.h: device memory on the current device, work
 * enqueued on `stream` without waiting, no allocation, every call returns an
 * eas_status, argument errors are found on the host before anything is
 * enqueued, no C++ exception crosses the boundary.  A device array named
 * below as such (lengths, page tables) is read by the kernels when they run;
 * what it may hold, and what happens with other values, is said at each call.
 * All calls can be captured into a graph; host arguments are fixed by the
 * capture, device arrays are read anew at each replay.
 *
 * Strides are in elements, multiples of 8, at least 0 and at most 2^23 a row
 * (2^31 a head); tensors start at multiples of 16 bytes.  Row r of head h of a
 * tensor starts at r * row + h * head and holds head_dim consecutive values.
 * An input's stride may be 0 (the same row or head for all); outputs must not
 * overlap themselves or an input.
 */
#ifndef EAS_ATTENTION_H
#define EAS_ATTENTION_H

#include "eas_encoder.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of q, k, v and outputs: EAS_BF16 or EAS_FP16.  EAS_FP32 is not
 * built (EAS_ERR_UNSUPPORTED). */
enum { EAS_FP16 = 2 };

/* A tensor's strides. */
typedef struct {
  int64_t row, head;
} eas_strides;

typedef struct {
  int32_t dtype;            /* EAS_BF16 or EAS_FP16: q, k, v and out             */
  int32_t heads, kv_heads;  /* query head h reads key / value head h / (heads / kv_heads); */
                            /* heads is a multiple of kv_heads, at most 1024     */
  int32_t head_dim;         /* 64 or 128                                         */
  int32_t causal;           /* 1 or 0                                            */
  float scale;              /* multiplies q . k; 2.3e38 at most, so that scale * log2(e) is finite */
  eas_strides q, k, v, out;
} eas_attn_shape;

/* Attention over packed prompts.  Sequence r has the queries
 * cu_q[r] .. cu_q[r+1] and the keys cu_k[r] .. cu_k[r+1]; Lq and Lk of them.
 * Its query i sees key j where j <= i + Lk - Lq (causal: the queries are the
 * last Lq of the Lk tokens) or every key (full):
 *   out[i, h] = sum_j p_j v[j, h'],  p = softmax_j(scale * q[i, h] . k[j, h']).
 * A query that sees no key gets zeros.  Sums and the softmax are held in fp32,
 * probabilities are rounded to the element type for the product with v.
 * cu_q, cu_k: host, [n_seqs + 1] prefix sums from 0, not decreasing, equal
 * neighbours allowed; cu_k NULL = cu_q.  0 <= n_seqs <= EAS_MAX_SEQS.
 * lse: device fp32 [cu_q[n_seqs], heads] or NULL: the natural logarithm of each
 * softmax's sum of exponentials, -inf where no key is seen.
 * Rows of out and lse outside [0, cu_q[n_seqs]) are not touched.  A sequence's
 * result does not depend on the others, to the bit.
 * k and v may hold anything, NaN included, outside the sequences' keys, and
 * what a query does not see never reaches its result.  A key whose score is
 * -inf (an infinite dimension, or products that overflow fp32) weighs nothing;
 * a query whose scores are all -inf gets zeros and lse -inf, as one that sees no
 * key.  A score of NaN or +inf makes a query's result and lse NaN; a value of
 * NaN or infinity makes that dimension of the result of who sees it infinite or
 * NaN, whatever its weight.
 * workspace: device, 16-byte aligned, at least the bytes that
 * eas_prompt_attention_workspace gives for the same arguments (0: NULL is
 * fine), which is more than 0 only where few queries see 2,048 keys or more;
 * calls that may overlap, captured ones included, need one each.  Nothing in it
 * has to be set before, or is kept from call to call.  A sequence's share goes by
 * its own sizes, as its result does: 2^19 * (head_dim + 1) * 4 bytes at most, 258
 * MiB at heads of 128 (1,024 queries of 32 heads over 65,536 keys), however many
 * are in the batch.
 * Errors: INVALID_ARG, SHAPE (cu_q, cu_k), CAPACITY (n_seqs, the workspace),
 * UNSUPPORTED (element type, head_dim, strides, more than 2^30 queries or keys,
 * more threads than a launch holds, 2^32 - 1: 2 for each query and head). */
eas_status eas_prompt_attention(const eas_attn_shape* shape, const void* q, const void* k, const void* v,
                                const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs, void* out, float* lse,
                                void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes of eas_prompt_attention (host only, no HIP calls; the
 * shape's strides are not read). */
eas_status eas_prompt_attention_workspace(const eas_attn_shape* shape, const int32_t* cu_q, const int32_t* cu_k,
                                          int32_t n_seqs, int64_t* bytes);

/* The cache.  A block -- page_tokens tokens of one head -- is held as 8-bit
 * codes and one scale, a power of two or 0: value = code * scale.  Scale 2^e
 * has the smallest e >= -126 under which the block's finite values fit into
 * [-127, 127] (int8) or [-448, 448] (e4m3); 0 stands for a block of zeros.
 * Powers of two make coding, decoding and every change of scale exact but for
 * the code's own rounding (to nearest, ties to even). */
enum { EAS_KV_INT8 = 0, EAS_KV_E4M3 = 1 };

typedef struct {
  int32_t format;           /* EAS_KV_INT8 or EAS_KV_E4M3                        */
  int32_t kv_heads, head_dim;   /* head_dim 64 or 128                            */
  int32_t page_tokens;      /* 16, 32, 64 or 128                                 */
  int32_t n_pages;
  void* k;                  /* device codes [n_pages, kv_heads, page_tokens, head_dim] */
  void* v;                  /* device codes [n_pages, kv_heads, head_dim, page_tokens]: */
                            /* a lane of the attention kernel wants one dimension of   */
                            /* consecutive tokens                                */
  float* k_scale;           /* device [n_pages, kv_heads]                        */
  float* v_scale;
} eas_kv8_cache;

/* The page table of the calls below: device int32 [n_seqs, max_pages]; token t
 * of sequence r lies in page pages[r, t / page_tokens]; max_pages * page_tokens
 * is at most 2^30.  An entry outside
 * [0, n_pages) is a page that is not held: tokens appended to it are dropped,
 * its rows read as zeros, and attention does not see its tokens.  Pages may be
 * shared between sequences for reading.  A page that gets tokens in a call is
 * named once in it: appended to from two places, its codes are undefined.
 * The calls launch workgroups of up to 256 threads for what the host's bounds
 * allow -- every sequence, head and page that max_new tokens, 64 rows of max_rows
 * or 16 queries of max_q and a run of max_len tokens can touch -- and refuse
 * bounds that allow 2^32 threads or more over the sequences (append, rows) or
 * over sequences and heads (attention) with EAS_ERR_UNSUPPORTED: bounds near the
 * batch's own avoid that. */

/* Appends new keys and values.  k, v: device [n_rows] rows of kv_heads heads.
 * Sequence r's new tokens are rows cu_new[r] .. cu_new[r+1] (device int32
 * [n_seqs + 1]) or, where cu_new is NULL, rows r * max_new .. (r+1) * max_new;
 * they become its tokens held[r], held[r] + 1, ... (held: device int32
 * [n_seqs], the tokens that it holds before the call; not changed here).
 * A block's scale only grows while it fills: where the new tokens need a
 * larger one, the codes of its earlier tokens are rounded anew to the larger
 * step; the block of a token at a page's start is begun anew.  NaN is stored
 * as 0 and infinities as the largest code of their sign; neither counts
 * towards the scale.
 * max_new: host, at least the number of new tokens of every sequence (tokens
 * beyond are dropped).  Rows outside [0, n_rows) and tokens at or beyond
 * max_pages * page_tokens are dropped, a sequence with held[r] < 0 is left out.
 * Codes of places that get no token and lie before none stay as they are. */
eas_status eas_kv8_append(const eas_kv8_cache* cache, int32_t dtype, const void* k, eas_strides k_strides,
                          const void* v, eas_strides v_strides, int32_t n_rows, const int32_t* cu_new,
                          int32_t max_new, const int32_t* held, const int32_t* pages, int32_t max_pages,
                          int32_t n_seqs, void* stream);

/* Cached tokens back as rows: rows cu_rows[r] .. cu_rows[r+1] (device int32
 * [n_seqs + 1]) of k and v receive sequence r's tokens first[r], first[r] + 1,
 * ... (first: device int32 [n_seqs]; NULL = 0).  k or v may be NULL: not read.
 * max_rows: host, at least the rows of every sequence (rows beyond are not
 * written).  Rows outside [0, n_rows) are not written; tokens below 0 or at or
 * beyond max_pages * page_tokens read as zeros.  A cached value that the
 * element type cannot hold is rounded to it (fp16: to infinity above 65504). */
eas_status eas_kv8_rows(const eas_kv8_cache* cache, int32_t dtype, const int32_t* pages, int32_t max_pages,
                        int32_t n_seqs, const int32_t* cu_rows, const int32_t* first, int32_t max_rows,
                        int32_t n_rows, void* k, eas_strides k_strides, void* v, eas_strides v_strides, void* stream);

/* Attention of new tokens over the cache, which holds them already.  shape:
 * as for eas_prompt_attention (its k and v strides are not read); kv_heads and
 * head_dim as the cache's.  q, out: device [n_rows] rows; sequence r's queries
 * are rows cu_q[r] .. cu_q[r+1] (device int32 [n_seqs + 1]) or, where cu_q is
 * NULL, rows r * max_q .. (r+1) * max_q.  It attends to its first lens[r]
 * tokens (device int32 [n_seqs]), its Lq queries being the last Lq of them
 * where causal: query i sees token j <= i + lens[r] - Lq.
 * max_q, max_len: host, at least the queries and tokens of every sequence
 * (queries beyond are not computed, tokens beyond are not seen).  Lengths are
 * cut to [0, max_pages * page_tokens]; rows outside [0, n_rows) are not
 * touched.  Queries and tokens that are left out so leave the others' places i
 * and j, Lq and lens[r] as they are.  A query that sees no token gets zeros and lse -inf.  Scores of -inf,
 * +inf and NaN do what they do in eas_prompt_attention.
 * lse: device fp32 [n_rows, heads] or NULL.
 * A row's values of q are taken to fp16 relative to its largest, each good to
 * 2^-39 of that (exactly, where it is 2^-31 of the largest or more); their
 * products with the codes are exact, sums and the softmax are held in fp32, and
 * weights are rounded to fp16 for the product with the values' codes.
 * workspace: device, 16-byte aligned, at least the bytes that
 * eas_kv8_attention_workspace gives for the same arguments (0, up to a max_len
 * of 1,024: NULL is fine); calls that may overlap, captured ones included, need
 * one each.  Nothing in it has to be set before, or is kept from call to call.
 * It grows with max_q up to 256 * heads * (head_dim + 1) * 4 bytes a sequence.
 * A sequence's result does not depend on the other sequences, on max_q, on
 * max_len or on which pages hold its tokens, to the bit.
 * Made for a few queries of each sequence.  From 128 on, eas_kv8_rows and
 * eas_prompt_attention over the rows take less time: 8 sequences of 4,096 tokens,
 * 32 heads of 128 over 8, with 64 queries each 102 us here and 105 there, with
 * 128 289 and 146, with 512 1,836 and 277. */
eas_status eas_kv8_attention(const eas_kv8_cache* cache, const eas_attn_shape* shape, const void* q, int32_t n_rows,
                             const int32_t* cu_q, int32_t max_q, const int32_t* lens, int32_t max_len,
                             const int32_t* pages, int32_t max_pages, int32_t n_seqs, void* out, float* lse,
                             void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes of eas_kv8_attention (host only, no HIP calls). */
eas_status eas_kv8_attention_workspace(const eas_attn_shape* shape, int32_t max_q, int32_t max_len, int32_t n_seqs,
                                       int64_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* EAS_ATTENTION_H */
