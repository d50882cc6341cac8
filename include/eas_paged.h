/*
 * eas_paged.h -- C ABI of prompts in pieces on the language side: rotary
 * positions with several axes, and a paged key / value cache in 16 bits
 * (libeas.so).
 *
 * A prefill worker that takes a long prompt of image and video rows in chunks,
 * and the decoding steps after it (paper Section 2.1), do three things in every
 * layer that eas_attention.h's calls over whole prompts and over the 8-bit cache
 * leave to the caller:
 *   eas_rotary_rows     rotates heads by positions of one to four axes (time,
 *                       height, width), or takes a rotation back;
 *   eas_kv16_append     new keys, rotated on the way, and values into the cache,
 *                       and the new queries rotated beside them;
 *   eas_kv16_attention  attention of new tokens -- one of each sequence, a few,
 *                       or whole chunks, mixed as they come -- over the cache.
 *
 * Conventions as in eas_attention.h: device memory on the current device, work
 * enqueued on `stream` without waiting, no allocation, argument errors found on
 * the host before anything is enqueued, device arrays read when the kernels
 * run, calls that can be captured into a graph.  Strides as there.
 */
#ifndef EAS_PAGED_H
#define EAS_PAGED_H

#include "eas_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { EAS_MAX_ROTARY_PAIRS = 128, EAS_MAX_ROTARY_AXES = 4 };

/* A rotation: what a model's positions do to a head.  Pair i of a head's
 * dimensions, (x, y), turns by the angle a = p[axis[i]] * freq[i], p the row's
 * positions:
 *   x' = x cos a - y sin a,  y' = x sin a + y cos a.
 * Pair i is dimensions (i, i + pairs), or (2 i, 2 i + 1) where adjacent;
 * dimensions from 2 pairs on pass as they are.  Filled by eas_rotary_make; plain
 * data, read on the host by the calls that take it. */
typedef struct {
  int32_t pairs;      /* 8 .. EAS_MAX_ROTARY_PAIRS, a multiple of 8             */
  int32_t axes;       /* 1 .. EAS_MAX_ROTARY_AXES                               */
  int32_t adjacent;   /* 1 or 0                                                 */
  int32_t reserved;   /* 0                                                      */
  uint64_t step[EAS_MAX_ROTARY_PAIRS];   /* a pair's turn for one position, in 2^-64 of a whole turn */
  uint8_t axis[EAS_MAX_ROTARY_PAIRS];
} eas_rotary;

/* freqs: [pairs] radians for one position, finite, less than 2^60 either way;
 * axis: [pairs], each in [0, axes), or NULL (0 for all).  A turn is kept to the
 * nearest 2^-64 of a whole one, so that positions multiply it exactly, modulo
 * whole turns: angles are good to about 2^-23 radians at any position of 32
 * bits.  Host only.
 * Errors: INVALID_ARG, UNSUPPORTED (pairs, axes, frequencies from 2^60 on). */
eas_status eas_rotary_make(const double* freqs, const int32_t* axis, int32_t pairs, int32_t axes, int32_t adjacent,
                           eas_rotary* rotary);

/* Rotates the rows of q [n_rows, heads, head_dim] and, where k is not NULL, of
 * k [n_rows, kv_heads, head_dim] into q_out and k_out, which may be q and k
 * themselves (with the same strides) and else overlap no input.
 * inverse: 0, or 1 for the opposite angles: takes a rotation back, and gives
 * from the gradients of rotated rows those of the rows themselves.
 * positions: device int32; axis a's of row r is at [a * axis_stride + r]
 * (axis_stride 0: the same for all axes), negative ones as they come.
 * head_dim: a multiple of 16 up to 256, 2 * pairs at least.  Sums are held in
 * fp32 and rounded once.
 * Errors: INVALID_ARG, UNSUPPORTED (element type, head_dim, strides, more
 * threads than a launch holds). */
eas_status eas_rotary_rows(const eas_rotary* rotary, int32_t dtype, int32_t head_dim, int32_t inverse,
                           const int32_t* positions, int64_t axis_stride, int32_t n_rows, const void* q,
                           eas_strides q_strides, int32_t heads, void* q_out, eas_strides q_out_strides, const void* k,
                           eas_strides k_strides, int32_t kv_heads, void* k_out, eas_strides k_out_strides,
                           void* stream);

/* The cache: keys and values as they are attended to, in the element type. */
typedef struct {
  int32_t dtype;                /* EAS_BF16 or EAS_FP16                         */
  int32_t kv_heads, head_dim;   /* at most 1024; 64 or 128                      */
  int32_t page_tokens;          /* 16, 32, 64 or 128                            */
  int32_t n_pages;
  void* k;                      /* device [n_pages, kv_heads, page_tokens, head_dim] */
  void* v;                      /* the same                                     */
} eas_kv16_cache;

/* Page tables as in eas_attention.h: device int32 [n_seqs, max_pages], an entry
 * outside [0, n_pages) is a page that is not held, pages may be shared for
 * reading, and a page that gets tokens in a call is named once in it. */

/* Appends new keys and values, and rotates new queries.
 * k, v: device [n_rows] rows of kv_heads heads.  Sequence r's new tokens are rows
 * cu_new[r] .. cu_new[r+1] (device int32 [n_seqs + 1], not decreasing) or, where
 * cu_new is NULL, rows r * max_new .. (r+1) * max_new; they become its tokens
 * held[r], held[r] + 1, ... (held: device int32 [n_seqs]; not changed here).
 * rotary: NULL, or the rotation of keys and queries; positions: device int32
 * [axes, n_rows] as in eas_rotary_rows, or NULL: a token's place in its
 * sequence, on all axes.
 * q: NULL, or device [n_rows] rows of heads heads that are rotated into q_out (q
 * itself, with the same strides, or rows that overlap no input); only with
 * rotary.
 * max_new: host, at least the number of new tokens of every sequence.  Left out,
 * keys, values and queries: rows of no sequence, tokens beyond max_new, sequences
 * with held[r] < 0.  Keys and values of pages that are not held and of tokens at
 * or beyond max_pages * page_tokens are dropped (their queries are rotated).
 * Places of the cache that get no token stay as they are.
 * Errors: INVALID_ARG, UNSUPPORTED (element type, head_dim, page_tokens, strides,
 * more than 2^30 tokens of a sequence or threads than a launch holds). */
eas_status eas_kv16_append(const eas_kv16_cache* cache, const eas_rotary* rotary, const int32_t* positions,
                           int64_t axis_stride, const void* q, eas_strides q_strides, int32_t heads, void* q_out,
                           eas_strides q_out_strides, const void* k, eas_strides k_strides, const void* v,
                           eas_strides v_strides, int32_t n_rows, const int32_t* cu_new, int32_t max_new,
                           const int32_t* held, const int32_t* pages, int32_t max_pages, int32_t n_seqs, void* stream);

/* Attention of new tokens over the cache, which holds them already: arguments,
 * what is seen, what is left out, and rows that see nothing as in
 * eas_kv8_attention (shape: its k and v strides are not read; dtype, kv_heads
 * and head_dim as the cache's), but that the prefix sums in cu_q must not
 * decrease: with sums that do, any row within [0, n_rows) may get anything.
 * A key's score of -inf, +inf or NaN and a value's infinities do what they do in
 * eas_prompt_attention, and what a query does not see never reaches its result.
 * Sums and the softmax are held in fp32, in whose range they stay for all finite
 * values; probabilities are rounded to the element type for the product with v.
 * A sequence's result does not depend on the other sequences, on max_q and
 * max_len that hold for it, on which pages hold its tokens, or on what is in
 * places of the cache that hold none of them, to the bit.
 * workspace: device, 16-byte aligned, at least the bytes that
 * eas_kv16_attention_workspace gives for the same arguments (0: NULL is fine);
 * calls that may overlap, captured ones included, need one each.  Nothing in it
 * has to be set before, or is kept from call to call. */
eas_status eas_kv16_attention(const eas_kv16_cache* cache, const eas_attn_shape* shape, const void* q, int32_t n_rows,
                              const int32_t* cu_q, int32_t max_q, const int32_t* lens, int32_t max_len,
                              const int32_t* pages, int32_t max_pages, int32_t n_seqs, void* out, float* lse,
                              void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes of eas_kv16_attention (host only, no HIP calls). */
eas_status eas_kv16_attention_workspace(const eas_attn_shape* shape, int32_t n_rows, int32_t max_q, int32_t max_len,
                                        int32_t n_seqs, int64_t* bytes);

#ifdef __cplusplus
}
#endif

#endif /* EAS_PAGED_H */
