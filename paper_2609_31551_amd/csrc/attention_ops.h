// Shared parts of the language side's attention operators (prompt attention and
// the 8-bit cache): element types, argument checks, the cache's scales and codes.
#pragma once

#include <cmath>

#include "../../include/eas_attention.h"
#include "common.h"

namespace eas {

typedef _Float16 f16;
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int64_t kMaxRowStride = 1 << 23, kMaxHeadStride = 1ll << 31;

// ---- argument checks (host) -------------------------------------------------

inline bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

inline eas_status check_dtype(int32_t dtype) {
  if (dtype == EAS_BF16 || dtype == EAS_FP16) return EAS_OK;
  return dtype == EAS_FP32 ? EAS_ERR_UNSUPPORTED : EAS_ERR_INVALID_ARG;
}

inline eas_status check_strides(const eas_strides& s) {
  if (s.row < 0 || s.head < 0 || s.row % 8 || s.head % 8) return EAS_ERR_INVALID_ARG;
  return s.row > kMaxRowStride || s.head > kMaxHeadStride ? EAS_ERR_UNSUPPORTED : EAS_OK;
}

// An output of `rows` rows must not overlap itself: either whole rows lie apart or whole heads do.
inline eas_status check_out_strides(const eas_strides& s, int64_t rows, int32_t heads, int32_t dim) {
  const eas_status st = check_strides(s);
  if (st != EAS_OK) return st;
  const int64_t by_row = heads > 1 ? (heads - 1) * s.head + dim : dim;   // span of a row's heads
  const int64_t by_head = rows > 1 ? (rows - 1) * s.row + dim : dim;     // span of a head's rows
  if (heads > 1 && s.head < dim) return EAS_ERR_INVALID_ARG;
  if (rows > 1 && s.row < dim) return EAS_ERR_INVALID_ARG;
  return rows <= 1 || heads <= 1 || s.row >= by_row || s.head >= by_head ? EAS_OK : EAS_ERR_INVALID_ARG;
}

inline eas_status check_shape(const eas_attn_shape* s) {
  if (!s) return EAS_ERR_INVALID_ARG;
  const eas_status st = check_dtype(s->dtype);
  if (st != EAS_OK) return st;
  if (s->heads <= 0 || s->kv_heads <= 0 || s->heads > 1024 || s->heads % s->kv_heads) return EAS_ERR_INVALID_ARG;
  // the kernels work on scale * log2(e)
  if ((s->causal != 0 && s->causal != 1) || !std::isfinite(s->scale * kLog2e) || s->head_dim <= 0)
    return EAS_ERR_INVALID_ARG;
  return s->head_dim == 64 || s->head_dim == 128 ? EAS_OK : EAS_ERR_UNSUPPORTED;
}

inline eas_status check_cache(const eas_kv8_cache* c) {
  if (!c || (c->format != EAS_KV_INT8 && c->format != EAS_KV_E4M3)) return EAS_ERR_INVALID_ARG;
  if (c->kv_heads <= 0 || c->kv_heads > 1024 || c->head_dim <= 0 || c->page_tokens <= 0 || c->n_pages <= 0)
    return EAS_ERR_INVALID_ARG;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !aligned16(c->k) || !aligned16(c->v) ||
      (uintptr_t)c->k_scale % 4 || (uintptr_t)c->v_scale % 4)
    return EAS_ERR_INVALID_ARG;
  const int p = c->page_tokens;
  if ((c->head_dim != 64 && c->head_dim != 128) || (p != 16 && p != 32 && p != 64 && p != 128))
    return EAS_ERR_UNSUPPORTED;
  return EAS_OK;
}

// The page table and the sizes that every cache call takes: at most 2^30 tokens of a sequence.
inline eas_status check_table(const eas_kv8_cache* c, const int32_t* pages, int32_t max_pages, int32_t n_seqs) {
  if ((!pages && n_seqs > 0) || max_pages <= 0 || n_seqs < 0 || (uintptr_t)pages % 4) return EAS_ERR_INVALID_ARG;
  return (int64_t)max_pages * c->page_tokens > (1 << 30) ? EAS_ERR_UNSUPPORTED : EAS_OK;
}

// A grid's dimension holds less than 2^32 threads.
inline bool fits_launch(int64_t workgroups, int threads) { return workgroups <= 0xffffffffll / threads; }

// ---- the cache's scales and codes (device) -----------------------------------

// The cache as the kernels get it.
struct Kv8Args {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  int kv_heads, n_pages, page_shift;   // page_tokens = 1 << page_shift
};

inline Kv8Args kv8_args(const eas_kv8_cache* c) {
  return {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, c->kv_heads, c->n_pages,
          __builtin_ctz((unsigned)c->page_tokens)};
}

// Scale for a block whose largest finite magnitude is `top`: 2^e with the smallest
// e >= -126 for which top <= M 2^e (M = 127 = 1.984375 * 2^6, 448 = 1.75 * 2^8); 0 for
// top = 0.  Read off the float's bits: top = m 2^x with 1 <= m < 2, so e = x - 6 (or 8)
// where m is at most M's own leading part, one more above it.
template <int FORMAT>
__device__ __forceinline__ float block_scale(float top) {
  if (!(top > 0.0f)) return 0.0f;
  const uint32_t b = __float_as_uint(top), part = FORMAT == EAS_KV_INT8 ? 0x7e0000u : 0x600000u;
  int e = (int)(b >> 23) - (FORMAT == EAS_KV_INT8 ? 6 : 8) + ((b & 0x7fffffu) > part ? 1 : 0);   // biased by 127
  e = max(e, 1);   // 2^-126 (a subnormal top has biased exponent 0)
  return __uint_as_float((uint32_t)e << 23);
}

// 1 / scale of a power of two in [2^-126, 2^122], 0 for 0 (bf16's largest needs 2^122 in int8)
__device__ __forceinline__ float inverse_scale(float s) {
  return s > 0.0f ? __uint_as_float(0x7f000000u - __float_as_uint(s)) : 0.0f;
}

template <class T>
__device__ __forceinline__ float finite_magnitude(T v) {
  const float a = fabsf((float)v);
  return a < INFINITY ? a : 0.0f;   // NaN compares false
}

// Code of y = x / scale, |y| <= M for finite x: NaN to 0, infinities to the largest code
template <int FORMAT>
__device__ __forceinline__ float code_value(float y) {
  constexpr float M = FORMAT == EAS_KV_INT8 ? 127.0f : 448.0f;
  return y == y ? fminf(fmaxf(y, -M), M) : 0.0f;
}
// Four codes in one word
template <int FORMAT>
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  a = code_value<FORMAT>(a), b = code_value<FORMAT>(b), c = code_value<FORMAT>(c), d = code_value<FORMAT>(d);
  if constexpr (FORMAT == EAS_KV_INT8) {
    const uint32_t ia = (uint32_t)(int)rintf(a) & 255u, ib = (uint32_t)(int)rintf(b) & 255u;
    const uint32_t ic = (uint32_t)(int)rintf(c) & 255u, id = (uint32_t)(int)rintf(d);
    return ia | ib << 8 | ic << 16 | id << 24;
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
}
// The four values that a word's codes stand for, without the scale
template <int FORMAT>
__device__ __forceinline__ void unpack_codes(uint32_t w, float* x) {
  if constexpr (FORMAT == EAS_KV_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> 8 * i);
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
}

}  // namespace eas
