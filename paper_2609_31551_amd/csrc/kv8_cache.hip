// The 8-bit key / value cache: append and rows (include/eas_attention.h).
//
// A workgroup owns one block -- a page's tokens of one head -- of one sequence, in
// both calls, so nothing is shared between workgroups and no order matters.  Both are
// bound by HBM: an append reads 2 bytes and writes 1 for each value, rows the reverse.
#include "attention_ops.h"

namespace eas {
namespace {

constexpr int NT = 256;

struct AppendArgs {
  Kv8Args c;
  const void* k;
  const void* v;
  eas_strides ks, vs;
  const int* cu_new;
  const int* held;
  const int* pages;
  int n_rows, max_new, max_pages, blocks;   // blocks: pages that one sequence's new tokens can touch
};

// The tokens [lo, hi) of one page that a sequence appends, and their first row.
struct Span {
  int page, lo, hi;
  long row;
};

__device__ __forceinline__ bool find_span(const AppendArgs& a, int r, int b, Span* s) {
  const int held = a.held[r];
  if (held < 0) return false;
  long row0, n;
  if (a.cu_new) {
    row0 = a.cu_new[r];
    n = (long)a.cu_new[r + 1] - row0;
  } else {
    row0 = (long)r * a.max_new;
    n = a.max_new;
  }
  if (row0 < 0) return false;
  n = min(n, min((long)a.max_new, a.n_rows - row0));
  const long slot = (held >> a.c.page_shift) + (long)b;
  if (n <= 0 || slot >= a.max_pages) return false;
  const long lo = max((long)held, slot << a.c.page_shift), hi = min(held + n, (slot + 1) << a.c.page_shift);
  if (lo >= hi) return false;
  s->page = a.pages[(long)r * a.max_pages + slot];
  if (s->page < 0 || s->page >= a.c.n_pages) return false;
  s->row = row0 + (lo - held);
  s->lo = (int)(lo - (slot << a.c.page_shift));
  s->hi = (int)(hi - (slot << a.c.page_shift));
  return true;
}

__device__ __forceinline__ float group_max(float v, float* red) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// One block of keys (TURNED false: codes [page][D]) or values (codes [D][page]).
template <class T, int FORMAT, int D, bool TURNED>
__device__ void append_block(const AppendArgs& a, const Span& s, int h, const T* x, const eas_strides& st,
                             uint8_t* codes, float* scales, float* red) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  const int page = 1 << a.c.page_shift, chunks = (s.hi - s.lo) * (D / 8);
  const long block = (long)s.page * a.c.kv_heads + h;
  codes += block << (a.c.page_shift + (D == 64 ? 6 : 7));
  x += s.row * st.row + h * st.head;
  float top = 0.0f;
  for (int i = threadIdx.x; i < chunks; i += NT) {
    const Tx8 v = *reinterpret_cast<const Tx8*>(x + (long)(i / (D / 8)) * st.row + i % (D / 8) * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_magnitude(v[e]));
  }
  top = group_max(top, red);
  const float before = s.lo > 0 ? scales[block] : 0.0f;
  const float scale = fmaxf(before, block_scale<FORMAT>(top)), inv = inverse_scale(scale);
  __syncthreads();   // every thread has read the old scale
  if (threadIdx.x == 0) scales[block] = scale;
  if (scale > before && before > 0.0f) {   // the earlier tokens' codes to the larger step
    const float ratio = before * inv;
    for (int i = threadIdx.x; i < s.lo * (D / 4); i += NT) {
      uint8_t* p;
      int step;
      if (TURNED) {
        p = codes + ((i / s.lo * 4) << a.c.page_shift) + i % s.lo;
        step = page;
      } else {
        p = codes + i * 4;
        step = 1;
      }
      float y[4];
      unpack_codes<FORMAT>(p[0] | p[step] << 8 | p[2 * step] << 16 | (uint32_t)p[3 * step] << 24, y);
      const uint32_t w = pack_codes<FORMAT>(y[0] * ratio, y[1] * ratio, y[2] * ratio, y[3] * ratio);
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e * step] = (uint8_t)(w >> 8 * e);
    }
  }
  for (int i = threadIdx.x; i < chunks; i += NT) {
    const int t = i / (D / 8), d = i % (D / 8) * 8;
    const Tx8 v = *reinterpret_cast<const Tx8*>(x + (long)t * st.row + d);
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const uint32_t w = pack_codes<FORMAT>((float)v[e] * inv, (float)v[e + 1] * inv, (float)v[e + 2] * inv,
                                            (float)v[e + 3] * inv);
      if (TURNED) {
#pragma unroll
        for (int f = 0; f < 4; ++f)
          codes[((d + e + f) << a.c.page_shift) + s.lo + t] = (uint8_t)(w >> 8 * f);
      } else {
        *reinterpret_cast<uint32_t*>(codes + (s.lo + t) * D + d + e) = w;
      }
    }
  }
}

template <class T, int FORMAT, int D>
__global__ __launch_bounds__(NT) void kv8_append_kernel(AppendArgs a) {
  __shared__ float red[4];
  Span s;
  if (!find_span(a, blockIdx.x / a.blocks, blockIdx.x % a.blocks, &s)) return;
  const int h = blockIdx.y;
  append_block<T, FORMAT, D, false>(a, s, h, static_cast<const T*>(a.k), a.ks, a.c.k, a.c.k_scale, red);
  append_block<T, FORMAT, D, true>(a, s, h, static_cast<const T*>(a.v), a.vs, a.c.v, a.c.v_scale, red);
}

struct RowsArgs {
  Kv8Args c;
  void* k;
  void* v;
  eas_strides ks, vs;
  const int* cu;
  const int* first;
  const int* pages;
  int n_rows, max_rows, max_pages, blocks;   // blocks: pages that one sequence's rows can touch
};

template <class T, int FORMAT, int D>
__global__ __launch_bounds__(NT) void kv8_rows_kernel(RowsArgs a) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  const int r = blockIdx.x / a.blocks, b = blockIdx.x % a.blocks, h = blockIdx.y;
  const int page = 1 << a.c.page_shift;
  const long row0 = a.cu[r], n = min((long)a.cu[r + 1] - row0, (long)a.max_rows);
  const long first = a.first ? a.first[r] : 0;
  const long slot = (first >> a.c.page_shift) + b;   // of a sequence that starts below 0, pages below 0 too
  const long lo = max(first, slot * page), hi = min(first + n, (slot + 1) * page);
  if (lo >= hi) return;
  int id = -1;
  if (slot >= 0 && slot < a.max_pages) id = a.pages[(long)r * a.max_pages + slot];
  const bool there = id >= 0 && id < a.c.n_pages;
  const long block = (long)(there ? id : 0) * a.c.kv_heads + h;
  const int chunks = (int)(hi - lo) * (D / 8), t0 = (int)(lo - slot * page);
  const uint8_t* kc = a.c.k + block * page * D;
  const uint8_t* vc = a.c.v + block * page * D;
  const float ks = there ? a.c.k_scale[block] : 0.0f, vs = there ? a.c.v_scale[block] : 0.0f;
  for (int i = threadIdx.x; i < chunks; i += NT) {
    const int t = i / (D / 8), d = i % (D / 8) * 8;
    const long row = row0 + (lo - first) + t;
    if (row < 0 || row >= a.n_rows) continue;
    if (a.k) {
      Tx8 o;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        float x[4];
        unpack_codes<FORMAT>(*reinterpret_cast<const uint32_t*>(kc + (t0 + t) * D + d + e), x);
#pragma unroll
        for (int f = 0; f < 4; ++f) o[e + f] = there ? (T)(x[f] * ks) : (T)0.0f;
      }
      *reinterpret_cast<Tx8*>(static_cast<T*>(a.k) + row * a.ks.row + h * a.ks.head + d) = o;
    }
    if (a.v) {
      Tx8 o;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x[4];
        unpack_codes<FORMAT>(vc[((d + e) << a.c.page_shift) + t0 + t], x);
        o[e] = there ? (T)(x[0] * vs) : (T)0.0f;
      }
      *reinterpret_cast<Tx8*>(static_cast<T*>(a.v) + row * a.vs.row + h * a.vs.head + d) = o;
    }
  }
}

// Pages that `tokens` consecutive tokens can touch, wherever they start
int touched(int tokens, int page, int max_pages) {
  const int64_t n = ((int64_t)tokens + page - 2) / page + 1;
  return (int)(n < max_pages ? n : max_pages);
}

template <template <class, int, int> class Launch, class Args>
eas_status by_type(int dtype, int format, int dim, const Args& a, dim3 grid, hipStream_t s) {
#define EAS_KV8_CASE(DT, T, F, D) \
  if (dtype == DT && format == F && dim == D) return Launch<T, F, D>::go(a, grid, s)
  EAS_KV8_CASE(EAS_BF16, bf16, EAS_KV_INT8, 64);
  EAS_KV8_CASE(EAS_BF16, bf16, EAS_KV_INT8, 128);
  EAS_KV8_CASE(EAS_BF16, bf16, EAS_KV_E4M3, 64);
  EAS_KV8_CASE(EAS_BF16, bf16, EAS_KV_E4M3, 128);
  EAS_KV8_CASE(EAS_FP16, f16, EAS_KV_INT8, 64);
  EAS_KV8_CASE(EAS_FP16, f16, EAS_KV_INT8, 128);
  EAS_KV8_CASE(EAS_FP16, f16, EAS_KV_E4M3, 64);
  EAS_KV8_CASE(EAS_FP16, f16, EAS_KV_E4M3, 128);
#undef EAS_KV8_CASE
  return EAS_ERR_UNSUPPORTED;
}

template <class T, int F, int D>
struct LaunchAppend {
  static eas_status go(const AppendArgs& a, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((kv8_append_kernel<T, F, D>), grid, dim3(NT), 0, s, a);
    return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
  }
};
template <class T, int F, int D>
struct LaunchRows {
  static eas_status go(const RowsArgs& a, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((kv8_rows_kernel<T, F, D>), grid, dim3(NT), 0, s, a);
    return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
  }
};

}  // namespace
}  // namespace eas

using namespace eas;

extern "C" eas_status eas_kv8_append(const eas_kv8_cache* cache, int32_t dtype, const void* k, eas_strides k_strides,
                                     const void* v, eas_strides v_strides, int32_t n_rows, const int32_t* cu_new,
                                     int32_t max_new, const int32_t* held, const int32_t* pages, int32_t max_pages,
                                     int32_t n_seqs, void* stream) {
  eas_status st = check_cache(cache);
  if (st == EAS_OK) st = check_dtype(dtype);
  if (st == EAS_OK) st = check_strides(k_strides);
  if (st == EAS_OK) st = check_strides(v_strides);
  if (st == EAS_OK) st = check_table(cache, pages, max_pages, n_seqs);
  if (st != EAS_OK) return st;
  if (n_rows < 0 || max_new < 0 || !held || (uintptr_t)held % 4 || (uintptr_t)cu_new % 4) return EAS_ERR_INVALID_ARG;
  if (n_rows == 0 || max_new == 0 || n_seqs == 0) return EAS_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return EAS_ERR_INVALID_ARG;
  AppendArgs a = {kv8_args(cache), k, v, k_strides, v_strides, cu_new, held, pages, n_rows, max_new, max_pages,
                  touched(max_new < n_rows ? max_new : n_rows, cache->page_tokens, max_pages)};
  if ((int64_t)a.blocks * n_seqs > 0x7fffffff) return EAS_ERR_UNSUPPORTED;
  return by_type<LaunchAppend>(dtype, cache->format, cache->head_dim, a,
                               dim3((unsigned)(a.blocks * n_seqs), (unsigned)cache->kv_heads), (hipStream_t)stream);
}

extern "C" eas_status eas_kv8_rows(const eas_kv8_cache* cache, int32_t dtype, const int32_t* pages, int32_t max_pages,
                                   int32_t n_seqs, const int32_t* cu_rows, const int32_t* first, int32_t max_rows,
                                   int32_t n_rows, void* k, eas_strides k_strides, void* v, eas_strides v_strides,
                                   void* stream) {
  eas_status st = check_cache(cache);
  if (st == EAS_OK) st = check_dtype(dtype);
  if (st == EAS_OK) st = check_table(cache, pages, max_pages, n_seqs);
  if (st != EAS_OK) return st;
  if (n_rows < 0 || max_rows < 0 || !cu_rows || (uintptr_t)cu_rows % 4 || (uintptr_t)first % 4)
    return EAS_ERR_INVALID_ARG;
  if (k) st = check_out_strides(k_strides, n_rows, cache->kv_heads, cache->head_dim);
  if (st == EAS_OK && v) st = check_out_strides(v_strides, n_rows, cache->kv_heads, cache->head_dim);
  if (st != EAS_OK) return st;
  if (!aligned16(k) || !aligned16(v)) return EAS_ERR_INVALID_ARG;
  if (n_rows == 0 || max_rows == 0 || n_seqs == 0) return EAS_OK;
  if (!k && !v) return EAS_ERR_INVALID_ARG;
  RowsArgs a = {kv8_args(cache), k, v, k_strides, v_strides, cu_rows, first, pages, n_rows, max_rows, max_pages,
                touched(max_rows, cache->page_tokens, 0x7fffffff)};
  if ((int64_t)a.blocks * n_seqs > 0x7fffffff) return EAS_ERR_UNSUPPORTED;
  return by_type<LaunchRows>(dtype, cache->format, cache->head_dim, a,
                             dim3((unsigned)(a.blocks * n_seqs), (unsigned)cache->kv_heads), (hipStream_t)stream);
}
