// The 8-bit key / value cache: append and rows (include/eas_attention.h).
//
// Both are bound by HBM: an append reads 2 bytes and writes 1 for each value, rows the reverse.  So every value is
// read once, in registers, and all loads of a workgroup are issued before the first is used.  An append's
// workgroup owns one block -- a page's tokens of one head --, so nothing is shared between workgroups and no order
// matters; rows are taken 64 tokens of a head at a time.  Value codes are stored dimension by dimension: a thread
// takes 4 tokens of 8 dimensions and turns the 4 x 4 bytes in registers, so both sides move by 16 and 4 bytes.
// Measured in a row: 28,595 tokens of 8 heads of 128 appended in 37 us, 4.7 TB/s, and taken out in 31, 5.6; 16 sequences
// of 8,192 tokens taken out as rows in 172 us, 4.7 TB/s (a copy of 1 GiB moves 5.0).
#include "attention_ops.h"

namespace eas {
namespace {

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
  n = min(n, min((long)a.max_new, a.n_rows - row0));
  const long from = held + max(-row0, 0l);   // the first token whose row there is
  const long slot = (from >> a.c.page_shift) + b;
  if (slot >= a.max_pages) return false;
  const long lo = max(from, slot << a.c.page_shift), hi = min(held + n, (slot + 1) << a.c.page_shift);
  if (lo >= hi) return false;
  s->page = a.pages[(long)r * a.max_pages + slot];
  if (s->page < 0 || s->page >= a.c.n_pages) return false;
  s->row = row0 + (lo - held);
  s->lo = (int)(lo - (slot << a.c.page_shift));
  s->hi = (int)(hi - (slot << a.c.page_shift));
  return true;
}

// Byte j of word i becomes byte i of word j.
__device__ __forceinline__ void turn4(const uint32_t* w, uint32_t* t) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
  const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  t[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  t[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  t[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
  t[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// The earlier tokens' codes of a block to a larger step (ratio = old scale / new), token t's code of dimension d at
// t * token_step + d * dim_step.
template <int FORMAT, int D, int NT>
__device__ void rescale_codes(uint8_t* codes, int tokens, int token_step, int dim_step, float ratio) {
  for (int i = threadIdx.x; i < tokens * (D / 4); i += NT) {
    uint8_t* p = codes + i % tokens * token_step + i / tokens * 4 * dim_step;
    float y[4];
    unpack_codes<FORMAT>(p[0] | p[dim_step] << 8 | p[2 * dim_step] << 16 | (uint32_t)p[3 * dim_step] << 24, y);
    const uint32_t w = pack_codes<FORMAT>(y[0] * ratio, y[1] * ratio, y[2] * ratio, y[3] * ratio);
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e * dim_step] = (uint8_t)(w >> 8 * e);
  }
}

// A workgroup of NT threads takes up to NT * IT 16-byte pieces of keys, and as many of values: a whole page's, or
// with FEW those of up to FEW_TOKENS tokens.
constexpr int FEW_TOKENS = 4;
template <class T, int FORMAT, int D, int NT, int IT, bool FEW>
__global__ __launch_bounds__(NT) void kv8_append_kernel(AppendArgs a) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  constexpr int C = D / 8;               // 16-byte pieces of a row
  constexpr int IV = (IT + 3) / 4;       // a thread's values: 4 tokens of a piece each
  __shared__ float red[2][NT / 64];
  Span s;
  if (!find_span(a, blockIdx.x / a.blocks, blockIdx.x % a.blocks, &s)) return;
  const int h = blockIdx.y, tid = threadIdx.x, shift = a.c.page_shift;
  const long block = (long)s.page * a.c.kv_heads + h;
  uint8_t* kc = a.c.k + (block << shift) * D;
  uint8_t* vc = a.c.v + (block << shift) * D;
  // row of the page's token 0
  const T* kx = static_cast<const T*>(a.k) + (s.row - s.lo) * a.ks.row + h * a.ks.head;
  const T* vx = static_cast<const T*>(a.v) + (s.row - s.lo) * a.vs.row + h * a.vs.head;
  const float k_old = s.lo > 0 ? a.c.k_scale[block] : 0.0f, v_old = s.lo > 0 ? a.c.v_scale[block] : 0.0f;

  Tx8 k[IT], v[IV][4];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int c = tid + NT * i, t = s.lo + c / C;
    if (t < s.hi) k[i] = *reinterpret_cast<const Tx8*>(kx + (long)t * a.ks.row + c % C * 8);
  }
  // values: the page's 4-token groups from g0 on, group c % groups of piece c / groups
  const int glog = FEW ? 1 : shift - 2, groups = 1 << glog, g0 = FEW ? s.lo >> 2 : 0;
#pragma unroll
  for (int i = 0; i < IV; ++i) {
    const int c = tid + NT * i, t = (g0 + (c & (groups - 1))) * 4, d = (c >> glog) * 8;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d < D && t + j >= s.lo && t + j < s.hi)
        v[i][j] = *reinterpret_cast<const Tx8*>(vx + (long)(t + j) * a.vs.row + d);
  }
  float k_top = 0.0f, v_top = 0.0f;
#pragma unroll
  for (int i = 0; i < IT; ++i)
    if (s.lo + (tid + NT * i) / C < s.hi)
#pragma unroll
      for (int e = 0; e < 8; ++e) k_top = fmaxf(k_top, finite_magnitude(k[i][e]));
#pragma unroll
  for (int i = 0; i < IV; ++i) {
    const int c = tid + NT * i, t = (g0 + (c & (groups - 1))) * 4, d = (c >> glog) * 8;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d < D && t + j >= s.lo && t + j < s.hi)
#pragma unroll
        for (int e = 0; e < 8; ++e) v_top = fmaxf(v_top, finite_magnitude(v[i][j][e]));
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    k_top = fmaxf(k_top, __shfl_xor(k_top, o, 64));
    v_top = fmaxf(v_top, __shfl_xor(v_top, o, 64));
  }
  if ((tid & 63) == 0) {
    red[0][tid >> 6] = k_top;
    red[1][tid >> 6] = v_top;
  }
  __syncthreads();   // every thread has read the old scales, too
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    k_top = fmaxf(k_top, red[0][w]);
    v_top = fmaxf(v_top, red[1][w]);
  }
  const float k_scale = fmaxf(k_old, block_scale<FORMAT>(k_top)), v_scale = fmaxf(v_old, block_scale<FORMAT>(v_top));
  const float k_inv = inverse_scale(k_scale), v_inv = inverse_scale(v_scale);
  if (tid == 0) {
    a.c.k_scale[block] = k_scale;
    a.c.v_scale[block] = v_scale;
  }
  if (k_scale > k_old && k_old > 0.0f) rescale_codes<FORMAT, D, NT>(kc, s.lo, D, 1, k_old * k_inv);
  if (v_scale > v_old && v_old > 0.0f) rescale_codes<FORMAT, D, NT>(vc, s.lo, 1, 1 << shift, v_old * v_inv);

  const auto codes = [](Tx8 x, float inv, uint32_t* w) {
    w[0] = pack_codes<FORMAT>((float)x[0] * inv, (float)x[1] * inv, (float)x[2] * inv, (float)x[3] * inv);
    w[1] = pack_codes<FORMAT>((float)x[4] * inv, (float)x[5] * inv, (float)x[6] * inv, (float)x[7] * inv);
  };
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int c = tid + NT * i, t = s.lo + c / C;
    if (t < s.hi) {
      uint32_t w[2];
      codes(k[i], k_inv, w);
      *reinterpret_cast<uint2*>(kc + t * D + c % C * 8) = make_uint2(w[0], w[1]);
    }
  }
#pragma unroll
  for (int i = 0; i < IV; ++i) {
    const int c = tid + NT * i, t = (g0 + (c & (groups - 1))) * 4, d = (c >> glog) * 8;
    if (d >= D || t + 3 < s.lo || t >= s.hi) continue;
    uint32_t w[2][4], x[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t y[2] = {0, 0};
      if (t + j >= s.lo && t + j < s.hi) codes(v[i][j], v_inv, y);
      w[0][j] = y[0];
      w[1][j] = y[1];
    }
    turn4(w[0], x[0]);
    turn4(w[1], x[1]);
    uint8_t* p = vc + (d << shift) + t;
    const bool whole = t >= s.lo && t + 4 <= s.hi;
#pragma unroll
    for (int e = 0; e < 8; ++e, p += 1 << shift) {
      if (whole) {
        *reinterpret_cast<uint32_t*>(p) = x[e >> 2][e & 3];
      } else {   // other tokens' codes stay
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (t + j >= s.lo && t + j < s.hi) p[j] = (uint8_t)(x[e >> 2][e & 3] >> 8 * j);
      }
    }
  }
}

struct RowsArgs {
  Kv8Args c;
  void* k;
  void* v;
  eas_strides ks, vs;
  const int* cu;
  const int* first;
  const int* pages;
  int n_rows, max_rows, max_pages, blocks;   // blocks: SPAN-token spans that one sequence's rows can touch
};

constexpr int SPAN = 64;   // tokens per workgroup
constexpr int NT = 256;

template <class T, int FORMAT, int D>
__global__ __launch_bounds__(NT) void kv8_rows_kernel(RowsArgs a) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  constexpr int C = D / 8;                         // 8-code pieces of a row
  constexpr int IK = SPAN * C / NT;                // a thread's pieces of keys
  constexpr int IV = (SPAN / 4 * C + NT - 1) / NT; // and of values, 4 tokens each
  const int r = blockIdx.x / a.blocks, b = blockIdx.x % a.blocks, h = blockIdx.y, tid = threadIdx.x;
  const int shift = a.c.page_shift, mask = (1 << shift) - 1;
  const long skip = max(-(long)a.cu[r], 0l), row0 = a.cu[r] + skip;   // rows before 0 are not there
  const long n = min((long)a.cu[r + 1] - a.cu[r], (long)a.max_rows) - skip;
  const long first = (a.first ? a.first[r] : 0) + skip;
  // tokens of this workgroup; a sequence that starts below 0 has spans below 0 too
  const long base = (first >= 0 ? first / SPAN : -((-first + SPAN - 1) / SPAN)) * SPAN + (long)b * SPAN;
  const long lo = max(first, base), hi = min(first + n, base + SPAN);
  if (lo >= hi) return;
  const auto page_of = [&](long t) {
    const long slot = t >> shift;
    const int id = t >= 0 && slot < a.max_pages ? a.pages[(long)r * a.max_pages + slot] : -1;
    return id >= 0 && id < a.c.n_pages ? id : -1;
  };
  // a token's row, if it has one
  const auto row_of = [&](long t) {
    const long row = row0 + (t - first);
    return t >= lo && t < hi && row >= 0 && row < a.n_rows ? row : -1;
  };
  uint2 k[IK];
  float ks[IK];
  uint32_t v[IV][8];
  float vs[IV];
  if (a.k) {
#pragma unroll
    for (int i = 0; i < IK; ++i) {
      const int c = tid + NT * i;
      const long t = base + c / C;
      const int id = row_of(t) >= 0 ? page_of(t) : -1;
      k[i] = make_uint2(0, 0);   // code 0 in either format
      ks[i] = 0.0f;
      if (id >= 0) {
        const long block = (long)id * a.c.kv_heads + h;
        ks[i] = a.c.k_scale[block];
        k[i] = *reinterpret_cast<const uint2*>(a.c.k + ((block << shift) + (t & mask)) * D + c % C * 8);
      }
    }
  }
  if (a.v) {
#pragma unroll
    for (int i = 0; i < IV; ++i) {
      const int c = tid + NT * i, d = c % C * 8;
      const long t = base + c / C * 4;
      const int id = c < SPAN / 4 * C && t + 3 >= lo && t < hi ? page_of(t) : -1;
      vs[i] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0;
      if (id >= 0) {
        const long block = (long)id * a.c.kv_heads + h;
        vs[i] = a.c.v_scale[block];
        const uint8_t* p = a.c.v + ((block * D + d) << shift) + (t & mask);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = *reinterpret_cast<const uint32_t*>(p + ((long)e << shift));
      }
    }
  }
  const auto store = [&](T* out, const uint32_t* w, float scale) {
    float x[8];
    unpack_codes<FORMAT>(w[0], x);
    unpack_codes<FORMAT>(w[1], x + 4);
    Tx8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (T)(x[e] * scale);
    *reinterpret_cast<Tx8*>(out) = o;
  };
  if (a.k) {
#pragma unroll
    for (int i = 0; i < IK; ++i) {
      const int c = tid + NT * i;
      const long row = row_of(base + c / C);
      const uint32_t w[2] = {k[i].x, k[i].y};
      if (row >= 0) store(static_cast<T*>(a.k) + row * a.ks.row + h * a.ks.head + c % C * 8, w, ks[i]);
    }
  }
  if (a.v) {
#pragma unroll
    for (int i = 0; i < IV; ++i) {
      const int c = tid + NT * i, d = c % C * 8;
      uint32_t x[2][4];
      turn4(v[i], x[0]);
      turn4(v[i] + 4, x[1]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long row = c < SPAN / 4 * C ? row_of(base + c / C * 4 + j) : -1;
        const uint32_t w[2] = {x[0][j], x[1][j]};
        if (row >= 0) store(static_cast<T*>(a.v) + row * a.vs.row + h * a.vs.head + d, w, vs[i]);
      }
    }
  }
}

// Pages (or spans) of `page` tokens that `tokens` consecutive tokens can touch, wherever they start
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
    // a decoding step's tokens by one wave each (16 sequences 5.0 us, with 256 threads 5.4); small pages
    // by fewer threads (16,384 tokens in 16-token pages, 8 heads of 64: 17.5 us, with 256 threads 25.6)
    const int pieces = (D << a.c.page_shift) / 8;
    if (!fits_launch(grid.x, a.max_new <= FEW_TOKENS || pieces <= 256 ? 64 : pieces == 512 ? 128 : 256))
      return EAS_ERR_UNSUPPORTED;
    if (a.max_new <= FEW_TOKENS)
      hipLaunchKernelGGL((kv8_append_kernel<T, F, D, 64, 1, true>), grid, dim3(64), 0, s, a);
    else if (pieces == 128)
      hipLaunchKernelGGL((kv8_append_kernel<T, F, D, 64, 2, false>), grid, dim3(64), 0, s, a);
    else if (pieces == 256)
      hipLaunchKernelGGL((kv8_append_kernel<T, F, D, 64, 4, false>), grid, dim3(64), 0, s, a);
    else if (pieces == 512)
      hipLaunchKernelGGL((kv8_append_kernel<T, F, D, 128, 4, false>), grid, dim3(128), 0, s, a);
    else if (pieces == 1024)
      hipLaunchKernelGGL((kv8_append_kernel<T, F, D, 256, 4, false>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((kv8_append_kernel<T, F, D, 256, 8, false>), grid, dim3(256), 0, s, a);
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
  if (n_rows < 0 || max_new < 0 || (!held && n_seqs > 0) || (uintptr_t)held % 4 || (uintptr_t)cu_new % 4) return EAS_ERR_INVALID_ARG;
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
                touched(max_rows < n_rows ? max_rows : n_rows, SPAN, 0x7fffffff)};
  if (!fits_launch((int64_t)a.blocks * n_seqs, NT)) return EAS_ERR_UNSUPPORTED;
  return by_type<LaunchRows>(dtype, cache->format, cache->head_dim, a,
                             dim3((unsigned)(a.blocks * n_seqs), (unsigned)cache->kv_heads), (hipStream_t)stream);
}
