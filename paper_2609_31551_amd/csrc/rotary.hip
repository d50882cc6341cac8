// Rotary positions with several axes, over rows and on the way into the paged 16-bit cache (include/eas_paged.h).
//
// Pair (x, y) of a head turns by a = p f: x' = x cos a - y sin a, y' = x sin a + y cos a.  f is held as whole 2^-64ths of
// a turn, so p f modulo a turn is the low 64 bits of an integer product: exact at any position, where a 32-bit product
// of a position of 10^5 would be off by 10^-2 radians.  Its top two bits, rounded, are a quarter turn (a swap and two
// signs); what is left, within an eighth of a turn, goes through the Taylor series of sine and cosine, whose first
// terms left out are below 2^-29 there.
//
// Bound by HBM: 2 bytes read and 2 written for each value.  A workgroup takes some rows and all their heads: sines
// and cosines are taken once for a row and kept in LDS, a thread then moves 16 values -- 8 pairs, in one of the layouts,
// or 16 that pass -- by 16-byte loads and stores.
#include <cmath>

#include "paged_ops.h"

namespace eas {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_BLOCK_ROWS = 8;

struct RotaryArgs {
  eas_rotary rot;         // pairs 0: nothing turns
  const void* q;
  const void* k;
  const void* v;
  void* q_out;            // rows
  void* k_out;            // rows, or the cache's pages
  void* v_out;
  eas_strides qs, ks, vs, qos, kos;
  const int* positions;   // null: a token's place
  long axis_stride;
  int heads, kv_heads, dim, n_rows, inverse;
  int rows_each;          // rows of a workgroup
  // append only
  int page_shift, n_pages, max_pages, n_seqs, max_new;
  const int* cu_new;
  const int* held;
  const int* pages;
};

// Cosine and sine of `phase` / 2^64 turns
__device__ __forceinline__ float2 turn(uint64_t phase) {
  const uint32_t u = (uint32_t)(phase >> 32);
  const uint32_t quarter = (u + (1u << 29)) >> 30;
  const float x = (float)(int)(u - (quarter << 30)) * 1.46291807927e-9f;   // 2 pi / 2^32; |x| <= pi / 4
  const float z = x * x;
  const float s = fmaf(fmaf(fmaf(fmaf(1.0f / 362880, z, -1.0f / 5040), z, 1.0f / 120), z, -1.0f / 6) * z, x, x);
  const float c = fmaf(fmaf(fmaf(fmaf(fmaf(-1.0f / 3628800, z, 1.0f / 40320), z, -1.0f / 720), z, 1.0f / 24), z, -0.5f), z,
                       1.0f);
  const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -cs : cs, quarter & 2 ? -sn : sn);
}

// Where a row goes
struct RowInfo {
  long page;    // of the cache's values, the first of head 0's place for the token; -1: none
  long place;   // the token's in its sequence
  bool real;    // the row is a sequence's
};

// The row's sequence: the last of those that begin at or before it.  All lanes of a wave ask for the same row, and look
// at 64 of the sequences that are left at a time, evenly spread (4,096 of one token, 28 heads and 4: 17 us, at one 64
// after the other 48; up to 64 are one look).
__device__ __forceinline__ RowInfo find_row(const RotaryArgs& a, int row) {
  RowInfo info = {-1, 0, false};
  int r, i;
  if (a.cu_new) {
    const int lane = threadIdx.x & 63;
    int before = 0, left = a.n_seqs;   // sequences known to begin at or before the row; those not known
    while (left > 0) {
      const int step = (unsigned)(left + 63) / 64, at = lane * step;
      const int there = __popcll(__ballot(at < left && a.cu_new[before + min(at, left)] <= row));
      const int known = there ? (there - 1) * step + 1 : 0;
      left = there ? min(step - 1, left - known) : 0;
      before += known;
    }
    r = before - 1;
    if (r < 0 || row >= a.cu_new[r + 1]) return info;
    i = (int)((unsigned)row - (unsigned)a.cu_new[r]);
  } else {
    r = (unsigned)row / (unsigned)a.max_new;
    i = row - r * a.max_new;
    if (r >= a.n_seqs) return info;
  }
  const int held = a.held[r];
  if ((unsigned)i >= (unsigned)a.max_new || held < 0) return info;
  const long place = (long)held + i;
  info.real = true;
  info.place = place;
  if (place >= (long)a.max_pages << a.page_shift) return info;
  const int page = a.pages[(long)r * a.max_pages + (place >> a.page_shift)];
  if (page < 0 || page >= a.n_pages) return info;
  info.page = (((long)page * a.kv_heads << a.page_shift) + (place & ((1 << a.page_shift) - 1))) * a.dim;
  return info;
}

// DIM: of a head, or 0 where it is none that has a kernel of its own
template <class T, int DIM, bool APPEND>
__global__ __launch_bounds__(THREADS) void rotary_kernel(RotaryArgs a) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  __shared__ float2 turns[MAX_BLOCK_ROWS][EAS_MAX_ROTARY_PAIRS];
  __shared__ RowInfo info[MAX_BLOCK_ROWS];
  const int row0 = blockIdx.x * a.rows_each, rows = min(a.rows_each, a.n_rows - row0);
  const int tid = threadIdx.x;
  if constexpr (APPEND) {
    for (int j = tid >> 6; j < rows; j += THREADS / 64) {
      const RowInfo x = find_row(a, row0 + j);
      if ((tid & 63) == 0) info[j] = x;
    }
    __syncthreads();
  }
  const int pairs = a.rot.pairs;
  for (int i = tid; i < rows * pairs; i += THREADS) {
    const int j = (unsigned)i / (unsigned)pairs, p = i - j * pairs;
    const int64_t at = APPEND && !a.positions ? info[j].place : a.positions[a.rot.axis[p] * a.axis_stride + row0 + j];
    float2 cs = turn((uint64_t)at * a.rot.step[p]);
    if (a.inverse) cs.y = -cs.y;
    turns[j][p] = cs;
  }
  __syncthreads();

  const unsigned chunks = DIM ? DIM / 16 : a.dim / 16;
  const unsigned each = a.heads + (APPEND ? 2 : 1) * a.kv_heads;   // heads of a row
  const int turning = pairs / 8;   // of a head's chunks
  for (unsigned i = tid; i < rows * each * chunks; i += THREADS) {
    const int c = i % chunks;
    const unsigned item = i / chunks;
    const int j = item / each;
    int h = item - j * each;
    const long row = row0 + j;
    if (APPEND && !info[j].real) continue;
    const T* src;
    T* dst;
    bool turned = c < turning;
    if (h < a.heads) {
      src = static_cast<const T*>(a.q) + row * a.qs.row + h * a.qs.head;
      dst = static_cast<T*>(a.q_out) + row * a.qos.row + h * a.qos.head;
    } else {
      h -= a.heads;
      const bool value = APPEND && h >= a.kv_heads;
      if (value) {
        h -= a.kv_heads;
        turned = false;
        src = static_cast<const T*>(a.v) + row * a.vs.row + h * a.vs.head;
      } else {
        src = static_cast<const T*>(a.k) + row * a.ks.row + h * a.ks.head;
      }
      if constexpr (APPEND) {
        const long page = info[j].page;
        if (page < 0) continue;
        dst = static_cast<T*>(value ? a.v_out : a.k_out) + page + ((long)h * a.dim << a.page_shift);
      } else {
        dst = static_cast<T*>(a.k_out) + row * a.kos.row + h * a.kos.head;
      }
    }
    const bool split = turned && !a.rot.adjacent;
    const int x0 = split ? 8 * c : 16 * c, y0 = split ? pairs + 8 * c : 16 * c + 8;
    Tx8 x = *reinterpret_cast<const Tx8*>(src + x0), y = *reinterpret_cast<const Tx8*>(src + y0);
    if (turned) {
      float f[16];   // the pairs, (x, y) each
      if (split) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[2 * e] = (float)x[e], f[2 * e + 1] = (float)y[e];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)x[e], f[8 + e] = (float)y[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = turns[j][8 * c + e];
        const float px = f[2 * e], py = f[2 * e + 1];
        f[2 * e] = fmaf(px, cs.x, -(py * cs.y));
        f[2 * e + 1] = fmaf(px, cs.y, py * cs.x);
        // rounded to fp32 here and to the type below, in every kernel: an FMA with an fp16 result rounds once, and the
        // compiler takes it for some pairs of some kernels
        asm("" : "+v"(f[2 * e]), "+v"(f[2 * e + 1]));
      }
      if (split) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (T)f[2 * e], y[e] = (T)f[2 * e + 1];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (T)f[e], y[e] = (T)f[8 + e];
      }
    }
    *reinterpret_cast<Tx8*>(dst + x0) = x;
    *reinterpret_cast<Tx8*>(dst + y0) = y;
  }
}

template <class T, bool APPEND>
eas_status launch(RotaryArgs& a, hipStream_t s) {
  // Rows of a workgroup: as many as give each thread one piece, of few rows one, so that each CU has four workgroups
  // (16,484 rows of 40 heads of 128: one row 62 us, with 8 pieces a thread 68; 7,816 rows of 20 heads of 64: three rows 9.9,
  // one 12.0)
  const int pieces = (a.heads + (APPEND ? 2 : 1) * a.kv_heads) * (a.dim / 16), want = THREADS / pieces;
  const int most = a.n_rows / (4 * device_cus()), each = want < most ? want : most;
  a.rows_each = each < 1 ? 1 : each < MAX_BLOCK_ROWS ? each : MAX_BLOCK_ROWS;
  const int64_t blocks = ((int64_t)a.n_rows + a.rows_each - 1) / a.rows_each;
  if (!fits_launch(blocks, THREADS)) return EAS_ERR_UNSUPPORTED;
  if (a.dim == 128)
    hipLaunchKernelGGL((rotary_kernel<T, 128, APPEND>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
  else if (a.dim == 64)
    hipLaunchKernelGGL((rotary_kernel<T, 64, APPEND>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
  else
    hipLaunchKernelGGL((rotary_kernel<T, 0, APPEND>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
  return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
}

eas_status check_rotary(const eas_rotary* r, int32_t head_dim) {
  if (!r || (r->adjacent != 0 && r->adjacent != 1) || r->reserved != 0) return EAS_ERR_INVALID_ARG;
  if (r->pairs < 8 || r->pairs > EAS_MAX_ROTARY_PAIRS || r->pairs % 8 || r->axes < 1 || r->axes > EAS_MAX_ROTARY_AXES)
    return EAS_ERR_INVALID_ARG;
  for (int i = 0; i < r->pairs; ++i)
    if (r->axis[i] >= r->axes) return EAS_ERR_INVALID_ARG;
  return 2 * r->pairs <= head_dim ? EAS_OK : EAS_ERR_INVALID_ARG;
}

// The turns of f radians, |f| < 2^60, modulo whole ones and to the nearest 2^-64: f is m 2^e with a whole m below 2^53, and
// m / (2 pi) is a whole number of 2^-128ths, m times those of 1 / (2 pi).  What these leave out is below 2^-68 of a turn.
uint64_t step_of(double f) {
  typedef unsigned __int128 u128;
  int e;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(f), &e), 53);
  const u128 low = (u128)m * 0x7f09d5f47d4d3770u, high = (u128)m * 0x28be60db9391054au + (low >> 64);
  const uint64_t rest = (uint64_t)low;
  const int n = 64 - (e - 53);   // bits below 2^-64 of a turn, 57 at least
  uint64_t step = 0;
  if (n < 64)
    step = ((uint64_t)(high << (64 - n)) | rest >> n) + (rest >> (n - 1) & 1);
  else if (n < 192)
    step = (uint64_t)(high >> (n - 64)) + (n == 64 ? rest >> 63 : (uint64_t)(high >> (n - 65)) & 1);
  return f < 0 ? 0 - step : step;
}

// What is rotated from x to out: rows of `heads` heads; out may be x
eas_status check_rows(const void* x, const eas_strides& xs, const void* out, const eas_strides& os, int64_t rows,
                      int32_t heads, int32_t dim) {
  if (!x || !out || !aligned16(x) || !aligned16(out)) return EAS_ERR_INVALID_ARG;
  return x != out || ((xs.row == os.row || rows <= 1) && (xs.head == os.head || heads <= 1)) ? EAS_OK
                                                                                             : EAS_ERR_INVALID_ARG;
}

}  // namespace
}  // namespace eas

using namespace eas;

extern "C" eas_status eas_rotary_make(const double* freqs, const int32_t* axis, int32_t pairs, int32_t axes,
                                      int32_t adjacent, eas_rotary* rotary) {
  if (!freqs || !rotary || (adjacent != 0 && adjacent != 1) || pairs <= 0 || axes <= 0) return EAS_ERR_INVALID_ARG;
  if (pairs > EAS_MAX_ROTARY_PAIRS || pairs % 8 || axes > EAS_MAX_ROTARY_AXES) return EAS_ERR_UNSUPPORTED;
  eas_rotary r = {};
  r.pairs = pairs, r.axes = axes, r.adjacent = adjacent;
  for (int i = 0; i < pairs; ++i) {
    const int a = axis ? axis[i] : 0;
    if (a < 0 || a >= axes || !std::isfinite(freqs[i])) return EAS_ERR_INVALID_ARG;
    if (fabs(freqs[i]) >= 0x1p60) return EAS_ERR_UNSUPPORTED;
    r.step[i] = step_of(freqs[i]);
    r.axis[i] = (uint8_t)a;
  }
  *rotary = r;
  return EAS_OK;
}

extern "C" eas_status eas_rotary_rows(const eas_rotary* rotary, int32_t dtype, int32_t head_dim, int32_t inverse,
                                      const int32_t* positions, int64_t axis_stride, int32_t n_rows, const void* q,
                                      eas_strides q_strides, int32_t heads, void* q_out, eas_strides q_out_strides,
                                      const void* k, eas_strides k_strides, int32_t kv_heads, void* k_out,
                                      eas_strides k_out_strides, void* stream) {
  eas_status st = check_dtype(dtype);
  if (st != EAS_OK) return st;
  if (head_dim <= 0 || (inverse != 0 && inverse != 1) || n_rows < 0 || axis_stride < 0 || heads <= 0 || heads > 1024 ||
      (k && (kv_heads <= 0 || kv_heads > 1024)))
    return EAS_ERR_INVALID_ARG;
  if (head_dim % 16 || head_dim > 256) return EAS_ERR_UNSUPPORTED;
  st = check_rotary(rotary, head_dim);
  if (st == EAS_OK) st = check_strides(q_strides);
  if (st == EAS_OK) st = check_out_strides(q_out_strides, n_rows, heads, head_dim);
  if (st == EAS_OK && k) st = check_strides(k_strides);
  if (st == EAS_OK && k) st = check_out_strides(k_out_strides, n_rows, kv_heads, head_dim);
  if (st != EAS_OK || n_rows == 0) return st;
  st = check_rows(q, q_strides, q_out, q_out_strides, n_rows, heads, head_dim);
  if (st == EAS_OK && k) st = check_rows(k, k_strides, k_out, k_out_strides, n_rows, kv_heads, head_dim);
  if (st != EAS_OK) return st;
  if (!positions || (uintptr_t)positions % 4) return EAS_ERR_INVALID_ARG;
  RotaryArgs a = {};
  a.rot = *rotary;
  a.q = q, a.k = k, a.q_out = q_out, a.k_out = k_out;
  a.qs = q_strides, a.ks = k_strides, a.qos = q_out_strides, a.kos = k_out_strides;
  a.positions = positions, a.axis_stride = axis_stride;
  a.heads = heads, a.kv_heads = k ? kv_heads : 0, a.dim = head_dim, a.n_rows = n_rows, a.inverse = inverse;
  return dtype == EAS_BF16 ? launch<bf16, false>(a, (hipStream_t)stream) : launch<f16, false>(a, (hipStream_t)stream);
}

extern "C" eas_status eas_kv16_append(const eas_kv16_cache* cache, const eas_rotary* rotary, const int32_t* positions,
                                      int64_t axis_stride, const void* q, eas_strides q_strides, int32_t heads,
                                      void* q_out, eas_strides q_out_strides, const void* k, eas_strides k_strides,
                                      const void* v, eas_strides v_strides, int32_t n_rows, const int32_t* cu_new,
                                      int32_t max_new, const int32_t* held, const int32_t* pages, int32_t max_pages,
                                      int32_t n_seqs, void* stream) {
  eas_status st = check_cache16(cache);
  if (st == EAS_OK) st = check_table16(cache, pages, max_pages, n_seqs);
  if (st == EAS_OK && rotary) st = check_rotary(rotary, cache->head_dim);
  if (st == EAS_OK) st = check_strides(k_strides);
  if (st == EAS_OK) st = check_strides(v_strides);
  if (st != EAS_OK) return st;
  if (n_rows < 0 || max_new < 0 || axis_stride < 0 || (!held && n_seqs > 0) || (uintptr_t)held % 4 ||
      (uintptr_t)cu_new % 4 || (uintptr_t)positions % 4)
    return EAS_ERR_INVALID_ARG;
  if (q) {
    if (!rotary || heads <= 0 || heads > 1024) return EAS_ERR_INVALID_ARG;
    st = check_strides(q_strides);
    if (st == EAS_OK) st = check_out_strides(q_out_strides, n_rows, heads, cache->head_dim);
    if (st != EAS_OK) return st;
  }
  if (n_rows == 0 || max_new == 0 || n_seqs == 0) return EAS_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return EAS_ERR_INVALID_ARG;
  if (q && (st = check_rows(q, q_strides, q_out, q_out_strides, n_rows, heads, cache->head_dim)) != EAS_OK) return st;
  RotaryArgs a = {};
  if (rotary) a.rot = *rotary;
  a.q = q, a.k = k, a.v = v, a.q_out = q_out, a.k_out = cache->k, a.v_out = cache->v;
  a.qs = q_strides, a.ks = k_strides, a.vs = v_strides, a.qos = q_out_strides;
  a.positions = positions, a.axis_stride = axis_stride;
  a.heads = q ? heads : 0, a.kv_heads = cache->kv_heads, a.dim = cache->head_dim, a.n_rows = n_rows;
  a.page_shift = __builtin_ctz((unsigned)cache->page_tokens), a.n_pages = cache->n_pages;
  a.max_pages = max_pages, a.n_seqs = n_seqs, a.max_new = max_new;
  a.cu_new = cu_new, a.held = held, a.pages = pages;
  return cache->dtype == EAS_BF16 ? launch<bf16, true>(a, (hipStream_t)stream)
                                  : launch<f16, true>(a, (hipStream_t)stream);
}
