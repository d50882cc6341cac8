// Attention of new tokens over the paged 16-bit cache (include/eas_paged.h).
//
// A row is one query of one head; the rows of a sequence that share a key / value head (its queries times the
// group's heads) are taken 16 at a time, as the columns of MFMA products whose rows are the cache's tokens and
// dimensions:
//   S^T = K Q^T,  O^T += V^T P^T   (v_mfma_f32_16x16x32),
// with one pass over the tokens, the running maximum and sum of the softmax in fp32, and P rounded to the element type.
// The four waves of a workgroup take tiles of 32 tokens in turn and are joined at the end; a sequence's tokens are
// split into runs by a rule on its own sizes, and the runs joined in order by a second kernel.
#include <type_traits>

#include "paged_ops.h"

namespace eas {
namespace {

constexpr int TILE = 32;         // tokens per wave and step
constexpr int NW = 4;            // waves per workgroup
constexpr int ROWS = 16;         // of a workgroup
static_assert(FEW_STEP == NW * TILE);

template <class T>
struct Mfma16;
template <>
struct Mfma16<bf16> {
  typedef bf16x8 x8;
  __device__ static f32x4 go(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma16<f16> {
  typedef f16x8 x8;
  __device__ static f32x4 go(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// maximum and sum over the four lanes that hold one query (lane, lane ^ 16, ^ 32, ^ 48)
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float column_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

template <class T, int D>
__global__ __launch_bounds__(64 * NW) void kv16_tokens_kernel(Kv16AttnArgs a) {
  typedef typename Mfma16<T>::x8 x8;
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  constexpr int KS = D / 32;   // 32-dimension steps of q . k
  constexpr int DB = D / 16;   // 16-dimension blocks of the output
  constexpr float TOP = std::is_same_v<T, f16> ? 15.0f : 0.0f;   // log2 of the largest weight
  __shared__ float o_part[NW][ROWS][D];
  __shared__ float m_part[NW][ROWS], l_part[NW][ROWS];

  unsigned b = blockIdx.x;
  const int rt = b % (unsigned)a.row_tiles;
  b /= (unsigned)a.row_tiles;
  const int run = b % (unsigned)a.most_runs;
  b /= (unsigned)a.most_runs;
  const int kvh = b % (unsigned)a.c.kv_heads, r = b / (unsigned)a.c.kv_heads;
  const Seq s = find_seq(a, r);
  const int group = a.heads / a.c.kv_heads;
  if (!takes_few(a, s) || rt * ROWS >= s.nq * group) return;
  const int runs = few_runs(s.len, s.nq, a.heads, a.c.kv_heads);
  if (run >= runs) return;
  const int each = few_run_tokens(s.len, runs);
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // this lane's query, and how many tokens it sees
  const int rho = rt * ROWS + c;
  const bool real = rho < s.nq * group;
  const int qi = real ? (unsigned)rho / (unsigned)group : 0, head = kvh * group + (real ? rho - qi * group : 0);
  const int sees = real ? seen_by(a, s, qi) : 0;
  const T* q = static_cast<const T*>(a.q) + (s.row0 + qi) * a.qs.row + head * a.qs.head;
  x8 qf[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = *reinterpret_cast<const x8*>(q + 32 * i + 8 * g);
  // the last query sees most
  const int most = seen_by(a, s, min(rt * ROWS + ROWS - 1, s.nq * group - 1) / group);
  const long t_begin = (long)run * each;
  const int t_end = (int)min((long)most, t_begin + each);
  const int* table = a.pages + (long)r * a.max_pages;
  // offset of a token's head in the cache, of tokens behind the last that of the last; *there: its page is held
  const auto place = [&](int t, bool* there) {
    t = min(t, t_end - 1);
    const int page = table[t >> a.c.page_shift];
    *there = held_page(a, page);
    return token_offset(a, page, kvh, t, D);
  };
  const T* keys = static_cast<const T*>(a.c.k);
  const T* values = static_cast<const T*>(a.c.v);

  f32x4 o[DB];
  float m, l;
  // The wave's tiles.  Row 4 g + e of score block i is token 8 g + 4 i + e, so that a lane ends with the scores of 8
  // consecutive tokens, 8 g .. + 8, of one query: as the products with the values want them.
  const auto walk = [&](auto careful) {
    m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int t0 = (int)t_begin + wave * TILE; t0 < t_end; t0 += NW * TILE) {
      f32x4 sc[2];
      bool there;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const T* kp = keys + place(t0 + 8 * (c >> 2) + 4 * i + (c & 3), &there) + 8 * g;
        sc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < KS; ++k) sc[i] = Mfma16<T>::go(*reinterpret_cast<const x8*>(kp + 32 * k), qf[k], sc[i]);
      }
      const T* vp = values + place(t0 + 8 * g, &there);   // 8 tokens lie in one page
      const int left = there ? sees - (t0 + 8 * g) : 0;   // of the lane's 8 tokens, those that its query sees
      float x[8], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = i < left ? sc[i >> 2][i & 3] * a.scale_log2 : -INFINITY;
        top = fmaxf(top, x[i]);
      }
      top = column_max(top);
      const float up = fmaxf(m, top), base = up == -INFINITY ? 0.0f : up;
      const float alpha = __builtin_amdgcn_exp2f(m - base);
      m = up;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[i] *= alpha;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(x[i] - base + TOP);
        l += x[i];
      }
      if constexpr (!decltype(careful)::value) {
        x8 p;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = (T)x[i];
        const int last = min(t0 + 8 * g + 7, t_end - 1) - min(t0 + 8 * g, t_end - 1);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          x8 v;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = vp[min(i, last) * D + 16 * d + c];
          o[d] = Mfma16<T>::go(v, p, o[d]);
        }
      } else {
        // token by token, by the queries that see it
        for (int from = 0; from < 4; ++from)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int t = t0 + 8 * from + i;
            const float p = __shfl(x[i], 16 * from + c, 64);
            const long at = place(t, &there);
            if (t < sees && there)
#pragma unroll
              for (int d = 0; d < DB; ++d) {
                const Tx4 v = *reinterpret_cast<const Tx4*>(values + at + 16 * d + 4 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][e] = fmaf(p, (float)v[e], o[d][e]);
              }
          }
      }
    }
  };
  walk(std::false_type{});
  // A hidden value went into the products with weight 0: where it is infinite or NaN it shows, and the tiles are walked
  // again without.
  uint32_t size = 0;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) size = max(size, __float_as_uint(o[i][e]) & 0x7fffffffu);
  if (__any(size >= 0x7f800000u)) walk(std::true_type{});

  // the four waves' sums: lane (c, g) holds dimensions 16 i + 4 g .. + 4 of query c
  l = column_sum(l);
  if (g == 0) m_part[wave][c] = m, l_part[wave][c] = l;
#pragma unroll
  for (int i = 0; i < DB; ++i) *reinterpret_cast<f32x4*>(&o_part[wave][c][16 * i + 4 * g]) = o[i];
  __syncthreads();
  for (int i = threadIdx.x; i < ROWS * (D / 4); i += 64 * NW) {
    const int row = i / (D / 4), d = i % (D / 4) * 4, rr = rt * ROWS + row;
    if (rr >= s.nq * group) break;
    float M = m_part[0][row];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, m_part[w][row]);
    const float M0 = M == -INFINITY ? 0.0f : M;
    float L = 0.0f;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float beta = __builtin_amdgcn_exp2f(m_part[w][row] - M0);
      L += l_part[w][row] * beta;
      sum += *reinterpret_cast<const f32x4*>(&o_part[w][row][d]) * beta;
    }
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const float lse2 = L == 0.0f ? -INFINITY : M0 + __log2f(L) - TOP;
    const int query = (unsigned)rr / (unsigned)group, h = kvh * group + rr - query * group;
    if (runs == 1) {
      const long orow = s.row0 + query;
      Tx4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (T)(sum[e] * inv);
      *reinterpret_cast<Tx4*>(static_cast<T*>(a.out) + orow * a.os.row + h * a.os.head + d) = y;
      if (d == 0 && a.lse) a.lse[orow * a.heads + h] = lse2 * kLn2;
    } else {
      const long slot = first_slot(a, s, r) + ((long)run * a.c.kv_heads + kvh) * s.nq * group + rr;
      *reinterpret_cast<f32x4*>(a.part + slot * D + d) = sum * inv;
      if (d == 0) a.part_lse[slot] = lse2;
    }
  }
}

// Joins the runs of the sequences that were split, in order: D / 4 threads for each row.
template <class T, int D>
__global__ __launch_bounds__(256) void kv16_join_kernel(Kv16AttnArgs a, int join_q) {
  constexpr int EACH = 256 / (D / 4);
  const unsigned row = blockIdx.x * EACH + threadIdx.x / (D / 4);   // (sequence, query, head), below 2^31
  const int d = threadIdx.x % (D / 4) * 4;
  const int h = row % (unsigned)a.heads, i = row / (unsigned)a.heads % (unsigned)join_q;
  const int r = row / (unsigned)a.heads / (unsigned)join_q;
  if (r >= a.n_seqs) return;
  const Seq s = find_seq(a, r);
  if (i >= s.nq) return;
  const int runs = runs_of(a, s);
  if (runs == 1) return;
  const int group = a.heads / a.c.kv_heads, kvh = h / group;
  const long rows = (long)s.nq * group, step = rows * a.c.kv_heads;   // from run to run
  const long slot = first_slot(a, s, r) + kvh * rows + (long)i * group + (h - kvh * group);
  float M = -INFINITY;
  for (int k = 0; k < runs; ++k) M = fmaxf(M, a.part_lse[slot + k * step]);
  const float base = M == -INFINITY ? 0.0f : M;
  float W = 0.0f;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int k = 0; k < runs; ++k) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + (slot + k * step) * D + d);
    const float wk = __builtin_amdgcn_exp2f(a.part_lse[slot + k * step] - base);
    W += wk;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(wk, x[e], sum[e]);
  }
  const float inv = W == 0.0f ? 0.0f : 1.0f / W;
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  Tx4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (T)(sum[e] * inv);
  *reinterpret_cast<Tx4*>(static_cast<T*>(a.out) + (s.row0 + i) * a.os.row + h * a.os.head + d) = y;
  if (d == 0 && a.lse) a.lse[(s.row0 + i) * a.heads + h] = W == 0.0f ? -INFINITY : (M + __log2f(W)) * kLn2;
}

// The most runs of a sequence within the bounds, and the slots of one that is split: runs * queries * heads.
int most_runs(int max_q, int max_len, int heads, int kv_heads) {
  const int group = heads / kv_heads, few = few_runs(max_len, 1, heads, kv_heads);
  if (few_rows(max_q, group)) return few;
  const int many = many_runs(max_len, 1, kv_heads);   // fewer rows, more runs
  return many > few ? many : few;
}
// Of sequences that are split, the most queries
int64_t split_queries(int max_q, int heads) {
  const int64_t many = MANY_ALONE * 128 / heads, few = FEW_ROWS, most = many > few ? many : few;
  return max_q < most ? max_q : most;
}
int64_t seq_slots(int max_q, int max_len, int heads, int kv_heads) {
  return split_queries(max_q, heads) * heads * most_runs(max_q, max_len, heads, kv_heads);
}
// Slots of a call: for each sequence, or for each row, whichever are fewer
int64_t all_slots(int64_t n_rows, int64_t n_seqs, int64_t each, int heads, int runs) {
  const int64_t by_row = n_rows * heads * runs;
  return n_seqs > by_row / each || n_seqs * each >= by_row ? by_row : n_seqs * each;
}

template <class T, int D>
eas_status launch(Kv16AttnArgs& a, hipStream_t s) {
  const int group = a.heads / a.c.kv_heads;
  const int64_t pairs = (int64_t)a.n_seqs * a.c.kv_heads;
  const bool many = !few_rows(a.most_q, group), few = a.cu_q || !many;
  const int64_t rows = (int64_t)a.most_q * group, tiles = ((rows < FEW_ROWS ? rows : FEW_ROWS) + ROWS - 1) / ROWS;
  constexpr int each = 256 / (D / 4);
  const int64_t join_q = split_queries(a.most_q, a.heads), joined = a.n_seqs * join_q;
  if (pairs > 0x7fffffff || (few && !fits_launch(tiles * a.most_runs * pairs, 64 * NW))) return EAS_ERR_UNSUPPORTED;
  if (a.most_runs > 1 && (joined * a.heads > 0x7fffffff || !fits_launch((joined * a.heads + each - 1) / each, 256)))
    return EAS_ERR_UNSUPPORTED;
  if (many) {
    const eas_status st = launch_kv16_many(a, std::is_same_v<T, bf16> ? EAS_BF16 : EAS_FP16, D, s);
    if (st != EAS_OK) return st;
  }
  if (few) {
    a.row_tiles = (int)tiles;
    const int64_t blocks = tiles * a.most_runs * pairs;
    hipLaunchKernelGGL((kv16_tokens_kernel<T, D>), dim3((unsigned)blocks), dim3(64 * NW), 0, s, a);
    if (hipGetLastError() != hipSuccess) return EAS_ERR_HIP;
  }
  if (a.most_runs == 1) return EAS_OK;
  hipLaunchKernelGGL((kv16_join_kernel<T, D>), dim3((unsigned)((joined * a.heads + each - 1) / each)), dim3(256), 0, s, a,
                     (int)join_q);
  return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
}

}  // namespace
}  // namespace eas

using namespace eas;

extern "C" eas_status eas_kv16_attention_workspace(const eas_attn_shape* shape, int32_t n_rows, int32_t max_q,
                                                   int32_t max_len, int32_t n_seqs, int64_t* bytes) {
  const eas_status st = check_shape(shape);
  if (st != EAS_OK) return st;
  if (n_rows < 0 || max_q < 0 || max_len < 0 || n_seqs < 0 || !bytes) return EAS_ERR_INVALID_ARG;
  const int most_q = max_q < n_rows ? max_q : n_rows;
  const int runs = most_runs(most_q, max_len, shape->heads, shape->kv_heads);
  *bytes = 0;
  if (runs == 1 || most_q == 0 || n_seqs == 0) return EAS_OK;
  *bytes = all_slots(n_rows, n_seqs, seq_slots(most_q, max_len, shape->heads, shape->kv_heads), shape->heads, runs) *
           (shape->head_dim + 1) * 4;
  return EAS_OK;
}

extern "C" eas_status eas_kv16_attention(const eas_kv16_cache* cache, const eas_attn_shape* shape, const void* q,
                                         int32_t n_rows, const int32_t* cu_q, int32_t max_q, const int32_t* lens,
                                         int32_t max_len, const int32_t* pages, int32_t max_pages, int32_t n_seqs,
                                         void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                         void* stream) {
  eas_status st = check_cache16(cache);
  if (st == EAS_OK) st = check_shape(shape);
  if (st != EAS_OK) return st;
  if (shape->kv_heads != cache->kv_heads || shape->head_dim != cache->head_dim || shape->dtype != cache->dtype)
    return EAS_ERR_INVALID_ARG;
  st = check_strides(shape->q);
  if (st == EAS_OK) st = check_table16(cache, pages, max_pages, n_seqs);
  if (st != EAS_OK) return st;
  if (n_rows < 0 || max_q < 0 || max_len < 0 || (!lens && n_seqs > 0) || (uintptr_t)lens % 4 || (uintptr_t)cu_q % 4 ||
      (uintptr_t)lse % 4)
    return EAS_ERR_INVALID_ARG;
  st = check_out_strides(shape->out, n_rows, shape->heads, shape->head_dim);
  if (st != EAS_OK) return st;
  if (n_rows == 0 || max_q == 0 || n_seqs == 0) return EAS_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return EAS_ERR_INVALID_ARG;
  Kv16AttnArgs a = {};
  a.c = kv16_args(cache);
  a.q = q, a.out = out, a.lse = lse;
  a.qs = shape->q, a.os = shape->out;
  a.cu_q = cu_q, a.lens = lens, a.pages = pages;
  a.scale_log2 = shape->scale * kLog2e;
  a.heads = shape->heads, a.causal = shape->causal;
  a.n_rows = n_rows, a.max_q = max_q, a.most_q = max_q < n_rows ? max_q : n_rows;
  a.max_pages = max_pages, a.n_seqs = n_seqs;
  const int64_t there = (int64_t)max_pages * cache->page_tokens;
  a.max_len = max_len < there ? max_len : (int)there;
  a.most_runs = most_runs(a.most_q, a.max_len, a.heads, a.c.kv_heads);
  if (a.most_runs > 1) {
    a.slots = seq_slots(a.most_q, a.max_len, a.heads, a.c.kv_heads);
    const int64_t slots = all_slots(n_rows, n_seqs, a.slots, a.heads, a.most_runs);
    if (slots < (int64_t)n_seqs * a.slots) a.slots = 0;
    if (!workspace || !aligned16(workspace)) return EAS_ERR_INVALID_ARG;
    if (workspace_bytes / ((shape->head_dim + 1) * 4) < slots) return EAS_ERR_CAPACITY;
    a.part = static_cast<float*>(workspace);
    a.part_lse = a.part + slots * shape->head_dim;
  }
#define EAS_KV16_CASE(DT, T, D) \
  if (shape->dtype == DT && shape->head_dim == D) return launch<T, D>(a, (hipStream_t)stream)
  EAS_KV16_CASE(EAS_BF16, bf16, 64);
  EAS_KV16_CASE(EAS_BF16, bf16, 128);
  EAS_KV16_CASE(EAS_FP16, f16, 64);
  EAS_KV16_CASE(EAS_FP16, f16, 128);
#undef EAS_KV16_CASE
  return EAS_ERR_UNSUPPORTED;
}
