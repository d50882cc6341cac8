// Attention of new tokens over the 8-bit cache (include/eas_attention.h).
//
// A row is one query of one head; the rows of a sequence that share a key / value head
// (its queries times the group's heads) are taken 16 at a time, as the columns of MFMA
// products whose rows are the cache's tokens and dimensions:
//   S^T = K Q^T,  O^T += V^T P^T   (v_mfma_f32_16x16x32_f16).
// A wave walks tiles of 64 tokens.  Which token sits in which MFMA row is free, and is
// chosen so that a lane ends with the 16 scores of 16 consecutive tokens of one query and
// needs the values of the same 16 tokens of one dimension: one 16-byte load from the value
// codes, which are stored dimension by dimension for that.  Nothing goes through LDS but
// the waves' final sums.  The 16 tokens lie in one page, whatever its size, so a lane
// looks up one scale of each kind.
//
// Codes are exact in fp16 (both formats).  Queries are multiplied by a power of two for each
// row that brings its largest value to [2^14, 2^15); in fp16 each is then good to 2^-25, which
// is 2^-39 of the largest (and exact from 2^-31 of it on, where 8 bits fit above fp16's last).
// Scores are exact products of such values, summed in fp32.  With block scales 2^f of the
// values, x = scale * q . k in log2 units and running maxima m of x and m' of x + f - 15, a
// lane sums l += 2^(x - m) and O += 2^(x + f - m') * code: whatever the scales, the largest
// weight of a code is 2^15, so rounding the weights to fp16 costs 2^-11 of each, or of those
// below fp16's normal range 2^-40 of the largest.
//
// A sequence's tokens are split into runs by a rule on its own length and queries only,
// so its result does not depend on the batch; each run's result goes to the workspace
// and a second kernel joins them in order.
//
// Bound by HBM, a byte of codes for each 2 (queries * group) multiply-adds: 16 sequences of 32,768 tokens, 8 heads of
// 128, 1,068 MB in 201 us, 5.3 TB/s.  32 sequences of 1 - 8,192 tokens, 4 heads, 71 MB, take 23 us: 14 of bytes, a wave's first
// loads one after the other (lengths, pages, scales, codes) and the join, 4 us.
#include <type_traits>

#include "attention_ops.h"

namespace eas {
namespace {

constexpr int TILE = 64;         // tokens per wave and step
constexpr int NW = 4;            // waves per workgroup
constexpr int MAX_RUNS = 64;     // runs per sequence
constexpr int RUN_ROWS = 256;    // runs * queries of a sequence that is split

// Runs that `len` tokens are split into for nq queries, and a run's tokens: 1,024 at least.  A run costs its first
// loads' latency and its share of the join, so full batches want long ones (16 sequences of 32,768 tokens, 8 heads of
// 128: 224 us with runs of 512 tokens, 206 with 1,024; 32 of 2,048, 20 heads of 64: 36.3 and 35.0), single sequences
// short ones (one of 4,096: 11.3 and 13.8 us).
constexpr int SHORTEST_RUN = 1024;
__host__ __device__ inline int n_runs(int len, int nq) {
  const int by_len = (int)(((unsigned)len + SHORTEST_RUN - 1) / SHORTEST_RUN);   // len <= 2^30: 32 bits hold all sums here
  int most = nq > 0 ? RUN_ROWS / nq : 1;
  most = most < 1 ? 1 : most > MAX_RUNS ? MAX_RUNS : most;
  return by_len < 1 ? 1 : by_len < most ? by_len : most;
}
__host__ __device__ inline int run_tokens(int len, int runs) {
  const unsigned all = (unsigned)runs * (NW * TILE);
  return (int)(((unsigned)len + all - 1) / all) * (NW * TILE);
}
// Workspace slots per sequence and head: at least n_runs * nq for every nq <= max_q, len <= max_len
// of a sequence that is split
inline int64_t slots(int max_q, int max_len) {
  const int64_t rows = (int64_t)n_runs(max_len, 1) * max_q;
  return rows < RUN_ROWS ? rows : RUN_ROWS;
}

struct Kv8AttnArgs {
  Kv8Args c;
  const void* q;
  void* out;
  float* lse;
  eas_strides qs, os;
  const int* cu_q;
  const int* lens;
  const int* pages;
  float* part;          // [n_seqs, heads, slots, D] results of runs, then [n_seqs, heads, slots] their log2 sums
  float* part_lse;
  float scale_log2;     // scale * log2(e)
  int heads, causal, n_rows, max_len, max_pages, n_seqs, slots, row_tiles, runs;
  int max_q, most_q;    // the caller's, and a bound of the queries of a sequence that are computed
};

struct Seq {
  long row0;     // row of the first query that is computed
  int before;    // tokens before that query's own, where causal: it sees before + 1
  int nq, len;   // queries that are computed, tokens that may be seen
};

// A sequence's queries without those beyond max_q and those of rows outside [0, n_rows): the others keep their places.
// Prefix sums that do not fit may wrap; what is computed lies in [0, n_rows) whatever they hold.
__device__ __forceinline__ Seq find_seq(const Kv8AttnArgs& a, int r) {
  Seq s;
  unsigned lq = a.max_q;
  s.row0 = (long)r * a.max_q;
  if (a.cu_q) {
    s.row0 = a.cu_q[r];
    lq = (unsigned)a.cu_q[r + 1] - (unsigned)a.cu_q[r];
  }
  const int len = max(0, min(a.lens[r], a.max_pages << a.c.page_shift));
  const int skip = (int)max(-s.row0, 0l) & 0x7fffffff;
  s.before = (int)((unsigned)len - lq + (unsigned)skip);
  s.row0 = max(s.row0, 0l);
  s.nq = (int)max(min((long)(min(max((int)lq, 0), a.max_q) - skip), a.n_rows - s.row0), 0l);
  s.len = min(len, a.max_len);
  return s;
}
// Tokens that computed query i sees
__device__ __forceinline__ int seen_by(const Kv8AttnArgs& a, const Seq& s, int i) {
  return a.causal ? max(0, min(s.len, s.before + i + 1)) : s.len;
}

// 16 codes to fp16, exactly: int8 by building 1024 + (code + 128) and taking 1152 off
template <int FORMAT>
__device__ __forceinline__ void codes_to_f16(const uint4& w, f16x8* lo, f16x8* hi) {
  union { f16x2 h[8]; f16x8 v[2]; } u;
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (FORMAT == EAS_KV_INT8) {
      const uint32_t b = x[i] ^ 0x80808080u;
      union { uint32_t u; f16x2 h; } p0, p1;
      p0.u = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
      p1.u = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
      u.h[2 * i] = p0.h - (f16)1152.0f;
      u.h[2 * i + 1] = p1.h - (f16)1152.0f;
    } else {
      u.h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[i], 1.0f, false);
      u.h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[i], 1.0f, true);
    }
  }
  *lo = u.v[0];
  *hi = u.v[1];
}

// the first n of 16 bytes, the others 0
__device__ __forceinline__ uint4 first_bytes(uint4 w, int n) {
  uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = min(max(n - 4 * i, 0), 4);
    x[i] &= k == 4 ? 0xffffffffu : (1u << 8 * k) - 1;
  }
  return make_uint4(x[0], x[1], x[2], x[3]);
}

// maximum over the four lanes that hold one query (lane, lane ^ 16, ^ 32, ^ 48)
__device__ __forceinline__ float column_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// C: tiles of 16 rows that a workgroup takes.  Two share what is loaded and turned to fp16, but a wave walks for
// both: see columns().
template <class T, int FORMAT, int D, int C>
__global__ __launch_bounds__(64 * NW) void kv8_attention_kernel(Kv8AttnArgs a) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  constexpr int DX = D / 64;   // 64-dimension parts of a key
  constexpr int DB = D / 16;   // 16-dimension blocks of the output
  constexpr int ROWS = 16 * C;
  __shared__ float o_part[NW][ROWS][D];
  __shared__ float m_part[NW][ROWS], mv_part[NW][ROWS], l_part[NW][ROWS];

  // Workgroups go to the 8 XCDs in turn.  The row tiles of one run, which read the same codes, are 8 apart, on one
  // XCD: 32 sequences of 2,048 tokens, 3 queries of 28 heads over 4, 27.2 us, dealt out in turn 32.5; 8 of 4,096, 16
  // queries of 32 heads over 8, 47.6 and 54.3; short ragged ones pay for the uneven load: 8 of 333 - 9,000, 5 of 16
  // over 4, 15.4 and 14.2.
  unsigned b = blockIdx.x / 8;
  const int rt = b % (unsigned)a.row_tiles;
  b = b / (unsigned)a.row_tiles * 8 + blockIdx.x % 8;
  const int run = b % (unsigned)a.runs;
  b /= (unsigned)a.runs;
  const int kvh = b % (unsigned)a.c.kv_heads, rb = b / (unsigned)a.c.kv_heads, r = min(rb, a.n_seqs - 1);
  const Seq s = find_seq(a, r);
  const int group = a.heads / a.c.kv_heads;
  if (rb != r || (long)rt * ROWS >= (long)s.nq * group) return;
  const int runs = n_runs(s.len, s.nq);
  if (run >= runs) return;
  const int each = run_tokens(s.len, runs);
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // this lane's queries, and how many tokens they see
  int sees[C];
  const T* q[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int rho = rt * ROWS + 16 * j + c;
    const bool real = rho < s.nq * group;
    const int qi = real ? (unsigned)rho / (unsigned)group : 0, h = kvh * group + (real ? rho - qi * group : 0);
    sees[j] = real ? seen_by(a, s, qi) : 0;
    q[j] = static_cast<const T*>(a.q) + (s.row0 + qi) * a.qs.row + h * a.qs.head + 16 * g;
  }
  // the last query sees most
  const int last = min(rt * ROWS + ROWS - 1, s.nq * group - 1) / group;
  const int most = seen_by(a, s, last);
  const long t_begin = (long)run * each;
  const int t_end = (int)min((long)most, t_begin + each);

  // The next tile's keys are fetched as soon as a tile's scores have taken theirs, its values behind the products with
  // this tile's, its page numbers a tile before and its scales before its keys: loads are in flight all the time, in one
  // tile's registers, and what is waited for is always older than they are (no load is in a branch, or the compiler
  // would count on none and wait for all; the last tile is a copy without loads).  Lane (c, g) holds scores and values
  // of tokens t0 + 16 g .. + 16, and loads keys of tokens t0 + 16 (c / 4) + 4 i + c % 4, i < 4.
  constexpr int STEP = NW * TILE;
  int t0 = (int)t_begin + wave * TILE;
  const int page_mask = (1 << a.c.page_shift) - 1;
  const int* table = a.pages + (long)r * a.max_pages;
  uint4 kw[4][DX], vw[DB];
  float ks, vs;
  int pv, pk;    // pages of the tokens whose scores and values the lane holds, and of those whose keys it loads
  bool there;    // pv is one
  const auto find = [&](int t) {   // behind the last token its page again (nothing of it is seen)
    pv = table[min(t + 16 * g, t_end - 1) >> a.c.page_shift];
    pk = table[min(t + 16 * (c >> 2), t_end - 1) >> a.c.page_shift];
  };
  const auto held_page = [&](int page) { return page >= 0 && page < a.c.n_pages; };
  const auto block_of = [&](int page) { return (long)(held_page(page) ? page : 0) * a.c.kv_heads + kvh; };
  const auto load_k = [&](int t, int page) {
    const int tk = t + 16 * (c >> 2);
    const uint8_t* kp = a.c.k + ((block_of(page) << a.c.page_shift) + (tk & page_mask) + (c & 3)) * D + 16 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < DX; ++x) kw[i][x] = *reinterpret_cast<const uint4*>(kp + 4 * i * D + 64 * x);
  };
  const auto load_v = [&](int t, int page) {
    const int tv = t + 16 * g;
    const uint8_t* vp = a.c.v + ((block_of(page) * D + c) << a.c.page_shift) + (tv & page_mask);
#pragma unroll
    for (int i = 0; i < DB; ++i) vw[i] = *reinterpret_cast<const uint4*>(vp + ((long)16 * i << a.c.page_shift));
  };
  const auto load_scales = [&](int page) {
    const long block = block_of(page);
    ks = a.c.k_scale[block];
    vs = a.c.v_scale[block];
  };
  if (t0 < t_end) find(t0);
  Tx8 qv[C][2 * DX];
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int x = 0; x < DX; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) qv[j][2 * x + y] = *reinterpret_cast<const Tx8*>(q[j] + 64 * x + 8 * y);

  // queries times a power of two that brings the row's largest to [2^14, 2^15)
  f16x8 qf[C][2 * DX];
  float q_scale[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 2 * DX; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)qv[j][i][e]));
    top = column_max(top);
    // 2^(14 - floor(log2 top)), kept in the normal range
    const int e = min(max((int)(__float_as_uint(top) >> 23), 15), 254);
    const float up = __uint_as_float((uint32_t)min(268 - e, 254) << 23);
    q_scale[j] = a.scale_log2 * __uint_as_float((uint32_t)max(e - 14, 0) << 23);
#pragma unroll
    for (int i = 0; i < 2 * DX; ++i)
#pragma unroll
      for (int e8 = 0; e8 < 8; ++e8) qf[j][i][e8] = (f16)((float)qv[j][i][e8] * up);
  }

  f32x4 o[C][DB];
  float m[C], mv[C], l[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
#pragma unroll
    for (int i = 0; i < DB; ++i) o[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m[j] = mv[j] = -INFINITY, l[j] = 0.0f;
  }

  if (t0 < t_end) {
    const int pv0 = pv, pk0 = pk;
    there = held_page(pv0);
    find(t0 + STEP);
    load_scales(pv0);
    load_k(t0, pk0);
    load_v(t0, pv0);
  }
  const auto tile = [&](auto last) {
    constexpr bool MORE = !decltype(last)::value;
    const int tv = t0 + 16 * g;
    // scores of tokens tv + 4 i + e of this lane's queries
    f32x4 sc[C][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < C; ++j) sc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int d = 0; d < DX; ++d) {
        f16x8 k0, k1;
        codes_to_f16<FORMAT>(kw[i][d], &k0, &k1);
#pragma unroll
        for (int j = 0; j < C; ++j) {
          sc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qf[j][2 * d], sc[j][i], 0, 0, 0);
          sc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qf[j][2 * d + 1], sc[j][i], 0, 0, 0);
        }
      }
    }
    const float k_scale = ks;
    const float f = vs > 0.0f ? (float)((int)(__float_as_uint(vs) >> 23) - 127) : -INFINITY;
    const bool was = there;
    const int held = was ? s.len - tv : 0;        // places behind the last token may hold anything
    const int pv1 = pv, pk1 = pk;
    if constexpr (MORE) {
      there = held_page(pv1);
      find(t0 + 2 * STEP);
      load_scales(pv1);
      load_k(t0 + STEP, pk1);
    }
    f16x8 p[C][2];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int left = was ? sees[j] - tv : 0;    // of the lane's 16 tokens, those its query sees
      const float ck = q_scale[j] * k_scale;
      // in log2 units
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = i < left ? sc[j][i >> 2][i & 3] * ck : -INFINITY;
      float top = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
      const float top_m = column_max(top), top_v = column_max(top + f) - 15.0f;
      if (__any(top_m > m[j])) {
        const float up = fmaxf(m[j], top_m);
        l[j] *= up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[j] - up);
        m[j] = up;
      }
      if (__any(top_v > mv[j])) {
        const float up = fmaxf(mv[j], top_v);
        const float alpha = up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mv[j] - up);
        mv[j] = up;
#pragma unroll
        for (int i = 0; i < DB; ++i) o[j][i] *= alpha;
      }
      // p = 2^(x - m); a code's weight is p 2^(m + f - m')
      const float m0 = m[j] == -INFINITY ? 0.0f : m[j], mv0 = mv[j] == -INFINITY ? 0.0f : mv[j];
      const float weight = f == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(fminf(m0 + f - mv0, 126.0f));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(x[i] - m0);
        l[j] += e;
        p[j][i >> 3][i & 7] = (f16)(e * weight);
      }
    }
    if (__any(held < 16)) {
#pragma unroll
      for (int i = 0; i < DB; ++i) vw[i] = first_bytes(vw[i], held);
    }
#pragma unroll
    for (int i = 0; i < DB; ++i) {
      f16x8 v0, v1;
      codes_to_f16<FORMAT>(vw[i], &v0, &v1);
#pragma unroll
      for (int j = 0; j < C; ++j) {
        o[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[j][0], o[j][i], 0, 0, 0);
        o[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[j][1], o[j][i], 0, 0, 0);
      }
    }
    if constexpr (MORE) load_v(t0 + STEP, pv1);
  };
  for (; t0 + STEP < t_end; t0 += STEP) tile(std::false_type{});
  if (t0 < t_end) tile(std::true_type{});
  // the four waves' sums: lane (c, g) holds dimensions 16 i + 4 g .. + 4 of query c of each column tile
#pragma unroll
  for (int j = 0; j < C; ++j) {
    l[j] += __shfl_xor(l[j], 16, 64);
    l[j] += __shfl_xor(l[j], 32, 64);
    if (g == 0) {
      m_part[wave][16 * j + c] = m[j];
      mv_part[wave][16 * j + c] = mv[j];
      l_part[wave][16 * j + c] = l[j];
    }
#pragma unroll
    for (int i = 0; i < DB; ++i) *reinterpret_cast<f32x4*>(&o_part[wave][16 * j + c][16 * i + 4 * g]) = o[j][i];
  }
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
      L += l_part[w][row] * __builtin_amdgcn_exp2f(m_part[w][row] - M0);
      const float beta = __builtin_amdgcn_exp2f(mv_part[w][row] - M0);
      sum += *reinterpret_cast<const f32x4*>(&o_part[w][row][d]) * beta;
    }
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const float lse2 = L == 0.0f ? -INFINITY : M0 + __log2f(L);
    const int q = (unsigned)rr / (unsigned)group, head = kvh * group + rr - q * group;
    if (runs == 1) {
      const long orow = s.row0 + q;
      typedef T Tx4 __attribute__((ext_vector_type(4)));
      Tx4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (T)(sum[e] * inv);
      *reinterpret_cast<Tx4*>(static_cast<T*>(a.out) + orow * a.os.row + head * a.os.head + d) = y;
      if (d == 0 && a.lse) a.lse[orow * a.heads + head] = lse2 * kLn2;
    } else {
      const long slot = ((long)r * a.heads + head) * a.slots + q * runs + run;
      *reinterpret_cast<f32x4*>(a.part + slot * D + d) = sum * inv;
      if (d == 0) a.part_lse[slot] = lse2;
    }
  }
}

// Joins the runs of the sequences that were split: a wave for each row.
template <class T, int D>
__global__ __launch_bounds__(64 * NW) void kv8_join_kernel(Kv8AttnArgs a) {
  const unsigned row = blockIdx.x * NW + (threadIdx.x >> 6);   // (sequence, query, head), below 2^31
  const int lane = threadIdx.x & 63;
  const int h = row % (unsigned)a.heads, q = row / (unsigned)a.heads % (unsigned)a.most_q;
  const int r = row / (unsigned)a.heads / (unsigned)a.most_q;
  if (r >= a.n_seqs) return;
  const Seq s = find_seq(a, r);
  if (q >= s.nq) return;
  const int runs = n_runs(s.len, s.nq);
  if (runs == 1) return;
  const long slot = ((long)r * a.heads + h) * a.slots + q * runs;
  const float lse2 = lane < runs ? a.part_lse[slot + lane] : -INFINITY;
  float M = lse2;
#pragma unroll
  for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float M0 = M == -INFINITY ? 0.0f : M;
  const float w = __builtin_amdgcn_exp2f(lse2 - M0);
  const float W = wave_sum(w), inv = W == 0.0f ? 0.0f : 1.0f / W;
  constexpr int E = D / 64;
  // runs in order, eight loads in flight; behind the last one the last again, with weight 0
  float sum[E] = {};
  for (int k = 0; k < runs; k += 8) {
    float x[8][E];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) x[i][e] = a.part[(slot + min(k + i, runs - 1)) * D + lane * E + e];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float wk = __shfl(w, min(k + i, 63), 64);
      if (k + i < runs)
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += wk * x[i][e];
    }
  }
  T* out = static_cast<T*>(a.out) + (s.row0 + q) * a.os.row + h * a.os.head + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] = (T)(sum[e] * inv);
  if (lane == 0 && a.lse) a.lse[(s.row0 + q) * a.heads + h] = W == 0.0f ? -INFINITY : (M0 + __log2f(W)) * kLn2;
}

// Workgroups that take `tiles` row tiles of all runs and heads
int64_t workgroups(const Kv8AttnArgs& a, int64_t tiles) {
  return ((int64_t)a.runs * a.c.kv_heads * a.n_seqs + 7) / 8 * 8 * tiles;
}

// Tiles of 16 rows per workgroup.  Two where they leave two workgroups a CU, the most that fit: 8 sequences of 4,096
// tokens, 8 key heads of 128, 64 queries of 32 heads 110 us against 138; 64 of 300, 5 queries 16.3 against 20.2.  With
// fewer a call waits for a wave's walk, which two make longer: one sequence, 5 queries 19.2 against 14.5.  Heads of 64,
// whose waves keep less, gain nothing up to 16 queries of 16 heads over 4 (30.3 and 29.5).  A row's result is the same.
template <int D>
int columns(const Kv8AttnArgs& a, int64_t rows) {
  return D == 128 && workgroups(a, (rows + 31) / 32) >= 2l * device_cus() ? 2 : 1;
}

template <class T, int FORMAT, int D>
eas_status launch(Kv8AttnArgs& a, int64_t rows, bool join, hipStream_t s) {
  const int64_t joined = (int64_t)a.n_seqs * a.most_q * a.heads;
  if (joined > 0x7fffffff || (join && !fits_launch((joined + NW - 1) / NW, 64 * NW))) return EAS_ERR_UNSUPPORTED;
  const int C = rows > 16 ? columns<D>(a, rows) : 1;
  const int64_t tiles = (rows + 16 * C - 1) / (16 * C), blocks = workgroups(a, tiles);
  if (!fits_launch(blocks, 64 * NW)) return EAS_ERR_UNSUPPORTED;
  a.row_tiles = (int)tiles;
  if constexpr (D == 128) {
    if (C == 2) hipLaunchKernelGGL((kv8_attention_kernel<T, FORMAT, D, 2>), dim3(blocks), dim3(64 * NW), 0, s, a);
  }
  if (C == 1) hipLaunchKernelGGL((kv8_attention_kernel<T, FORMAT, D, 1>), dim3(blocks), dim3(64 * NW), 0, s, a);
  if (hipGetLastError() != hipSuccess) return EAS_ERR_HIP;
  if (!join) return EAS_OK;
  hipLaunchKernelGGL((kv8_join_kernel<T, D>), dim3((unsigned)((joined + NW - 1) / NW)), dim3(64 * NW), 0, s, a);
  return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
}

}  // namespace
}  // namespace eas

using namespace eas;

extern "C" eas_status eas_kv8_attention_workspace(const eas_attn_shape* shape, int32_t max_q, int32_t max_len,
                                                  int32_t n_seqs, int64_t* bytes) {
  const eas_status st = check_shape(shape);
  if (st != EAS_OK) return st;
  if (max_q < 0 || max_len < 0 || n_seqs < 0 || !bytes) return EAS_ERR_INVALID_ARG;
  *bytes = n_runs(max_len, 1) == 1 ? 0 : (int64_t)n_seqs * shape->heads * slots(max_q, max_len) * (shape->head_dim + 1) * 4;
  return EAS_OK;
}

extern "C" eas_status eas_kv8_attention(const eas_kv8_cache* cache, const eas_attn_shape* shape, const void* q,
                                        int32_t n_rows, const int32_t* cu_q, int32_t max_q, const int32_t* lens,
                                        int32_t max_len, const int32_t* pages, int32_t max_pages, int32_t n_seqs,
                                        void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                        void* stream) {
  eas_status st = check_cache(cache);
  if (st == EAS_OK) st = check_shape(shape);
  if (st != EAS_OK) return st;
  if (shape->kv_heads != cache->kv_heads || shape->head_dim != cache->head_dim) return EAS_ERR_INVALID_ARG;
  st = check_strides(shape->q);
  if (st == EAS_OK) st = check_table(cache, pages, max_pages, n_seqs);
  if (st != EAS_OK) return st;
  if (n_rows < 0 || max_q < 0 || max_len < 0 || (!lens && n_seqs > 0) || (uintptr_t)lens % 4 || (uintptr_t)cu_q % 4 ||
      (uintptr_t)lse % 4)
    return EAS_ERR_INVALID_ARG;
  st = check_out_strides(shape->out, n_rows, shape->heads, shape->head_dim);
  if (st != EAS_OK) return st;
  if (n_rows == 0 || max_q == 0 || n_seqs == 0) return EAS_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return EAS_ERR_INVALID_ARG;
  Kv8AttnArgs a = {};
  a.c = kv8_args(cache);
  a.q = q, a.out = out, a.lse = lse;
  a.qs = shape->q, a.os = shape->out;
  a.cu_q = cu_q, a.lens = lens, a.pages = pages;
  a.scale_log2 = shape->scale * kLog2e;
  a.heads = shape->heads, a.causal = shape->causal;
  a.n_rows = n_rows, a.max_q = max_q, a.most_q = cu_q && n_rows < max_q ? n_rows : max_q;
  a.max_pages = max_pages, a.n_seqs = n_seqs;
  const int64_t held = (int64_t)max_pages * cache->page_tokens;
  a.max_len = max_len < held ? max_len : (int)held;
  a.runs = n_runs(a.max_len, 1);
  const bool join = a.runs > 1;
  a.slots = (int)slots(a.most_q, a.max_len);
  if (join) {
    const int64_t parts = (int64_t)n_seqs * a.heads * a.slots;
    if (!workspace || !aligned16(workspace)) return EAS_ERR_INVALID_ARG;
    if (workspace_bytes < parts * (shape->head_dim + 1) * 4) return EAS_ERR_CAPACITY;
    a.part = static_cast<float*>(workspace);
    a.part_lse = a.part + parts * shape->head_dim;
  }
  const int group = a.heads / a.c.kv_heads;
  const int64_t rows = (int64_t)(max_q < n_rows ? max_q : n_rows) * group;
#define EAS_KV8_CASE(DT, T, F, D)                                                   \
  if (shape->dtype == DT && cache->format == F && shape->head_dim == D) \
    return launch<T, F, D>(a, rows, join, (hipStream_t)stream)
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
