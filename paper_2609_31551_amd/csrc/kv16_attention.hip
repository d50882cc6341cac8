// Attention of new tokens over the paged 16-bit cache (include/eas_paged.h): the call, sequences with few rows, and the
// join of runs.  Sequences with many rows are kv16_chunks.h's.
//
// A row is one query of one head; the rows of a sequence that share a key / value head (its queries times the
// group's heads) are the columns, 16 or 32 of them, of MFMA products whose rows are the cache's tokens and dimensions:
//   S^T = K Q^T,  O^T += V^T P^T   (v_mfma_f32_16x16x32),
// with one pass over the tokens, the running maximum and sum of the softmax in fp32, and P rounded to the element type
// (2^-8 or 2^-11 of each weight at most, as the result itself).
// The four waves of a workgroup take a quarter of its run's tokens each, 32 at a time, without a barrier between them.
// Keys and values are on their way a tile ahead (two for 16 rows of 64), into registers, in loads that no branch stands
// around, so that each is waited for alone.  Keys are taken by the products as they come; values have to be turned: a wave
// stores its tile to LDS of its own and reads it back by transposing reads.
//
// Bound by HBM, 4 * head_dim bytes a cached token and key / value head: 16 sequences of 32,768 tokens, 8 heads of 128,
// 2,136 MB, take 379 us, 5.6 TB/s (a copy of 1 GiB runs at 5.2).  Short ones are bound by what comes before and behind:
// lengths, pages and first tokens one after the other, 4 us; a workgroup draws 60 GB/s at most, however far ahead its
// loads are (1,023 tokens of one head 13 us, 127 5.3); the join of runs is a launch of 5 us.  32 sequences of 1 to 8,192
// tokens, 4 heads, 141 MB, 41 us.
#include "kv16_chunks.h"

namespace eas {
namespace {

constexpr int TILE = 32;         // tokens per wave and step
constexpr int NW = 4;            // waves per workgroup
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

// maximum and sum over the four lanes that hold one row (lane, lane ^ 16, ^ 32, ^ 48)
__device__ __forceinline__ float column_max(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A tile of values.  Chunk L (16 bytes) of a token's row is stored at chunk L ^ rot: a transposing read takes 32 bytes
// of tokens 8 g + 4 half + e, e and g = 0 .. 3, and hits all banks once for each eight of them.
template <int D>
struct Values {
  static constexpr int R = D / 8;               // chunks per row
  static constexpr int BYTES = TILE * D * 2;
  static constexpr int N = BYTES / 1024;        // loads and stores, 64 chunks each
  static constexpr int TOKENS = 64 / R;         // of a load
  __device__ static int rot(int row) {
    return R == 16 ? 2 * (row & 3) + 8 * (row >> 3 & 1) : 2 * (row >> 1 & 1) + 4 * (row >> 3 & 1);
  }
};

// Bytes of LDS of a workgroup: the waves' tiles of values, and, when they are read, the waves' sums
template <int D, int C>
constexpr int few_lds() {
  return NW * (Values<D>::BYTES > 16 * C * D * 4 ? Values<D>::BYTES : 16 * C * D * 4);
}

// Run `run` of sequence r, whose rows of key / value head kvh are few; C: columns of 16 rows that the workgroup takes;
// smem: few_lds()
template <class T, int D, int C>
__device__ __forceinline__ void few_rows_run(const Kv16AttnArgs& a, int kvh, int r, const Seq& s, int run, char* smem,
                                             int tid) {
  typedef typename Mfma16<T>::x8 x8;
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  using V = Values<D>;
  constexpr int ROWS = 16 * C;
  constexpr int KS = D / 32;   // 32-dimension steps of q . k
  constexpr int DB = D / 16;   // 16-dimension blocks of the output
  constexpr int SETS = C * D == 64 ? 2 : 1;   // tiles on their way
  // log2 of the largest weight: fp16's small weights do not vanish (below 2^-24, 2^-39 of the largest); bf16's sums over
  // all tokens that there may be do not overflow where a softmax's do not
  constexpr float TOP = std::is_same_v<T, f16> ? 15.0f : -30.0f;
  __shared__ float m_part[NW][ROWS], l_part[NW][ROWS];

  const int group = a.heads / a.c.kv_heads, rows = s.nq * group, runs = few_runs(s.len, a.c.kv_heads);
  const int each = few_run_tokens(s.len, runs);
  const int lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // the last query sees most; the run's tokens, and of these the wave's
  const long t_begin = (long)run * each;
  const int t_end = (int)min((long)seen_by(a, s, s.nq - 1), t_begin + each);
  const long w_begin = t_begin + wave * (each / NW);
  const int w0 = (int)min(w_begin, (long)t_end), w1 = (int)min((long)t_end, w_begin + each / NW), last = w1 - 1;
  const int tiles = (w1 - w0 + TILE - 1) / TILE;
  const int* table = a.pages + (long)r * a.max_pages;

  // this lane's rows, and how many tokens they see
  int sees[C];
  x8 qf[C][KS];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int rho = 16 * j + c;
    const bool real = rho < rows;
    const int qi = real ? (unsigned)rho / (unsigned)group : 0, head = kvh * group + (real ? rho - qi * group : 0);
    sees[j] = real ? seen_by(a, s, qi) : 0;
    const T* q = static_cast<const T*>(a.q) + (s.row0 + qi) * a.qs.row + head * a.qs.head;
#pragma unroll
    for (int i = 0; i < KS; ++i) qf[j][i] = *reinterpret_cast<const x8*>(q + 32 * i + 8 * g);
  }

  f32x4 o[C][DB];
  float m[C], l[C];
  const auto clear = [&] {
#pragma unroll
    for (int j = 0; j < C; ++j) {
      m[j] = -INFINITY, l[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  };
  // Weights x of a tile's scores, in place; left: of the lane's 8 tokens, those that its row may see at most
  const auto weigh = [&](f32x4 (*sc)[2], int t0, bool there, float (*x)[8]) {
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int left = there ? sees[j] - (t0 + 8 * g) : 0;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[j][i] = i < left ? sc[j][i >> 2][i & 3] * a.scale_log2 : -INFINITY;
        top = fmaxf(top, x[j][i]);
      }
      top = column_max(top);
      if (__any(top > m[j])) {
        const float up = fmaxf(m[j], top), alpha = up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[j] - up);
        m[j] = up;
        l[j] *= alpha;
#pragma unroll
        for (int i = 0; i < DB; ++i) o[j][i] *= alpha;
      }
      const float base = m[j] == -INFINITY ? 0.0f : m[j];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[j][i] = __builtin_amdgcn_exp2f(x[j][i] - base + TOP);
        l[j] += x[j][i];
      }
    }
  };
  const T* keys = static_cast<const T*>(a.c.k);
  const T* values = static_cast<const T*>(a.c.v);
  const int page_mask = (1 << a.c.page_shift) - 1;

  // Row 4 g + e of score block i is token 8 g + 4 i + e, so that a lane ends with the scores of 8 consecutive tokens, 8 g
  // .. + 8, of its rows: as the products with the values want them.
  const int ktok = 8 * (c >> 2) + (c & 3);   // + 4 i: the token whose key the lane loads for block i
  x8 kf[SETS][2][KS];
  x8 vf[SETS][V::N];
  int parts[SETS];   // which halves of a tile lie in pages that are held
  // The pages of a tile's halves, behind the last token the last one's, by scalar loads: they count apart from the others
  struct Pages { int half[2]; };
  const auto pages_of = [&](int t) {
    const auto* scalar = (const __attribute__((address_space(4))) int*)(uintptr_t)table;
    const int first = w0 + t * TILE;
    return Pages{{scalar[min(first, last) >> a.c.page_shift], scalar[min(first + 16, last) >> a.c.page_shift]}};
  };
  Pages next;   // of the tile that is asked for next
  const int vrow = lane / V::R, vcol = lane % V::R;
  const auto load = [&](int t, int set) {
    const Pages now = next;
    next = pages_of(t + 1);
    parts[set] = (held_page(a, now.half[0]) ? 1 : 0) | (held_page(a, now.half[1]) ? 2 : 0);
    long block[2];   // elements before the head's block
#pragma unroll
    for (int h = 0; h < 2; ++h)
      block[h] = ((long)(held_page(a, now.half[h]) ? now.half[h] : 0) * a.c.kv_heads + kvh) * D << a.c.page_shift;
    const T* kp = keys + (c < 8 ? block[0] : block[1]) + 8 * g;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = min(w0 + t * TILE + ktok + 4 * i, last) & page_mask;   // behind the last token it again
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[set][i][k] = *reinterpret_cast<const x8*>(kp + at * D + 32 * k);
    }
#pragma unroll
    for (int n = 0; n < V::N; ++n) {
      const int first = min(w0 + t * TILE + n * V::TOKENS, last);
      const T* vp = values + block[n * V::TOKENS / 16] + (first & page_mask) * D;
      vf[set][n] = *reinterpret_cast<const x8*>(vp + (unsigned)(min(vrow, last - first) * D + 8 * vcol));
    }
  };
  // V^T operand: lane 16 g + 4 e + i reads token 8 g + 4 half + e, dimensions 16 d + 4 i .. + 4
  const unsigned stage = (unsigned)(size_t)(__attribute__((address_space(3))) char*)smem + wave * V::BYTES;
  const int vtok = 8 * g + (lane >> 2 & 3);
  const unsigned vat = vtok * D * 2 + (V::rot(vtok) + (lane >> 1 & 1)) * 16 + (lane & 1) * 8;   // rot is even, at most R - 2
  const auto read_v = [&](int d) {
    union { x8 v; v4i16 h[2]; } u;
#pragma unroll
    for (int half = 0; half < 2; ++half)
      u.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_v4i16*)(size_t)(stage + (vat ^ d * 32) + half * 4 * D * 2));
    return u.v;
  };
  // Tile t, whose keys and values are in kf[set] and vf[set]; MORE: tile t + SETS follows.
  const auto tile = [&](int t, auto set_, auto more) {
    constexpr int set = decltype(set_)::value;
    f32x4 sc[C][2];
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < KS; ++k) sc[j][i] = Mfma16<T>::go(kf[set][i][k], qf[j][k], sc[j][i]);
      }
    const bool there = parts[set] >> (g >> 1) & 1;
    const auto store = [&](int n, const x8& v) {
      const int row = n * V::TOKENS + vrow;
      *reinterpret_cast<x8*>(smem + wave * V::BYTES + row * D * 2 + (vcol ^ V::rot(row)) * 16) = v;
    };
#pragma unroll
    for (int n = 0; n < V::N; ++n) store(n, vf[set][n]);
    const int held = parts[set];
    if constexpr (decltype(more)::value) load(t + SETS, set);
    float x[C][8];
    weigh(sc, w0 + t * TILE, there, x);
    x8 p[C];
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) p[j][i] = (T)x[j][i];
    if (held != 3)   // for a page that is not held, page 0 was read: another sequence's, with what no weight of 0 may hide
#pragma unroll
      for (int n = 0; n < V::N; ++n)
        if (!(held >> n * V::TOKENS / 16 & 1)) store(n, x8{});
    asm volatile("" ::: "memory");   // the wave's stores come before its reads, which LDS keeps in order
    x8 v[4];   // read ahead
#pragma unroll
    for (int d = 0; d < 4; ++d) v[d] = read_v(d);
#pragma unroll
    for (int d = 0; d < DB; ++d) {
#pragma unroll
      for (int j = 0; j < C; ++j) o[j][d] = Mfma16<T>::go(v[d & 3], p[j], o[j][d]);
      if (d + 4 < DB) v[d & 3] = read_v(d + 4);
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("" ::: "memory");   // and those before the next tile's stores
  };
  clear();
  if (tiles > 0) {
    constexpr std::integral_constant<bool, true> yes{};
    constexpr std::integral_constant<bool, false> no{};
    next = pages_of(0);
    // tiles behind the last are asked for too, the last token again and again: no branch stands around a load
    const auto sets = [&](auto&& f) {
      f(std::integral_constant<int, 0>{});
      if constexpr (SETS == 2) f(std::integral_constant<int, 1>{});
    };
    sets([&](auto set) { load(set, set); });
    int t = 0;
    for (; t + SETS < tiles; t += SETS) sets([&](auto set) { tile(t + set, set, yes); });
    sets([&](auto set) {
      if (t + set < tiles) tile(t + set, set, no);
    });
  }
  // A hidden value went into the products with weight 0: where it is infinite or NaN it shows, and the wave's tokens are
  // walked again, value by value, by the rows that see them.
  uint32_t size = 0;
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) size = max(size, __float_as_uint(o[j][i][e]) & 0x7fffffffu);
  if (__any(size >= 0x7f800000u)) {
    const auto place = [&](int t, bool* there) {
      t = min(t, last);
      const int page = table[t >> a.c.page_shift];
      *there = held_page(a, page);
      return token_offset(a, page, kvh, t, D);
    };
    clear();
    for (int t0 = w0; t0 < w1; t0 += TILE) {
      f32x4 sc[C][2];
      bool there;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const T* kp = keys + place(t0 + ktok + 4 * i, &there) + 8 * g;
#pragma unroll
        for (int j = 0; j < C; ++j) sc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const x8 kk = *reinterpret_cast<const x8*>(kp + 32 * k);
#pragma unroll
          for (int j = 0; j < C; ++j) sc[j][i] = Mfma16<T>::go(kk, qf[j][k], sc[j][i]);
        }
      }
      place(t0 + 8 * g, &there);
      float x[C][8];
      weigh(sc, t0, there, x);
#pragma unroll 1
      for (int from = 0; from < 4; ++from)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = t0 + 8 * from + i;
          const T* vp = values + place(t, &there) + 4 * g;
#pragma unroll
          for (int j = 0; j < C; ++j) {
            const float p = __shfl(x[j][i], 16 * from + c, 64);
            if (t < sees[j] && there)
#pragma unroll
              for (int d = 0; d < DB; ++d) {
                const Tx4 v = *reinterpret_cast<const Tx4*>(vp + 16 * d);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][d][e] = fmaf(p, (float)v[e], o[j][d][e]);
              }
          }
        }
    }
  }

  // the four waves' sums: lane (c, g) holds dimensions 16 i + 4 g .. + 4 of its rows
  __syncthreads();   // the values are read
  float (*o_part)[ROWS][D] = reinterpret_cast<float (*)[ROWS][D]>(smem);
#pragma unroll
  for (int j = 0; j < C; ++j) {
    l[j] = column_sum(l[j]);
    if (g == 0) m_part[wave][16 * j + c] = m[j], l_part[wave][16 * j + c] = l[j];
#pragma unroll
    for (int i = 0; i < DB; ++i) *reinterpret_cast<f32x4*>(&o_part[wave][16 * j + c][16 * i + 4 * g]) = o[j][i];
  }
  __syncthreads();
  for (int i = tid; i < ROWS * (D / 4); i += 64 * NW) {
    const int row = i / (D / 4), d = i % (D / 4) * 4;
    if (row >= rows) break;
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
    if (runs == 1) {
      const int query = (unsigned)row / (unsigned)group, h = kvh * group + row - query * group;
      const long orow = s.row0 + query;
      Tx4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (T)(sum[e] * inv);
      *reinterpret_cast<Tx4*>(static_cast<T*>(a.out) + orow * a.os.row + h * a.os.head + d) = y;
      if (d == 0 && a.lse) a.lse[orow * a.heads + h] = lse2 * kLn2;
    } else {
      const long slot = first_slot(a, s, r) + ((long)run * a.c.kv_heads + kvh) * rows + row;
      *reinterpret_cast<f32x4*>(a.part + slot * D + d) = sum * inv;
      if (d == 0) a.part_lse[slot] = lse2;
    }
  }
}

// One workgroup's work, number `block` of a.few_blocks: of the runs of all sequences with few rows and key / value heads
// the block-th, and where there may be more (MORE) every a.few_blocks-th from it on (as a loop, one run takes 0.3 - 1 us
// longer).
template <class T, int D, int C, bool MORE>
__device__ __forceinline__ void few_rows_runs(const Kv16AttnArgs& a, int block, char* smem) {
  for (;; block += a.few_blocks) {
    int run = (unsigned)block / (unsigned)a.c.kv_heads;
    const auto count = [&](const Seq& s) { return takes_few(a, s) && s.nq > 0 ? few_runs(s.len, a.c.kv_heads) : 0; };
    Seq s;
    int r, all;
    if (a.most_runs == 1) {   // no look at the others' lengths
      r = run, run = 0, all = a.n_seqs;
      if (r >= all) return;
      s = find_seq(a, r);
    } else {
      Items<decltype(count)> items(a, count);
      all = items.all();
      if (run >= all) return;
      r = items.find(&run, &s);
    }
    int tid = threadIdx.x;
    if constexpr (MORE) asm volatile("" : "+v"(tid));   // what follows from it is not kept in registers from run to run
    if (a.most_runs > 1 || count(s)) few_rows_run<T, D, C>(a, block % (unsigned)a.c.kv_heads, r, s, run, smem, tid);
    if (!MORE || (long)block + a.few_blocks >= (long)all * a.c.kv_heads) return;
    __syncthreads();   // the sums are read
  }
}

template <class T, int D, int C, bool MORE>
__global__ __launch_bounds__(64 * NW, 2) void kv16_tokens_kernel(Kv16AttnArgs a) {
  // Of heads of 128 two workgroups a CU, by 56 KB, also where registers are left for three, whose loads stand in each
  // other's way (32 sequences of 1 to 8,192 tokens, 4 heads, 40.9 us, with three 42.1)
  constexpr int LDS = few_lds<D, C>(), TWO = D == 128 ? 56 << 10 : 0;
  __shared__ __attribute__((aligned(1024))) char smem[LDS > TWO ? LDS : TWO];
  few_rows_runs<T, D, C, MORE>(a, blockIdx.x, smem);
}

template <class T, int D, int W>
__global__ __launch_bounds__(64 * W, 2) void kv16_chunks_kernel(Kv16AttnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  many_rows<T, D, W>(a, blockIdx.x, smem);
}

// Both: single tokens' loads beside chunks' products (1,024, 777 and 512 tokens beside five: 132 us, in two launches 144)
template <class T, int D, bool MORE>
__global__ __launch_bounds__(64 * NW, 2) void kv16_mixed_kernel(Kv16AttnArgs a) {
  constexpr int MANY = 4 * KT * D * 2, FEW = few_lds<D, 2>();
  __shared__ __attribute__((aligned(1024))) char smem[MANY > FEW ? MANY : FEW];
  if ((int)blockIdx.x < a.few_blocks)
    few_rows_runs<T, D, 2, MORE>(a, blockIdx.x, smem);
  else
    many_rows<T, D, NW>(a, blockIdx.x - a.few_blocks, smem);
}

// Joins the runs of the sequences that were split, a row by D / 4 threads, or, where rows are few and runs are many, by
// four times as many, each for every fourth run, and their four sums in order (a sequence of 16,384 tokens in 64 runs
// 20 us, joined one run after the other 55).  DIRECT: a.items workgroups for each sequence; else they go over the split
// rows of the batch in strides, as only the sequences' lengths say how many there are, which takes 2 - 3 us more but no
// workgroup for rows that are not split.  The runs' results are means of values that may be as large as bf16's largest, so
// their weights, which sum to 64 at most, are taken by 2^-6: the sum stays in fp32's range, and its bits are the same.
template <class T, int D, bool DIRECT>
__global__ __launch_bounds__(256) void kv16_join_kernel(Kv16AttnArgs a) {
  constexpr int L = D / 4, GROUPS = 256 / L;
  __shared__ f32x4 sums[2][GROUPS][L];
  const int sub = threadIdx.x / L, in = threadIdx.x % L;
  const int group = a.heads / a.c.kv_heads;
  const auto slices_of = [&](const Seq& s) { return takes_few(a, s) ? 4 : 1; };
  const auto count = [&](const Seq& s) {
    const int each = GROUPS / slices_of(s);
    return runs_of(a, s) > 1 ? (int)(((long)s.nq * a.heads + each - 1) / each) : 0;
  };
  const auto find = [&](int* item, Seq* s) {
    if constexpr (DIRECT) {
      const int r = (unsigned)*item / (unsigned)a.items;
      if (r >= a.n_seqs) return -1;
      *item -= r * a.items;
      *s = find_seq(a, r);
      return *item < count(*s) ? r : -1;
    } else {
      Items<decltype(count)> items(a, count);
      return *item < items.all() ? items.find(item, s) : -1;
    }
  };
  for (int first = blockIdx.x, turn = 0;; first += gridDim.x, turn ^= 1) {
    int item = first;
    Seq s;
    const int r = find(&item, &s);
    if (r < 0) return;
    const int runs = runs_of(a, s), slices = slices_of(s), slice = sub % slices;
    const int row = item * (GROUPS / slices) + sub / slices;     // [key / value head, query and head of the group]
    const int rows = s.nq * group, all = rows * a.c.kv_heads;    // all: from run to run, too
    const long slot = first_slot(a, s, r) + min(row, all - 1);
    float M = -INFINITY, W = 0.0f;
    float lse[64 / L];   // of runs in + L e
#pragma unroll
    for (int e = 0; e < 64 / L; ++e) {
      lse[e] = a.part_lse[slot + (long)min(in + L * e, runs - 1) * all];
      M = fmaxf(M, lse[e]);
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
    const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int e = 0; e < 64 / L; ++e) W += in + L * e < runs ? __builtin_amdgcn_exp2f(lse[e] - base) : 0.0f;
#pragma unroll
    for (int o = L / 2; o; o >>= 1) W += __shfl_xor(W, o, 64);
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int k = slice; k < runs; k += slices) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + (slot + (long)k * all) * D + in * 4);
      const float wk = __builtin_amdgcn_exp2f(a.part_lse[slot + (long)k * all] - base) * 0x1p-6f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(wk, x[e], sum[e]);
    }
    sums[turn][sub][in] = sum;
    __syncthreads();   // what is read here is written again two turns on, behind the next barrier
    if (slices > 1) {
#pragma unroll
      for (int k = 1; k < 4; ++k) sum += sums[turn][(sub + k) % GROUPS][in];   // slice 0's: of slices 1, 2, 3
    }
    if (slice || row >= all) continue;
    const float inv = W == 0.0f ? 0.0f : 1.0f / W * 0x1p6f;
    typedef T Tx4 __attribute__((ext_vector_type(4)));
    Tx4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (T)(sum[e] * inv);
    const int kvh = (unsigned)row / (unsigned)rows, in_head = row - kvh * rows, i = (unsigned)in_head / (unsigned)group;
    const int h = kvh * group + in_head - i * group;
    *reinterpret_cast<Tx4*>(static_cast<T*>(a.out) + (s.row0 + i) * a.os.row + h * a.os.head + in * 4) = y;
    if (in == 0 && a.lse)
      a.lse[(s.row0 + i) * a.heads + h] = W == 0.0f ? -INFINITY : ((M == -INFINITY ? 0.0f : M) + __log2f(W)) * kLn2;
  }
}

// The most runs of a sequence within the bounds, and the slots of one that is split: runs * queries * heads.
int most_runs(int max_q, int max_len, int heads, int kv_heads) {
  const int group = heads / kv_heads, few = few_runs(max_len, kv_heads);
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
  const int64_t rows = (int64_t)max_q * heads, few = few_runs(max_len, kv_heads), most_few = FEW_ROWS * kv_heads;
  const int64_t of_few = (rows < most_few ? rows : most_few) * few;
  if (few_rows(max_q, heads / kv_heads)) return of_few;
  const int64_t many = split_queries(max_q, heads) * heads * many_runs(max_len, 1, kv_heads), most = MANY_FILL * 128;
  const int64_t of_many = many < most ? many : most;
  return of_few > of_many ? of_few : of_many;
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
  // 256 rows a workgroup share what is fetched among twice the rows of 128; where they leave each CU a workgroup, and
  // little of one idle behind a sequence's last row: 4,096 tokens of 28 heads over 4 behind 32,768 1,830 us and 1,982, but
  // 2,048 of 20 over 20 behind 8,192 175 and 163, and chunks of 512 to 1,024 beside single tokens 155 and 143.  A row's
  // arithmetic is the same.
  const bool wide = (int64_t)a.n_rows * a.heads >= 256ll * device_cus() && (int64_t)a.n_rows * group >= 1024ll * a.n_seqs;
  const int64_t items = !many ? 0 : wide ? many_items<D, 8>(a) : many_items<D, 4>(a);
  const int64_t many_blocks = tile_workgroups(items, a.c.kv_heads, a.c.kv_heads);
  // Runs of short and long sequences are packed, so that workgroups without work leave no XCD or CU with less than others
  // (eight of 333 to 9,000 tokens 16 us, 21 with a place for each that there may be), and as many workgroups are launched
  // as have work where sequences are split in two: only the device knows, and one without work costs a look at the lengths
  // (128 sequences of 1,024 tokens, 131,072 allowed: 101 us, with places for all 155)
  const int64_t two_each = 2 * pairs < 4096 ? 4096 : 2 * pairs;
  const int64_t few_blocks = !few ? 0 : a.most_runs * pairs < two_each ? a.most_runs * pairs : two_each;
  if (pairs * a.most_runs > 0x7fffffff || items > 0x7fffffff || (int64_t)a.n_rows * group > 0x7fffff00 ||
      !fits_launch(many_blocks, 512) || !fits_launch(few_blocks, 64 * NW) ||
      !fits_launch(many_blocks + few_blocks + 8, 64 * NW))
    return EAS_ERR_UNSUPPORTED;
  a.items = (int)items, a.few_blocks = (int)few_blocks;
  constexpr int lds = 4 * KT * D * 2;   // of many_rows
  const dim3 few_grid((unsigned)few_blocks), many_grid((unsigned)many_blocks);
  const bool more = few_blocks < a.most_runs * pairs;
  const auto run = [&](auto kernel, dim3 grid, int threads, int shared) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), shared, s, a);
  };
  if (few && many && !wide) {
    a.few_blocks = (int)((few_blocks + 7) / 8 * 8);   // the others' numbers still tell their XCD
    const dim3 grid((unsigned)(a.few_blocks + many_blocks));
    run(more ? kv16_mixed_kernel<T, D, true> : kv16_mixed_kernel<T, D, false>, grid, 64 * NW, 0);
  } else {
    if (many) run(wide ? kv16_chunks_kernel<T, D, 8> : kv16_chunks_kernel<T, D, 4>, many_grid, wide ? 512 : 256, lds);
    if (few && (int64_t)a.most_q * group <= 16)
      run(more ? kv16_tokens_kernel<T, D, 1, true> : kv16_tokens_kernel<T, D, 1, false>, few_grid, 64 * NW, 0);
    else if (few)
      run(more ? kv16_tokens_kernel<T, D, 2, true> : kv16_tokens_kernel<T, D, 2, false>, few_grid, 64 * NW, 0);
  }
  if (hipGetLastError() != hipSuccess) return EAS_ERR_HIP;
  if (a.most_runs == 1) return EAS_OK;
  constexpr int64_t each = 256 / (D / 4);   // rows of a workgroup; of one for a sequence's few rows a quarter
  const int64_t every = (int64_t)a.n_rows * a.heads / each + a.n_seqs;
  const int64_t of_many = many ? split_queries(a.most_q, a.heads) * a.heads / each + 1 : 0;
  const int64_t few_most = (int64_t)a.most_q * group < FEW_ROWS ? (int64_t)a.most_q * group : FEW_ROWS;
  const int64_t of_few = few ? (4 * few_most * a.c.kv_heads + each - 1) / each : 0;
  const int64_t seq = of_many > of_few ? of_many : of_few;
  if (a.n_seqs * seq <= 8192) {
    a.items = (int)seq;
    hipLaunchKernelGGL((kv16_join_kernel<T, D, true>), dim3((unsigned)(a.n_seqs * seq)), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
  }
  const int64_t blocks = 4 * every;
  constexpr int64_t most = 4096;
  hipLaunchKernelGGL((kv16_join_kernel<T, D, false>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, a);
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
  // where all sequences have the same number of queries it is known here
  a.most_runs = !cu_q && (int64_t)max_q * n_seqs == n_rows && !few_rows(max_q, a.heads / a.c.kv_heads)
                    ? many_runs(a.max_len, (long)max_q * (a.heads / a.c.kv_heads), a.c.kv_heads)
                    : most_runs(a.most_q, a.max_len, a.heads, a.c.kv_heads);
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
