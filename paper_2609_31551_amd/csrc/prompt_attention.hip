// Attention over packed prompts, causal or full, with grouped heads
// (include/eas_attention.h).
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup owns 128 or 256 queries of one
// (sequence, head), a wave 32 of them; keys and values stream through LDS in tiles of 64, anchored at the sequence's
// first key, so a query's result does not depend on where its sequence lies.
//   S^T = K Q^T (v_mfma_f32_32x32x16: keys are rows, so a lane holds 16 scores of one query), softmax in fp32 on exp2,
//   O^T += V^T P^T with P rounded to the element type: by 2^-8 (bf16) or 2^-11 (fp16) of each weight at most, as the
//   result itself.
// The tiles come by DMA, two of each kind in LDS, while the tile before is worked on; a wave's softmax stands between
// the MFMAs of the next tile's scores and of its own values, step by step.
//
// Bound by the matrix units: 4 * head_dim flops for each visible (query, key) pair.  16,484 causal tokens of 32 heads
// of 128 take 1,912 - 2,010 us from card to card, 1,107 - 1,164 TFLOP/s, the units 60% busy at 1.76 GHz; 8,192 with all
// keys 926 - 970 (a matrix product of 8,192^3 from the library reaches 1,175: the board's power, not the instruction's
// rate, is the limit; with the MFMAs and the DMA alone the full 8,192 take 692 us).  Eight prompts of 97 to 2,309
// tokens, 104 - 120 us, keep them 38% busy at 2.0 GHz: the queries' loads and the results' stores, which nothing of the
// same workgroup runs beside, and waves that wait for their workgroup's last.
#include <type_traits>

#include "attention_ops.h"

namespace eas {
namespace {

constexpr int KT = 64;               // keys per tile
constexpr int kMaxRows = 1 << 30;    // queries or keys of a call
constexpr int MAX_RUNS = 16;         // runs that a sequence's keys are split into

// Runs of keys that each query tile of a sequence is split into, a workgroup each, where the sequence alone leaves CUs
// without one: of 4,096 keys at least, or fewer where it has less than 128 workgroups without, down to 1,024 with 32.
// A call waits for its longest walk: 128 queries over 32,896 keys of 32 heads 92 us, in one walk 472; 64 over 5,064 31
// and in runs of 4,096 79; 300 over 6,300 64 and 100; 512 over 8,704 93 and in one 138; chunks of 700 - 1,024 queries
// over 1,535 - 9,916 keys of 16 heads 102 and 124.  A batch that fills the chip anyway pays for the runs' sums: sixteen
// chunks of 64 over 8,256 keys 276, in runs of 4,096 244; eight of 512 over 9,512 keys 631, in one 570, in runs of
// 1,024 838.  By a sequence's own sizes only: the join rounds otherwise, and a result must not depend on the batch.
__host__ __device__ inline int n_runs(int lq, int lk, int heads) {
  const int64_t alone = ((int64_t)lq + 127) / 128 * heads;   // workgroups of one run
  if (alone > 256) return 1;
  const int shortest = alone <= 32 ? 1024 : alone >= 128 ? 4096 : 32 * (int)alone;
  const int runs = lk / shortest;
  return runs < 1 ? 1 : runs < MAX_RUNS ? runs : MAX_RUNS;
}

// Key tiles of each run, the last ones' fewer or none
__host__ __device__ inline int run_tiles(int lk, int runs) { return ((lk + KT - 1) / KT + runs - 1) / runs; }

// Work list: the query tiles of all sequences, a run each, those with most keys first where they are few enough to be
// listed (when they are many, what the last ones leave idle is little).
constexpr int LISTED = 768;
struct PromptWork {
  int n, listed;
  int cu_q[kMaxSeqs + 1], cu_k[kMaxSeqs + 1];
  int slot0[kMaxSeqs + 1];        // prefix sums of the split sequences' slots in the workspace, queries * heads * runs
  union {
    int tile_start[kMaxSeqs + 1];   // not listed: prefix sums of tiles * runs, each sequence's from its last on
    uint16_t tile[LISTED];          // listed: sequence | (tile * runs + run) << 6
  };
};

struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  eas_strides qs, ks, vs, os;
  int heads, group, causal, tiles;
  float scale_log2;
  float* part;       // results of runs [slots, head_dim]
  float* part_lse;   // and their softmax's log2 sums [slots]
};

template <class T>
struct Mfma;
template <>
struct Mfma<bf16> {
  typedef bf16x8 x8;
  __device__ static f32x16 go(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mfma<f16> {
  typedef f16x8 x8;
  __device__ static f32x16 go(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Key of a wave's weight v (of 32) in a tile; the other lane of the query, g ^ 1, has the others
__device__ __forceinline__ int key_of(int v, int g) { return (v >> 4) * 32 + (v & 15) / 4 * 8 + g * 4 + (v & 3); }

// The wave's queries over key tiles from .. to again, into O, m and l, in the layout that the loop leaves them in; no
// value reaches a query that does not see it.  Only for results that the loop, in which a hidden value is multiplied by
// a weight of 0, leaves infinite or NaN.  Tiles that all the wave's queries see whole go through the matrix units,
// straight from memory; at the border values are taken key by key, by the queries that see them, the weights from
// `stage`, 4 KB of LDS for each wave.  4,096 tokens of 8 heads that all come this way take 0.49 ms, without a NaN 0.084.
template <class T, int HD, class X8>
__device__ __forceinline__ void careful_rows(const X8* qf, const T* kp, long k_row, const T* vp, long v_row, int lk,
                                             int from, int to, int fewest, int sees, float scale_log2, char* stage,
                                             f32x16* o, float* m_out, float* l_out) {
  constexpr int KS = HD / 16, HB = HD / 32;
  constexpr float TOP = std::is_same_v<T, f16> ? 15.0f : 0.0f;   // log2 of the largest weight, as in the loop
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, g = lane >> 5, l32 = lane & 31;
  const f32x16 zero = {};
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) o[hb] = zero;
  for (int t = from; t < to; ++t) {
    const int k0 = t * KT;
    f32x16 s[2] = {zero, zero};
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      const long row = min(k0 + 32 * (i & 1) + l32, lk - 1);
      s[i & 1] = Mfma<T>::go(*reinterpret_cast<const X8*>(kp + row * k_row + (i >> 1) * 16 + g * 8), qf[i >> 1], s[i & 1]);
    }
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < 32; ++v) {
      float x = s[v >> 4][v & 15] * scale_log2;
      if (k0 + key_of(v, g) >= sees) x = -INFINITY;
      top = fmaxf(top, x);
      s[v >> 4][v & 15] = x;
    }
    top = fmaxf(m, fmaxf(top, __shfl_xor(top, 32, 64)));
    const float base = top == -INFINITY ? 0.0f : top, alpha = __builtin_amdgcn_exp2f(m - base);
    m = top;
    l *= alpha;
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) o[hb] *= alpha;
#pragma unroll
    for (int v = 0; v < 32; ++v) {
      const float p = __builtin_amdgcn_exp2f(s[v >> 4][v & 15] - base + TOP);
      l += p;
      s[v >> 4][v & 15] = p;
    }
    if (k0 + KT <= fewest) {
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {   // 16 keys
        X8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (T)(c == 0 ? s[0][e] : c == 1 ? s[0][8 + e] : c == 2 ? s[1][e] : s[1][8 + e]);
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
          X8 v;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = vp[(k0 + key_of(8 * c + e, g)) * v_row + hb * 32 + l32];
          o[hb] = Mfma<T>::go(v, p, o[hb]);
        }
      }
    } else {
      float* w = reinterpret_cast<float*>(stage) + l32 * 32;   // of 32 keys
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int v = 0; v < 16; ++v) w[key_of(v, g)] = s[kb][v];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
        for (int i = 0; i < 32; ++i) {
          const int key = k0 + kb * 32 + i;
          if (key < sees) {
            const float p = w[i];
#pragma unroll
            for (int hb = 0; hb < HB; ++hb)
#pragma unroll
              for (int e4 = 0; e4 < 4; ++e4) {
                const Tx4 x = *reinterpret_cast<const Tx4*>(vp + key * v_row + hb * 32 + e4 * 8 + g * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[hb][e4 * 4 + e] = fmaf(p, (float)x[e], o[hb][e4 * 4 + e]);
              }
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
  }
  *m_out = m - TOP;
  *l_out = l;
}

// Whether any of n floats is infinite or NaN in any lane
template <int N>
__device__ __forceinline__ bool any_not_finite(const f32x16* o) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(o[i][e]) & 0x7fffffffu);
  return __any(top >= 0x7f800000u);
}

#pragma clang diagnostic ignored "-Winline-asm"
// 64 lanes' 16-byte pieces at base + voff, to 1 KB of LDS in lane order
__device__ __forceinline__ void dma16(unsigned lds_addr, unsigned voff, const void* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n"
               :: "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

template <int HD, int NW_>
struct Cfg {
  static constexpr int NW = NW_;                 // waves per workgroup, 32 queries each
  static constexpr int QT = 32 * NW;             // queries per workgroup
  static constexpr int R = HD / 8;               // 16-byte chunks per row
  static constexpr int KS = HD / 16;             // 16-wide steps of q . k
  static constexpr int HB = HD / 32;             // 32-row blocks of O^T
  static constexpr int TILE = KT * HD * 2;       // bytes of a key or value tile
  static constexpr int NDMA = TILE / 1024 / NW;  // DMA instructions per wave and tile
  // Chunk L of a tile's row is stored at chunk (L + rot) % R.  A key read takes one chunk of 16 consecutive
  // rows at a time, a transposing value read 64 bytes of 4 consecutive rows: both hit all banks once.
  __device__ static int rot(int row) {
    return R == 16 ? 4 * (row & 3) + ((row >> 2) & 3) : 2 * (row & 3) + ((row >> 2) & 1);
  }
  __device__ static int phys(int row, int L) { return (L + rot(row)) % R; }
  __device__ static int logical(int row, int p) { return (p + R - rot(row)) % R; }
};

// The head and query tile of a workgroup.  Workgroups go to the 8 XCDs in turn, each with an L2 of its own, so the
// query heads of one key / value head, which read the same keys, are kept on one XCD (of 8 or more heads a whole
// number each; 1, 2 or 4 heads get 8, 4 or 2 XCDs each); other numbers are dealt out as they come.  All heads of a
// query tile, then those of the next.
__device__ __forceinline__ bool place(const PromptArgs& a, int* h, int* tile) {
  const int b = blockIdx.x, xcd = b & 7, i = b >> 3, kv_heads = a.heads / a.group;
  if (kv_heads % 8 == 0) {
    const int each = a.heads / 8;
    *h = xcd * each + i % each;
    *tile = i / each;
  } else if (8 % kv_heads == 0) {
    const int xcds = 8 / kv_heads, item = i * xcds + xcd % xcds;
    *h = xcd / xcds * a.group + item % a.group;
    *tile = item / a.group;
  } else {
    *h = b % a.heads;
    *tile = b / a.heads;
  }
  return *tile < a.tiles;
}
// Workgroups that place() spreads `tiles` tiles of all heads over
int64_t workgroups(int64_t tiles, int heads, int kv_heads) {
  if (kv_heads % 8 == 0 || 8 % kv_heads) return tiles * heads;
  const int64_t xcds = 8 / kv_heads;
  return (tiles * (heads / kv_heads) + xcds - 1) / xcds * 8;
}

template <class T, int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void prompt_kernel(PromptArgs a, PromptWork w) {
  using C = Cfg<HD, NW>;
  typedef typename Mfma<T>::x8 x8;
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // keys x 2, values x 2
  __attribute__((address_space(3))) char* lds = (__attribute__((address_space(3))) char*)smem;
  const unsigned lds0 = (unsigned)(size_t)lds;

  int h, tile;
  if (!place(a, &h, &tile)) return;
  int r = 0, item;
  if (w.listed) {
    r = w.tile[tile] & 63;
    item = w.tile[tile] >> 6;
  } else {
    while (r + 1 < w.n && w.tile_start[r + 1] <= tile) ++r;
    item = w.tile_start[r + 1] - 1 - tile;
  }
  const int lq = w.cu_q[r + 1] - w.cu_q[r], lk = w.cu_k[r + 1] - w.cu_k[r];
  const int runs = n_runs(lq, lk, a.heads), qt = item / runs, run = item % runs;
  const int q0 = qt * C::QT;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* qp = static_cast<const T*>(a.q) + w.cu_q[r] * a.qs.row + h * a.qs.head;
  const T* kp = static_cast<const T*>(a.k) + w.cu_k[r] * a.ks.row + h / a.group * a.ks.head;
  const T* vp = static_cast<const T*>(a.v) + w.cu_k[r] * a.vs.row + h / a.group * a.vs.head;

  // keys that a query sees: this lane's, the wave's fewest and most, the workgroup's most
  auto seen = [&](int q) { return a.causal ? max(0, min(lk, lk - lq + min(q, lq - 1) + 1)) : lk; };
  const int qw = q0 + wave * 32, qi = qw + l32;
  const int sees = seen(qi), fewest = seen(qw), most = qw < lq ? seen(qw + 31) : 0;
  // key tiles of the query tile, from tb on those of the run, and of these the wave's; the runs' borders go by the
  // sequence's keys alone, so that they are the same for 128 and 256 queries a workgroup
  const int all = (seen(q0 + C::QT - 1) + KT - 1) / KT, each = run_tiles(lk, runs), tb = run * each;
  const int nt = max(0, min(each, all - tb)), nt_w = max(0, min(nt, (most + KT - 1) / KT - tb));

  x8 qf[C::KS];
#pragma unroll
  for (int ks = 0; ks < C::KS; ++ks)
    qf[ks] = *reinterpret_cast<const x8*>(qp + min(qi, lq - 1) * a.qs.row + ks * 16 + g * 8);

  // a tile's DMA: instruction wave + NW j fills LDS slots (its number) * 64 + lane; slot s is chunk s % R of row s / R
  int drow[C::NDMA], dcol[C::NDMA];
#pragma unroll
  for (int j = 0; j < C::NDMA; ++j) {
    const int slot = (wave + NW * j) * 64 + lane;
    drow[j] = slot / C::R;
    dcol[j] = C::logical(drow[j], slot % C::R) * 16;
  }
  auto fetch = [&](const T* p, long stride, int t, int lds_off) {
    const int left = lk - 1 - (tb + t) * KT;   // rows behind the last key read it again
    const T* base = p + (long)(tb + t) * KT * stride;
#pragma unroll
    for (int j = 0; j < C::NDMA; ++j)
      dma16(lds0 + lds_off + (wave + NW * j) * 1024, (unsigned)min(drow[j], left) * (unsigned)(stride * 2) + dcol[j],
            base);
  };
  auto fetch_k = [&](int t) { fetch(kp, a.ks.row, t, (t & 1) * C::TILE); };
  auto fetch_v = [&](int t) { fetch(vp, a.vs.row, t, (2 + (t & 1)) * C::TILE); };

  int kofs[C::KS];
#pragma unroll
  for (int ks = 0; ks < C::KS; ++ks) kofs[ks] = l32 * HD * 2 + C::phys(l32, 2 * ks + g) * 16;
  // V^T operand: lane 16 q + 4 e + t reads row 16 (..) + 8 half + 4 g + e, columns 32 hb + 16 (q % 2) + 4 t .. + 4
  int vofs[C::HB][2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = 8 * half + 4 * g + ((lane >> 2) & 3);
#pragma unroll
    for (int hb = 0; hb < C::HB; ++hb) {
      const int col = hb * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      vofs[hb][half] = row * HD * 2 + C::phys(row, col >> 3) * 16 + (col & 7) * 2;
    }
  }

  f32x16 o[C::HB];
#pragma unroll
  for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[hb][e] = 0.0f;
  float m = 0.0f, l = 0.0f;
  bool unset = true;   // no score above -inf yet; the same in both lanes of a query, as m is

  constexpr int NK = 2 * C::KS, NV = 4 * C::HB;   // MFMAs of a tile's scores, and of its products with the values
  // A operand of score MFMA i: keys 32 (i % 2) .. of k-step i / 2; of value MFMA j: block j % HB, keys 16 (j / HB) ..
  const auto read_k = [&](int t, int i) {
    return *reinterpret_cast<const x8*>(smem + (t & 1) * C::TILE + (i & 1) * 32 * HD * 2 + kofs[i >> 1]);
  };
  const auto read_v = [&](int t, int j) {
    union { x8 v; v4i16 h[2]; } u;
#pragma unroll
    for (int half = 0; half < 2; ++half)
      u.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_v4i16*)(lds + (2 + (t & 1)) * C::TILE + j / C::HB * 16 * HD * 2 + vofs[j % C::HB][half]));
    return u.v;
  };
  const f32x16 zero = {};
  constexpr float TOP = std::is_same_v<T, f16> ? 15.0f : 0.0f;
  // The scores of tile t, keys 32 .. in s[1].
  const auto scores = [&](int t, f32x16* s) {
#pragma unroll
    for (int i = 0; i < NK; ++i)
      s[i & 1] = Mfma<T>::go(read_k(t, i), qf[i >> 1], i < 2 ? zero : s[i & 1]);
  };
  // Tile t: the online softmax of its scores s and O^T += V^T P^T, and beside them the next tile's scores n.  One
  // FMA turns a score into x = s c - m, in log2 units over m, the maximum less TOP - 8.  m is raised lazily, when some
  // x exceeds TOP, so p = 2^x <= 2^TOP and O is rarely scaled; O and l share m, so O / l is the same.  The first score
  // above -inf sets it, in whichever tile that is: until then O and l are 0.  TOP keeps bf16's sums from overflow where
  // a softmax's do not, and fp16's small weights from vanishing: what is lost below 2^-24 is 2^-32 of the largest
  // weight.  The matrix unit takes 32 cycles an MFMA, in which the wave issues some 8 other instructions: the softmax's
  // are dealt out behind the MFMAs by hand, in steps that nothing is moved across, each with the operands of the MFMA
  // four steps on.  (Left to the compiler they come in blocks, and both waves of a SIMD wait for the same unit: 8,192
  // tokens with all keys 942 us, so 897.)
  const auto step = [&](int t, f32x16* s, f32x16* n, auto masked, auto next) {
    constexpr bool MASKED = decltype(masked)::value, NEXT = decltype(next)::value;
    const int k0 = (tb + t) * KT;
    x8 kf[4], vf[4], p[4];
    if constexpr (NEXT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) kf[i] = read_k(t + 1, i);
    }
    float mx = -INFINITY;
    constexpr int H = NK / 2, E = 32 / H;   // steps of the first part, and scores of each
#pragma unroll
    for (int i = 0; i < H; ++i) {
      if constexpr (NEXT) {
        n[i & 1] = Mfma<T>::go(kf[i & 3], qf[i >> 1], i < 2 ? zero : n[i & 1]);
        kf[i & 3] = read_k(t + 1, i + 4);
      }
#pragma unroll
      for (int v = E * i; v < E * i + E; ++v) {
        float x = fmaf(s[v >> 4][v & 15], a.scale_log2, -m);
        if (MASKED && k0 + (v >> 4) * 32 + (v & 15) / 4 * 8 + g * 4 + (v & 3) >= sees) x = -INFINITY;
        mx = fmaxf(mx, x);
        s[v >> 4][v & 15] = x;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    {   // the query's other half of the keys is in lane ^ 32
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    }
    const bool need = mx > (unset ? -INFINITY : TOP);   // a query that sees nothing keeps m = 0, l = 0
    if (__any(need)) {
      const float d = need ? mx - (TOP - 8.0f) : 0.0f;
      const float alpha = unset ? 0.0f : __builtin_amdgcn_exp2f(-d);
      unset = unset && !need;
      m += d;
      l *= alpha;
#pragma unroll
      for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[hb][e] *= alpha;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] -= d;
    }
    float sum[4];
    const auto weigh = [&](int v) {
      const float x = __builtin_amdgcn_exp2f(s[v >> 4][v & 15]);
      sum[v >> 3] = v & 7 ? sum[v >> 3] + x : x;
      p[v >> 3][v & 7] = (T)x;
    };
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!NEXT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) vf[i] = read_v(t, i);
    }
    constexpr int W = 16 / H;   // weights of the first 32 keys, a step
#pragma unroll
    for (int i = H; i < NK; ++i) {
      if constexpr (NEXT) {
        n[i & 1] = Mfma<T>::go(kf[i & 3], qf[i >> 1], n[i & 1]);
        if (i + 4 < NK)
          kf[i & 3] = read_k(t + 1, i + 4);
        else
          vf[i + 4 - NK] = read_v(t, i + 4 - NK);
      }
#pragma unroll
      for (int v = W * (i - H); v < W * (i - H) + W; ++v) weigh(v);
      __builtin_amdgcn_sched_barrier(0);
    }
    constexpr int Y = 32 / NV;   // of the others, beside the products with the first half's values
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      o[j % C::HB] = Mfma<T>::go(vf[j & 3], p[j / C::HB], o[j % C::HB]);
      if (j + 4 < NV) vf[j & 3] = read_v(t, j + 4);
      if (j < NV / 2)
#pragma unroll
        for (int v = 16 + Y * j; v < 16 + Y * j + Y; ++v) weigh(v);
      __builtin_amdgcn_sched_barrier(0);
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  constexpr std::integral_constant<bool, true> yes{};
  constexpr std::integral_constant<bool, false> no{};
  // Waits until the wave's own DMA has landed and its LDS reads are done, and for the other waves to be as far.  One
  // asm: no read may move up between the wait and the barrier.  Every wave passes it once a tile, from whichever of
  // the loops below it is in.
  const auto meet = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  const auto arrive = [&](int t) {
    meet();   // keys t + 1 and values t are there, keys t and values t - 1 read by all
    if (t + 2 < nt) fetch_k(t + 2);
    if (t + 1 < nt) fetch_v(t + 1);
  };
  if (nt > 0) {
    f32x16 sa[2], sb[2];
    fetch_k(0);
    fetch_v(0);
    if (nt > 1) fetch_k(1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // the queries, whose loads are in flight with the first tiles', are taken here, so that no wait for them is
    // left to the loop, where it would wait for a tile
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) asm volatile("" ::"v"(qf[ks]));
    meet();
    int t = 0;
    if (nt_w > 0) {
      scores(0, sa);
      // tiles that all the wave's queries see whole, in pairs; those at the border; the last one
      for (const int whole = min(fewest / KT - tb, nt_w - 1); t + 2 <= whole; t += 2) {
        arrive(t);
        step(t, sa, sb, no, yes);
        arrive(t + 1);
        step(t + 1, sb, sa, no, yes);
      }
      for (; t + 1 < nt_w; ++t) {
        arrive(t);
        step(t, sa, sb, yes, yes);
        sa[0] = sb[0];
        sa[1] = sb[1];
      }
      arrive(t);
      step(t, sa, sb, yes, no);
      ++t;
    }
    for (; t < nt; ++t) arrive(t);
  }

  // every wave is past its last read
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();
  if (qw >= lq) return;
  char* stage = smem + wave * 32 * HD * 2;
  if (a.causal && any_not_finite<C::HB>(o))
    careful_rows<T, HD>(qf, kp, a.ks.row, vp, a.vs.row, lk, tb, tb + nt_w, fewest, sees, a.scale_log2, stage, o, &m, &l);
  l += __shfl_xor(l, 32, 64);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l, lse2 = l == 0.0f ? -INFINITY : m + __log2f(l);
  if (runs > 1) {
    const long slot = w.slot0[r] + ((long)run * a.heads + h) * lq + qi;   // [run, head, query]: a wave's are consecutive
    if (qi < lq) {
#pragma unroll
      for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<float4*>(a.part + slot * HD + hb * 32 + e * 2 + g * 4) =
              make_float4(o[hb][e] * inv, o[hb][e + 1] * inv, o[hb][e + 2] * inv, o[hb][e + 3] * inv);
      if (g == 0) a.part_lse[slot] = lse2;
    }
    return;
  }
  if (a.lse && g == 0 && qi < lq) a.lse[((long)w.cu_q[r] + qi) * a.heads + h] = lse2 * kLn2;
  T* out = static_cast<T*>(a.out) + w.cu_q[r] * a.os.row + h * a.os.head;   // of the sequence's first query
  // the tiles' memory stages each wave's 32 x HD results, chunks of row r rotated by r, so that the stores are of
  // whole rows
#pragma unroll
  for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      union { uint2 u; T e[4]; } st;
#pragma unroll
      for (int e = 0; e < 4; ++e) st.e[e] = (T)(o[hb][e4 * 4 + e] * inv);
      *reinterpret_cast<uint2*>(stage + l32 * HD * 2 + (hb * 4 + e4 + l32) % C::R * 16 + g * 8) = st.u;
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int k = 0; k < C::R / 2; ++k) {
    const int c = lane + 64 * k, row = c / C::R, ch = c % C::R;
    const uint4 x = *reinterpret_cast<const uint4*>(stage + row * HD * 2 + (ch + row) % C::R * 16);
    if (qw + row < lq) *reinterpret_cast<uint4*>(out + (qw + row) * a.os.row + ch * 8) = x;
  }
}

// Joins the runs of the split sequences, in order.
struct JoinWork {
  int n;
  int seq[kMaxSeqs], row0[kMaxSeqs + 1];   // split sequences, prefix sums of their queries
};
template <class T, int HD>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a, PromptWork w, JoinWork j) {
  constexpr int ROWS = 256 / (HD / 4);   // queries of a workgroup, a thread 4 dimensions; a run's of a head lie together
  const int row = blockIdx.x * ROWS + threadIdx.x / (HD / 4), h = blockIdx.y, d = threadIdx.x % (HD / 4) * 4;
  if (row >= j.row0[j.n]) return;
  int s = 0;
  while (j.row0[s + 1] <= row) ++s;
  const int r = j.seq[s], i = row - j.row0[s];
  const int lq = w.cu_q[r + 1] - w.cu_q[r], runs = n_runs(lq, w.cu_k[r + 1] - w.cu_k[r], a.heads);
  const long slot = w.slot0[r] + (long)h * lq + i, step = (long)a.heads * lq;   // of run 0, and from run to run
  float M = -INFINITY;
  for (int k = 0; k < runs; ++k) M = fmaxf(M, a.part_lse[slot + k * step]);
  const float base = M == -INFINITY ? 0.0f : M;
  float W = 0.0f;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int k = 0; k < runs; ++k) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + (slot + k * step) * HD + d);
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
  *reinterpret_cast<Tx4*>(static_cast<T*>(a.out) + (w.cu_q[r] + i) * a.os.row + h * a.os.head + d) = y;
  if (d == 0 && a.lse) a.lse[(long)(w.cu_q[r] + i) * a.heads + h] = W == 0.0f ? -INFINITY : (M + __log2f(W)) * kLn2;
}

template <class T, int HD, int NW>
eas_status launch(const PromptArgs& a, const PromptWork& w, unsigned grid, hipStream_t s) {
  constexpr int lds = 4 * Cfg<HD, NW>::TILE;
  hipLaunchKernelGGL((prompt_kernel<T, HD, NW>), dim3(grid), dim3(64 * NW), lds, s, a, w);
  return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
}

// Key tiles that query tile t of a sequence walks
int64_t key_tiles(int64_t lq, int64_t lk, int64_t t, int qt, int causal) {
  const int64_t last = (t + 1) * qt < lq ? (t + 1) * qt : lq;
  const int64_t keys = causal ? (last + lk - lq < 0 ? 0 : last + lk - lq) : lk;
  return (keys + KT - 1) / KT;
}

// Queries per workgroup.  256 share each key and value tile among twice the queries, which halves the DMA per score:
// 2-5% faster where both fill the chip (16,484 causal tokens of 32 heads 1,917 us against 1,966; 8,192 full 927
// against 975).  128 leave less of a workgroup idle behind a sequence's end and at the diagonal, spread few queries
// over more CUs, and put two workgroups on a CU, one's loads and stores beside the other's products: eight image
// prompts of 97 to 2,309 tokens 119 us against 125, 64 prompts of 256 106 against 123.  So 256 where they
// take at most 8% more key tiles per query, walk 16 at least, and two workgroups a CU remain.  A query's arithmetic
// is the same in both.
int query_tile(const PromptWork& w, int heads, int causal) {
  int64_t cost[2] = {}, tiles = 0;
  for (int big = 0; big < 2; ++big)
    for (int r = 0; r < w.n; ++r) {
      const int64_t lq = (int64_t)w.cu_q[r + 1] - w.cu_q[r], lk = (int64_t)w.cu_k[r + 1] - w.cu_k[r];
      const int qt = big ? 256 : 128;
      const int64_t n = (lq + qt - 1) / qt;
      // twice the key tiles of all: of the first and the last, as they grow evenly
      cost[big] += n ? (key_tiles(lq, lk, 0, qt, causal) + key_tiles(lq, lk, n - 1, qt, causal)) * n : 0;
      if (big) tiles += n;
    }
  return 2 * cost[1] * 100 <= cost[0] * 108 && cost[1] >= 32 * tiles && tiles * heads >= 2l * device_cus() ? 256 : 128;
}

// Fills the work list for tiles of qt queries; their number, one for each run.
int64_t list_tiles(PromptWork* w, int heads, int qt, int causal) {
  const auto queries = [&](int r) { return (int64_t)w->cu_q[r + 1] - w->cu_q[r]; };
  const auto keys = [&](int r) { return (int64_t)w->cu_k[r + 1] - w->cu_k[r]; };
  const auto runs = [&](int r) { return n_runs((int)queries(r), (int)keys(r), heads); };
  int64_t tiles = 0, most = 0;
  for (int r = 0; r < w->n; ++r) {
    tiles += (queries(r) + qt - 1) / qt * runs(r);
    most = keys(r) > most ? keys(r) : most;
  }
  w->listed = tiles <= LISTED;
  if (!w->listed) {
    int64_t at = 0;
    for (int r = 0; r < w->n; ++r) {
      w->tile_start[r] = (int)at;
      at += (queries(r) + qt - 1) / qt * runs(r);
    }
    w->tile_start[w->n] = (int)at;
    return tiles;
  }
  // sorted by key tiles into 128 classes, most first
  constexpr int CLASSES = 128;
  int at[CLASSES + 1] = {};
  const int64_t top = (most + KT - 1) / KT + 1;
  const auto every = [&](auto&& f) {
    for (int r = 0; r < w->n; ++r)
      for (int64_t t = 0; t * qt < queries(r); ++t) {
        const int n = runs(r);
        const int64_t walk = key_tiles(queries(r), keys(r), t, qt, causal), each = run_tiles((int)keys(r), n);
        for (int k = 0; k < n; ++k) {
          const int64_t left = walk - k * each, own = left < 0 ? 0 : left < each ? left : each;
          f(r, (int)t * n + k, (int)(CLASSES - 1 - own * CLASSES / top));
        }
      }
  };
  every([&](int, int, int c) { ++at[c + 1]; });
  for (int c = 0; c < CLASSES; ++c) at[c + 1] += at[c];
  every([&](int r, int t, int c) { w->tile[at[c]++] = (uint16_t)(r | t << 6); });
  return tiles;
}

// The sequences, their slots in the workspace, and those that are split
void fill_work(PromptWork* w, JoinWork* j, const int32_t* cu_q, const int32_t* cu_k, int32_t n, int heads) {
  w->n = n;
  j->n = 0;
  int slots = 0, rows = 0;   // at most 64 * 256 * 128 * MAX_RUNS slots
  for (int r = 0; r <= n; ++r) {
    w->cu_q[r] = cu_q[r], w->cu_k[r] = cu_k[r];
    w->slot0[r] = slots;
    if (r == n) break;
    const int lq = cu_q[r + 1] - cu_q[r], runs = n_runs(lq, cu_k[r + 1] - cu_k[r], heads);
    if (runs == 1 || lq == 0) continue;
    slots += lq * heads * runs;
    j->seq[j->n] = r;
    j->row0[j->n++] = rows;
    rows += lq;
  }
  j->row0[j->n] = rows;
}

template <class T, int HD>
eas_status launch_all(const eas_attn_shape* shape, PromptArgs a, PromptWork* w, const JoinWork& j, hipStream_t s) {
  const int qt = query_tile(*w, shape->heads, shape->causal);
  const int64_t tiles = list_tiles(w, shape->heads, qt, shape->causal);
  const int64_t blocks = workgroups(tiles, shape->heads, shape->kv_heads);
  if (!fits_launch(blocks, 2 * qt)) return EAS_ERR_UNSUPPORTED;   // a wave for 32 queries
  a.tiles = (int)tiles;
  const eas_status st = qt == 256 ? launch<T, HD, 8>(a, *w, (unsigned)blocks, s)
                                  : launch<T, HD, 4>(a, *w, (unsigned)blocks, s);
  if (st != EAS_OK || !j.n) return st;
  constexpr int each = 256 / (HD / 4);
  const dim3 grid((unsigned)((j.row0[j.n] + each - 1) / each), (unsigned)shape->heads);
  hipLaunchKernelGGL((prompt_join_kernel<T, HD>), grid, dim3(256), 0, s, a, *w, j);
  return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
}

eas_status check_cu(const int32_t* cu, int32_t n) {
  if (cu[0] != 0) return EAS_ERR_SHAPE;
  for (int r = 0; r < n; ++r)
    if (cu[r + 1] < cu[r]) return EAS_ERR_SHAPE;
  return EAS_OK;
}

}  // namespace
}  // namespace eas

using namespace eas;

namespace {
// What both calls refuse; *work and *join are filled
eas_status check_call(const eas_attn_shape* shape, const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs,
                      PromptWork* work, JoinWork* join) {
  eas_status st = check_shape(shape);
  if (st != EAS_OK) return st;
  if (!cu_q) return EAS_ERR_INVALID_ARG;
  if (n_seqs < 0 || n_seqs > EAS_MAX_SEQS) return EAS_ERR_CAPACITY;
  if (!cu_k) cu_k = cu_q;
  st = check_cu(cu_q, n_seqs);
  if (st == EAS_OK) st = check_cu(cu_k, n_seqs);
  if (st != EAS_OK) return st;
  if (cu_q[n_seqs] > kMaxRows || cu_k[n_seqs] > kMaxRows) return EAS_ERR_UNSUPPORTED;
  fill_work(work, join, cu_q, cu_k, n_seqs, shape->heads);
  return EAS_OK;
}
int64_t workspace_bytes_of(const PromptWork& w, int head_dim) { return (int64_t)w.slot0[w.n] * (head_dim + 1) * 4; }
}  // namespace

extern "C" eas_status eas_prompt_attention_workspace(const eas_attn_shape* shape, const int32_t* cu_q,
                                                     const int32_t* cu_k, int32_t n_seqs, int64_t* bytes) {
  PromptWork w;
  JoinWork j;
  const eas_status st = check_call(shape, cu_q, cu_k, n_seqs, &w, &j);
  if (st != EAS_OK) return st;
  if (!bytes) return EAS_ERR_INVALID_ARG;
  *bytes = workspace_bytes_of(w, shape->head_dim);
  return EAS_OK;
}

extern "C" eas_status eas_prompt_attention(const eas_attn_shape* shape, const void* q, const void* k, const void* v,
                                           const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs, void* out,
                                           float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  PromptWork w;
  JoinWork j;
  eas_status st = check_call(shape, cu_q, cu_k, n_seqs, &w, &j);
  if (st == EAS_OK) st = check_strides(shape->q);
  if (st == EAS_OK) st = check_strides(shape->k);
  if (st == EAS_OK) st = check_strides(shape->v);
  if (st == EAS_OK) st = check_out_strides(shape->out, cu_q[n_seqs], shape->heads, shape->head_dim);
  if (st != EAS_OK) return st;
  if (cu_q[n_seqs] == 0) return EAS_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out) || (uintptr_t)lse % 4) return EAS_ERR_INVALID_ARG;
  if (w.cu_k[n_seqs] > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return EAS_ERR_INVALID_ARG;
  if (j.n && (!workspace || !aligned16(workspace))) return EAS_ERR_INVALID_ARG;
  if (j.n && workspace_bytes < workspace_bytes_of(w, shape->head_dim)) return EAS_ERR_CAPACITY;

  float* part = static_cast<float*>(workspace);
  const PromptArgs a = {q, k, v, out, lse, shape->q, shape->k, shape->v, shape->out, shape->heads,
                        shape->heads / shape->kv_heads, shape->causal, 0, shape->scale * kLog2e, part,
                        j.n ? part + (int64_t)w.slot0[n_seqs] * shape->head_dim : nullptr};
#define EAS_PROMPT_CASE(DT, T, D) \
  if (shape->dtype == DT && shape->head_dim == D) return launch_all<T, D>(shape, a, &w, j, (hipStream_t)stream)
  EAS_PROMPT_CASE(EAS_BF16, bf16, 64);
  EAS_PROMPT_CASE(EAS_BF16, bf16, 128);
  EAS_PROMPT_CASE(EAS_FP16, f16, 64);
  EAS_PROMPT_CASE(EAS_FP16, f16, 128);
#undef EAS_PROMPT_CASE
  return EAS_ERR_UNSUPPORTED;
}
