// The walk over tiles of 64 keys that prompt attention and the chunks over the paged cache share: a wave's 32 rows --
// queries of one head, or queries and heads of a group -- against keys and values that stand in LDS.
#pragma once

#include <type_traits>

#include "attention_ops.h"

namespace eas {

constexpr int KT = 64;               // keys per tile

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

template <class T>
constexpr float careful_lift = std::is_same_v<T, f16> ? 1.0f : 0x1p30f;

// The wave's queries over key tiles from .. to again, into O, m and l, in the layout that the loop leaves them in; no
// value reaches a query that does not see it.  Only for results that the loop, in which a hidden value is multiplied by
// a weight of 0, leaves infinite or NaN.  Tiles that all the wave's queries see whole go through the matrix units,
// straight from memory; at the border values are taken key by key, by the queries that see them, the weights from
// `stage`, 4 KB of LDS for each wave.  4,096 tokens of 8 heads that all come this way take 0.49 ms, without a NaN 0.084.
// bf16's values may also be finite and the loop's sums of them not: here their weights, and with them O and l, are taken by
// 1 / careful_lift, 2^-30 (2^30 keys at most), exactly but for those below 2^-96 of the largest.
// key_at(i), value_at(i): key and value i; hidden(i): whether the lane's query does not see key i; whole(t): whether all
// the wave's queries see all of tile t.
template <class T, int HD, class X8, class Key, class Value, class Hidden, class Whole>
__device__ __forceinline__ void careful_rows(const X8* qf, const Key& key_at, const Value& value_at, const Hidden& hidden,
                                             const Whole& whole, int lk, int from, int to, float scale_log2, char* stage,
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
      s[i & 1] = Mfma<T>::go(*reinterpret_cast<const X8*>(key_at(row) + (i >> 1) * 16 + g * 8), qf[i >> 1], s[i & 1]);
    }
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < 32; ++v) {
      float x = s[v >> 4][v & 15] * scale_log2;
      if (hidden(k0 + key_of(v, g))) x = -INFINITY;
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
      const float p = __builtin_amdgcn_exp2f(s[v >> 4][v & 15] - base + TOP) * (1.0f / careful_lift<T>);
      l += p;
      s[v >> 4][v & 15] = p;
    }
    if (whole(t)) {
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {   // 16 keys
        X8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (T)(c == 0 ? s[0][e] : c == 1 ? s[0][8 + e] : c == 2 ? s[1][e] : s[1][8 + e]);
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
          X8 v;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = value_at(k0 + key_of(8 * c + e, g))[hb * 32 + l32];
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
          if (!hidden(key)) {
            const float p = w[i];
#pragma unroll
            for (int hb = 0; hb < HB; ++hb)
#pragma unroll
              for (int e4 = 0; e4 < 4; ++e4) {
                const Tx4 x = *reinterpret_cast<const Tx4*>(value_at(key) + hb * 32 + e4 * 8 + g * 4);
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
// 64 lanes' 16-byte pieces at base + voff, to 1 KB of LDS in lane order.  A base that comes from a vector instruction
// (READLANE) may be read by a memory instruction five wait states after it was written; the compiler, which keeps that
// for its own instructions, does not see one in here.
template <bool READLANE = false>
__device__ __forceinline__ void dma16(unsigned lds_addr, unsigned voff, const void* base) {
  if constexpr (READLANE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2\n"
                 :: "s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
  else
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


// The head and tile of workgroup b.  Workgroups go to the 8 XCDs in turn, each with an L2 of its own, so the heads of one
// key / value head, which read the same keys, are kept on one XCD (of 8 or more key / value heads a whole number each; 1,
// 2 or 4 get 8, 4 or 2 XCDs each); other numbers are dealt out as they come.  All heads of a tile, then those of the next.
__device__ __forceinline__ void place(int b, int heads, int kv_heads, int* h, int* tile) {
  const int xcd = b & 7, i = b >> 3;
  if (kv_heads % 8 == 0) {
    const int each = heads / 8;
    *h = xcd * each + i % each;
    *tile = i / each;
  } else if (8 % kv_heads == 0) {
    const int group = heads / kv_heads, xcds = 8 / kv_heads, item = i * xcds + xcd % xcds;
    *h = xcd / xcds * group + item % group;
    *tile = item / group;
  } else {
    *h = b % heads;
    *tile = b / heads;
  }
}
// Workgroups that place() spreads `tiles` tiles of all heads over
inline int64_t tile_workgroups(int64_t tiles, int heads, int kv_heads) {
  if (kv_heads % 8 == 0 || 8 % kv_heads) return tiles * heads;
  const int64_t xcds = 8 / kv_heads;
  return (tiles * (heads / kv_heads) + xcds - 1) / xcds * 8;
}

// A wave's walk.  Keys of tile t stand in LDS tile t % 2, values in 2 + t % 2, chunks of a row as Cfg says.
template <class T, int HD, int NW>
struct TileWalk {
  using C = Cfg<HD, NW>;
  typedef typename Mfma<T>::x8 x8;
  const char* smem;
  __attribute__((address_space(3))) char* lds;
  const x8* qf;        // the wave's rows
  float scale_log2;
  int g, kofs[C::KS], vofs[C::HB][2];
  f32x16 o[C::HB];     // O^T
  float m, l;          // this lane's share of the sum l
  bool unset;          // no score above -inf yet; the same in both lanes of a query, as m is

  __device__ __forceinline__ TileWalk(char* smem_, const x8* qf_, float scale_log2_)
      : smem(smem_), lds((__attribute__((address_space(3))) char*)smem_), qf(qf_), scale_log2(scale_log2_) {
    const int lane = threadIdx.x & 63, l32 = lane & 31;
    g = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) kofs[ks] = l32 * HD * 2 + C::phys(l32, 2 * ks + g) * 16;
    // V^T operand: lane 16 q + 4 e + t reads row 16 (..) + 8 half + 4 g + e, columns 32 hb + 16 (q % 2) + 4 t .. + 4
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = 8 * half + 4 * g + ((lane >> 2) & 3);
#pragma unroll
      for (int hb = 0; hb < C::HB; ++hb) {
        const int col = hb * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        vofs[hb][half] = row * HD * 2 + C::phys(row, col >> 3) * 16 + (col & 7) * 2;
      }
    }
#pragma unroll
    for (int hb = 0; hb < C::HB; ++hb)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[hb][e] = 0.0f;
    m = 0.0f, l = 0.0f;
    unset = true;
  }

  static constexpr int NK = 2 * C::KS, NV = 4 * C::HB;   // MFMAs of a tile's scores, and of its products with the values
  // A operand of score MFMA i: keys 32 (i % 2) .. of k-step i / 2; of value MFMA j: block j % HB, keys 16 (j / HB) ..
  __device__ __forceinline__ x8 read_k(int t, int i) const {
    return *reinterpret_cast<const x8*>(smem + (t & 1) * C::TILE + (i & 1) * 32 * HD * 2 + kofs[i >> 1]);
  }
  __device__ __forceinline__ x8 read_v(int t, int j) const {
    union { x8 v; v4i16 h[2]; } u;
#pragma unroll
    for (int half = 0; half < 2; ++half)
      u.h[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_v4i16*)(lds + (2 + (t & 1)) * C::TILE + j / C::HB * 16 * HD * 2 + vofs[j % C::HB][half]));
    return u.v;
  }
  static constexpr float TOP = std::is_same_v<T, f16> ? 15.0f : 0.0f;
  // The scores of tile t, keys 32 .. in s[1].
  __device__ __forceinline__ void scores(int t, f32x16* s) const {
    const f32x16 zero = {};
#pragma unroll
    for (int i = 0; i < NK; ++i)
      s[i & 1] = Mfma<T>::go(read_k(t, i), qf[i >> 1], i < 2 ? zero : s[i & 1]);
  }
  // Tile t: the online softmax of its scores s and O^T += V^T P^T, and beside them the next tile's scores n; hidden(v):
  // whether the lane's query does not see the key of weight v (key_of), asked where Masked.  One
  // FMA turns a score into x = s c - m, in log2 units over m, the maximum less TOP - 8.  m is raised lazily, when some
  // x exceeds TOP, so p = 2^x <= 2^TOP and O is rarely scaled; O and l share m, so O / l is the same.  The first score
  // above -inf sets it, in whichever tile that is: until then O and l are 0.  TOP keeps bf16's sums from overflow where
  // a softmax's do not, and fp16's small weights from vanishing: what is lost below 2^-24 is 2^-32 of the largest
  // weight.  The matrix unit takes 32 cycles an MFMA, in which the wave issues some 8 other instructions: the softmax's
  // are dealt out behind the MFMAs by hand, in steps that nothing is moved across, each with the operands of the MFMA
  // four steps on.  (Left to the compiler they come in blocks, and both waves of a SIMD wait for the same unit: 8,192
  // tokens with all keys 942 us, so 897.)
  template <class Hidden, class Masked, class Next>
  __device__ __forceinline__ void step(int t, f32x16* s, f32x16* n, const Hidden& hidden, Masked, Next) {
    constexpr bool MASKED = Masked::value, NEXT = Next::value;
    const f32x16 zero = {};
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
        float x = fmaf(s[v >> 4][v & 15], scale_log2, -m);
        if (MASKED && hidden(v)) x = -INFINITY;
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
  }
};

}  // namespace eas
