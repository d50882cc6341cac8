// Attention over packed prompts, causal or full, with grouped heads
// (include/eas_attention.h).
//
// One pass over the keys with the running maximum and sum of the softmax.  A
// workgroup of 4 waves owns 128 queries of one (sequence, head), each wave 32 of
// them; keys and values stream through LDS in tiles of 64, anchored at the sequence's
// first key, so a query's result does not depend on where its sequence lies.
//   S^T = K Q^T (v_mfma_f32_32x32x16: keys are rows, so a lane holds 16 scores of one
//   query), softmax in fp32 on exp2, O^T += V^T P^T with P rounded to the element type.
// Bound by the matrix units: 4 * head_dim flops for each visible (query, key) pair.
#include "attention_ops.h"

namespace eas {
namespace {

constexpr int QT = 128;   // queries per workgroup
constexpr int KT = 64;    // keys per tile

// Work list: the query tiles of all sequences.
struct PromptWork {
  int n;
  int cu_q[kMaxSeqs + 1], cu_k[kMaxSeqs + 1];
  int order[kMaxSeqs];           // order[i]: sequence of the i-th group of tiles
  int tile_start[kMaxSeqs + 1];  // prefix sums of query tiles over `order`
};

struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  eas_strides qs, ks, vs, os;
  int heads, group, causal;
  float scale_log2;
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

// Queries first .. first + 32 of a sequence by one wave, query by query and key by key, a lane holding HD / 64
// dimensions: touches no key or value that a query does not see.  Only for results that the tiled products, in
// which a hidden value is multiplied by a weight of 0, leave infinite or NaN.
template <class T, int HD>
__device__ void careful_rows(const PromptArgs& a, const T* qp, const T* kp, const T* vp, int lq, int lk, int first,
                             T* out, float* lse) {
  constexpr int E = HD / 64;
  const int d = (threadIdx.x & 63) * E;
  for (int i = first; i < min(first + 32, lq); ++i) {
    const int sees = a.causal ? max(0, min(lk, i + lk - lq + 1)) : lk;
    float q[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = (float)qp[i * a.qs.row + d + e], o[e] = 0.0f;
    for (int j = 0; j < sees; ++j) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) s = fmaf(q[e], (float)kp[j * a.ks.row + d + e], s);
      s = wave_sum(s) * a.scale_log2;
      const float top = s > m ? s : m, base = top == -INFINITY ? 0.0f : top;
      const float alpha = __builtin_amdgcn_exp2f(m - base), p = __builtin_amdgcn_exp2f(s - base);
      m = top;
      l = fmaf(l, alpha, p);
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], alpha, p * (float)vp[j * a.vs.row + d + e]);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) out[i * a.os.row + d + e] = (T)(o[e] * inv);
    if (lse && d == 0) lse[(long)i * a.heads] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
  }
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

template <class T, int HD>
__global__ __launch_bounds__(256) void prompt_kernel(PromptArgs a, PromptWork w) {
  typedef typename Mfma<T>::x8 x8;
  constexpr int KS = HD / 16;      // 16-wide steps of q . k
  constexpr int HB = HD / 32;      // 32-row blocks of O^T
  constexpr int LDK = HD + 8;      // row stride of the key tile
  constexpr int LDV = KT + 4;      // row stride of the transposed value tile
  __shared__ __attribute__((aligned(16))) T Ks[KT * LDK];
  __shared__ __attribute__((aligned(16))) T Vt[HD * LDV];

  const int h = blockIdx.x % a.heads, tile = blockIdx.x / a.heads;
  int i = 0;
  while (i + 1 < w.n && w.tile_start[i + 1] <= tile) ++i;
  const int r = w.order[i];
  const int lq = w.cu_q[r + 1] - w.cu_q[r], lk = w.cu_k[r + 1] - w.cu_k[r];
  const int q0 = (tile - w.tile_start[i]) * QT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, l32 = lane & 31;
  const T* qp = static_cast<const T*>(a.q) + w.cu_q[r] * a.qs.row + h * a.qs.head;
  const T* kp = static_cast<const T*>(a.k) + w.cu_k[r] * a.ks.row + h / a.group * a.ks.head;
  const T* vp = static_cast<const T*>(a.v) + w.cu_k[r] * a.vs.row + h / a.group * a.vs.head;

  const int qi = q0 + wave * 32 + l32;   // this lane's query; past the end it is computed, not stored
  const int qr = min(qi, lq - 1);
  const int sees = a.causal ? max(0, min(lk, qr + lk - lq + 1)) : lk;
  const int most = a.causal ? max(0, min(lk, min(q0 + QT, lq) + lk - lq)) : lk;   // over the workgroup
  x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const x8*>(qp + qr * a.qs.row + ks * 16 + g * 8);

  f32x16 o[HB];
#pragma unroll
  for (int hb = 0; hb < HB; ++hb)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[hb][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  for (int k0 = 0; k0 < most; k0 += KT) {
    __syncthreads();
    for (int c = tid; c < KT * (HD / 8); c += 256) {
      const int key = c / (HD / 8), d = c % (HD / 8) * 8;
      uint4 x = make_uint4(0, 0, 0, 0);
      if (k0 + key < lk) x = *reinterpret_cast<const uint4*>(kp + (k0 + key) * a.ks.row + d);
      *reinterpret_cast<uint4*>(Ks + key * LDK + d) = x;
    }
    for (int c = tid; c < KT * (HD / 8); c += 256) {
      const int key = c % KT, d = c / KT * 8;
      union { uint4 u; T e[8]; } x;
      x.u = make_uint4(0, 0, 0, 0);   // values behind the last key may be anything, and 0 * NaN is NaN
      if (k0 + key < lk) x.u = *reinterpret_cast<const uint4*>(vp + (k0 + key) * a.vs.row + d);
#pragma unroll
      for (int e = 0; e < 8; ++e) Vt[(d + e) * LDV + key] = x.e[e];
    }
    __syncthreads();

    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kb][e] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const x8 kf = *reinterpret_cast<const x8*>(Ks + (kb * 32 + l32) * LDK + ks * 16 + g * 8);
        s[kb] = Mfma<T>::go(kf, qf[ks], s[kb]);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = k0 + kb * 32 + (e >> 2) * 8 + g * 4 + (e & 3);
        s[kb][e] = key < sees ? s[kb][e] * a.scale_log2 : -INFINITY;
        mx = fmaxf(mx, s[kb][e]);
      }
    mx = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, 64)));
    const float base = mx == -INFINITY ? 0.0f : mx;   // a query that has seen no key yet
    const float alpha = __builtin_amdgcn_exp2f(m - base);
    m = mx;
    l *= alpha;
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[hb][e] *= alpha;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = __builtin_amdgcn_exp2f(s[kb][8 * ch + e] - base);
          l += x;
          p[e] = (T)x;
        }
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
          const T* t = Vt + (hb * 32 + l32) * LDV + kb * 32 + ch * 16 + 4 * g;
          union { x8 v; uint2 u[2]; } va;
          va.u[0] = *reinterpret_cast<const uint2*>(t);
          va.u[1] = *reinterpret_cast<const uint2*>(t + 8);
          o[hb] = Mfma<T>::go(va.v, p, o[hb]);
        }
      }
  }

  l += __shfl_xor(l, 32, 64);
  T* first = static_cast<T*>(a.out) + w.cu_q[r] * a.os.row + h * a.os.head;
  float* first_lse = a.lse ? a.lse + (long)w.cu_q[r] * a.heads + h : nullptr;
  if (a.causal && any_not_finite<HB>(o)) {
    careful_rows<T, HD>(a, qp, kp, vp, lq, lk, q0 + wave * 32, first, first_lse);
    return;
  }
  if (qi >= lq) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T* out = first + qi * a.os.row;
#pragma unroll
  for (int hb = 0; hb < HB; ++hb)
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      union { uint2 u; T e[4]; } st;
#pragma unroll
      for (int e = 0; e < 4; ++e) st.e[e] = (T)(o[hb][e4 * 4 + e] * inv);
      *reinterpret_cast<uint2*>(out + hb * 32 + e4 * 8 + g * 4) = st.u;
    }
  if (first_lse && g == 0) first_lse[(long)qi * a.heads] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
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

extern "C" eas_status eas_prompt_attention(const eas_attn_shape* shape, const void* q, const void* k, const void* v,
                                           const int32_t* cu_q, const int32_t* cu_k, int32_t n_seqs, void* out,
                                           float* lse, void* stream) {
  eas_status st = check_shape(shape);
  if (st == EAS_OK) st = check_strides(shape->q);
  if (st == EAS_OK) st = check_strides(shape->k);
  if (st == EAS_OK) st = check_strides(shape->v);
  if (st != EAS_OK) return st;
  if (!cu_q) return EAS_ERR_INVALID_ARG;
  if (n_seqs < 0 || n_seqs > EAS_MAX_SEQS) return EAS_ERR_CAPACITY;
  if (!cu_k) cu_k = cu_q;
  st = check_cu(cu_q, n_seqs);
  if (st == EAS_OK) st = check_cu(cu_k, n_seqs);
  if (st == EAS_OK) st = check_out_strides(shape->out, cu_q[n_seqs], shape->heads, shape->head_dim);
  if (st != EAS_OK) return st;
  if (cu_q[n_seqs] == 0) return EAS_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out) || (uintptr_t)lse % 4) return EAS_ERR_INVALID_ARG;
  if (cu_k[n_seqs] > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return EAS_ERR_INVALID_ARG;

  PromptWork w = {};
  w.n = n_seqs;
  int64_t tiles = 0;
  for (int r = 0; r < n_seqs; ++r) {
    w.order[r] = r;
    w.tile_start[r] = (int)tiles;
    tiles += ((int64_t)cu_q[r + 1] - cu_q[r] + QT - 1) / QT;
  }
  w.tile_start[n_seqs] = (int)tiles;
  for (int r = 0; r <= n_seqs; ++r) w.cu_q[r] = cu_q[r], w.cu_k[r] = cu_k[r];
  if (tiles * shape->heads > 0x7fffffff) return EAS_ERR_UNSUPPORTED;
  const PromptArgs a = {q, k, v, out, lse, shape->q, shape->k, shape->v, shape->out, shape->heads,
                        shape->heads / shape->kv_heads, shape->causal, shape->scale * kLog2e};
  const dim3 grid((unsigned)(tiles * shape->heads));
  const hipStream_t s = (hipStream_t)stream;
  if (shape->dtype == EAS_BF16 && shape->head_dim == 64)
    hipLaunchKernelGGL((prompt_kernel<bf16, 64>), grid, dim3(256), 0, s, a, w);
  else if (shape->dtype == EAS_BF16)
    hipLaunchKernelGGL((prompt_kernel<bf16, 128>), grid, dim3(256), 0, s, a, w);
  else if (shape->head_dim == 64)
    hipLaunchKernelGGL((prompt_kernel<f16, 64>), grid, dim3(256), 0, s, a, w);
  else
    hipLaunchKernelGGL((prompt_kernel<f16, 128>), grid, dim3(256), 0, s, a, w);
  return hipGetLastError() == hipSuccess ? EAS_OK : EAS_ERR_HIP;
}
