// Shared by the base losses' kernels: a row's members (the label of the cross
// entropy, the teacher's top logits of the distillation) and log-sum-exps.
//
// A row's log-sum-exp is held as (m, s): m its largest logit (raw), s the sum
// of exp2((x - m) c), c = log2(e) / T.  The difference x - m is formed before
// it is scaled: near the maximum, where the large probabilities are, it is
// exact or nearly so, while x c - m c would carry half an ulp of the product.
// A row that has seen nothing has m = -FLT_MAX and s = 0; a -inf logit adds 0
// to it.  (s is finite or, from a NaN or +inf logit, NaN, and stays NaN.)
#pragma once

#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

__device__ __forceinline__ float lse_term(float x, float m, float c) {
  return __builtin_amdgcn_exp2f((x - m) * c);
}
__device__ __forceinline__ void lse_join(float& m, float& s, float om, float os, float c) {
  const float nm = fmaxf(m, om);
  s = s * lse_term(m, nm, c) + os * lse_term(om, nm, c);
  m = nm;
}
template <int CTRL>
__device__ __forceinline__ void lse_step(float& m, float& s, float c) {
  lse_join(m, s, dpp_f<CTRL>(m), dpp_f<CTRL>(s), c);
}
__device__ __forceinline__ void wave_lse(float& m, float& s, float c) {
  lse_step<kDppQuad1>(m, s, c);
  lse_step<kDppQuad2>(m, s, c);
  lse_step<kDppHalfMirror>(m, s, c);
  lse_step<kDppMirror>(m, s, c);
  float rm = lane_f(m, 0), rs = lane_f(s, 0);
#pragma unroll
  for (int r = 1; r < 4; ++r) lse_join(rm, rs, lane_f(m, 16 * r), lane_f(s, 16 * r), c);
  m = rm;
  s = rs;
}
// Eight logits of a row.
__device__ __forceinline__ void lse_add8(const float (&x)[8], float& m, float& s, float c) {
  const float nm = fmaxf(m, max8(x));
  s *= lse_term(m, nm, c);
  m = nm;
#pragma unroll
  for (int k = 0; k < 8; ++k) s += lse_term(x[k], m, c);
}

// Eight consecutive logits as they lie in memory.
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
  uint4 a;
  __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void clear() { a = make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x);
    v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
    v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z);
    v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
  }
  __device__ __forceinline__ void load_part(const bf16_t* p, int n) {
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = k < n ? p[k] : 0xFF80u;
    a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void clear() {
    a = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    b = a;
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void load_part(const float* p, int n) {
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = k < n ? p[k] : -INFINITY;
    a = make_float4(w[0], w[1], w[2], w[3]);
    b = make_float4(w[4], w[5], w[6], w[7]);
  }
};
// Columns base .. base + 7 of a row of V columns, -inf past its end (nothing is
// read there).
template <typename T>
__device__ __forceinline__ void load_cols(Raw8<T>& x, const T* row, int base, int V) {
  if (base + 8 <= V)
    x.load(row + base);
  else if (base < V)
    x.load_part(row + base, V - base);
  else
    x.clear();
}

// One row's members, lane k holding member k: its column (-1: none), its
// probability p and p log p.  Teacher values val / T_p are normalised over the
// row's members or by the teacher's log-sum-exp.  A member of value -inf has
// probability 0 and takes no further part.
struct Member {
  int id;
  float p, plogp;
};
__device__ __forceinline__ int member_id(const LossArgs& a, int64_t r, int lane) {
  const int id = lane < a.K ? a.idx[r * a.K + lane] : -1;
  if ((uint32_t)id < (uint32_t)a.V) return id;
  if (id != -1) report_error(a.err, VSD_DEVERR_TOKEN_RANGE);
  return -1;
}
// What lane k needs for member k: its teacher logit / T_p and the teacher's log-sum-exp.
struct MemberValue {
  float v, lse;
};
__device__ __forceinline__ MemberValue load_value(const LossArgs& a, int64_t r, int lane, int id) {
  MemberValue m{-INFINITY, a.teacher_lse != nullptr ? a.teacher_lse[r] : 0.0f};
  if (id >= 0) {
    const int64_t at = r * a.K + lane;
    m.v = (a.val_bf16 ? load1(static_cast<const bf16_t*>(a.val) + at) : static_cast<const float*>(a.val)[at]) * a.inv_tp;
  }
  return m;
}
__device__ __forceinline__ Member member_of(const LossArgs& a, int id, const MemberValue& m) {
  Member e{id, 0.0f, 0.0f};
  const bool in = id >= 0 && m.v != -INFINITY;
  float lp;
  if (a.teacher_lse != nullptr) {
    lp = m.v - m.lse;
  } else {
    const float top = wave_max(m.v);
    const float sum = wave_sum(in ? expf(m.v - top) : 0.0f);
    lp = (m.v - top) - logf(sum);
  }
  if (in) {
    e.p = expf(lp);
    e.plogp = e.p > 0.0f || e.p != e.p ? e.p * lp : 0.0f;
  } else {
    e.id = -1;
  }
  return e;
}

// Whether a row takes part by its weight.
__device__ __forceinline__ float row_weight(const LossArgs& a, int64_t r) {
  return a.weight != nullptr ? a.weight[r] : 1.0f;
}

// loss_scale sum_r w_r l_r over a call's rows, in 64 bits and in one order
// whatever workgroup forms it: 1024 partial sums of every 1024th row, then
// those (of 64 consecutive ones a tree, of the 16 results a chain).
constexpr int kTotalThreads = 1024;
template <int kThreads>
__device__ __forceinline__ void row_total(const float* loss, const float* weight, int64_t R, float scale,
                                          float* total) {
  __shared__ double part[kTotalThreads / kWave];
  constexpr int U = 8;  // rows in flight per thread
  for (int t = threadIdx.x; t < kTotalThreads; t += kThreads) {
    double acc = 0.0;
    for (int64_t r0 = t; r0 < R; r0 += U * kTotalThreads) {
      float l[U], w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * kTotalThreads;
        l[u] = r < R ? __hip_atomic_load(loss + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0f;
        w[u] = r < R && weight != nullptr ? weight[r] : 1.0f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) acc += l[u] != 0.0f ? (double)l[u] * w[u] : 0.0;  // (out of play: any weight)
    }
    for (int n = kWave / 2; n > 0; n /= 2) acc += __shfl_xor(acc, n);
    if ((threadIdx.x & 63) == 0) part[t / kWave] = acc;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  double acc = part[0];
  for (int k = 1; k < kTotalThreads / kWave; ++k) acc += part[k];
  *total = (float)(acc * scale);
}

// The last of a launch's workgroups to come here forms the total (its thread 0
// having stored the losses of its own rows device-wide, or after a barrier that
// follows such stores).
template <int kThreads>
__device__ __forceinline__ void total_by_last(const LossArgs& a) {
  if (a.total == nullptr || a.counter == nullptr) return;
  __shared__ int last;
  if (threadIdx.x == 0)
    last = __hip_atomic_fetch_add(a.counter, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  if (threadIdx.x == 0) *a.counter = 0;
  row_total<kThreads>(a.loss, a.weight, a.R, a.scale, a.total);
}

}  // namespace vsd
