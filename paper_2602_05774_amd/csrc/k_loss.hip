// The base losses of draft training on materialised logits, and their total.
//
//   cross entropy  l = log sum_v exp(x_v / T) - x_y / T
//   distillation   l = sum_k p_k (log p_k - log q(i_k)),  q = softmax(x / T)
//   gradient       g_v = scale w / T (P q_v - sum_{k: i_k = v} p_k)
// (the cross entropy is P = 1 with one member, the label).
//
// One workgroup per row: its log-sum-exp in one sweep, then, with the gradient,
// a second sweep that writes g.  A row out of play is not read.
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"
#include "vsd_loss.hpp"

namespace vsd {

namespace {

constexpr int kThreads = 256;

template <typename T, bool DISTILL, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_row_loss(LossArgs a) {
  constexpr int kWaves = kThreads / kWave, kStep = kThreads * 8;
  __shared__ float red_m[kWaves], red_s[kWaves];
  __shared__ int sid[DISTILL ? kMaxMembers : 1];
  __shared__ float sp[DISTILL ? kMaxMembers : 1];
  __shared__ float sum_p;
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t r = blockIdx.x;
  const T* X = static_cast<const T*>(a.X) + r * a.ld;
  T* G = static_cast<T*>(a.G) + (GRAD ? r * a.ldg : 0);
  const float w = row_weight(a, r);

  // the row's members (every wavefront has the label; the first one the teacher's)
  Member e{-1, 1.0f, 0.0f};
  float mass = 1.0f;
  if (DISTILL) {
    if (wave == 0) {
      e = load_member(a, r, lane);
      const float total = wave_sum(e.p);
      sid[lane] = e.id;
      sp[lane] = e.p;
      if (lane == 0) sum_p = total;
    }
    __syncthreads();
    mass = sum_p;
  } else {
    e.id = a.idx[r];
    if ((uint32_t)e.id >= (uint32_t)a.V) {
      if (e.id != -1 && threadIdx.x == 0) report_error(a.err, VSD_DEVERR_TOKEN_RANGE);
      mass = 0.0f;
    }
  }
  bool live = mass != 0.0f && w != 0.0f;
  // the members' logits: read ahead of the sweeps' barrier, since G may be X
  float x_mine = -INFINITY;
  if (wave == 0 && live && e.id >= 0) x_mine = load1(X + e.id);

  float m = kNegBig, s = 0.0f;
  if (live) {
    int base = threadIdx.x * 8;
    for (; base + 8 <= a.V; base += kStep) {
      float x[8];
      load8(X + base, x);
      lse_add8(x, m, s, a.c);
    }
    for (int v = base; v < min(a.V, base + 8); ++v) lse_join(m, s, load1(X + v), 1.0f, a.c);
    wave_lse(m, s, a.c);
    if (lane == 0) {
      red_m[wave] = m;
      red_s[wave] = s;
    }
    __syncthreads();
    m = red_m[0];
    s = red_s[0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) lse_join(m, s, red_m[k], red_s[k], a.c);
  }
  const bool empty = live && s == 0.0f;  // no logit above -inf
  live = live && !empty;

  // the loss, by the first wavefront
  if (wave == 0) {
    float loss = 0.0f;
    const float tail = logf(s);
    if (live && e.id >= 0) {
      const float log_q = (x_mine - m) * a.inv_t - tail;
      loss = e.p != 0.0f ? e.plogp - e.p * log_q : 0.0f;
    }
    if (DISTILL) loss = wave_sum(loss);
    if (lane == 0) {
      a.loss[r] = loss;
      if (a.lse != nullptr) a.lse[r] = live ? m * a.inv_t + tail : empty ? -INFINITY : 0.0f;
    }
  }
  if (!GRAD) return;

  const float k = a.scale * w * a.inv_t;
  const float kq = live ? k * mass / s : 0.0f;
  auto grad_of = [&](float x) { return live ? kq * lse_term(x, m, a.c) : 0.0f; };
  const int label = DISTILL || !live ? -1 : e.id;
  int base = threadIdx.x * 8;
  for (; base + 8 <= a.V; base += kStep) {
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, g[8];
    if (live) load8(X + base, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = grad_of(x[j]) - (base + j == label ? k : 0.0f);
    store8(G + base, g);
  }
  for (int v = base; v < min(a.V, base + 8); ++v)
    store1(G + v, (live ? grad_of(load1(X + v)) : 0.0f) - (v == label ? k : 0.0f));
  if (!DISTILL || !live) return;
  // the members' columns again, each from its own logit and by the first of
  // the members that name it, so that every element is rounded once
  __syncthreads();
  if (wave != 0 || e.id < 0) return;
  float p = 0.0f;
  bool first = true;
  for (int j = 0; j < a.K; ++j) {
    const bool same = sid[j] == e.id;
    p += same ? sp[j] : 0.0f;
    first = first && !(same && j < lane);
  }
  if (first) store1(G + e.id, grad_of(x_mine) - k * p);
}

// loss_scale sum_r w_r l_r over a call's rows, in a fixed order (64-bit sums:
// one thread adds R / 1024 rows).
constexpr int kTotalThreads = 1024;
__global__ __launch_bounds__(kTotalThreads) void k_row_total(const float* loss, const float* weight, int64_t R,
                                                             float scale, float* total) {
  __shared__ double part[kTotalThreads];
  double acc = 0.0;
  for (int64_t r = threadIdx.x; r < R; r += kTotalThreads) {
    const float l = loss[r];
    if (l != 0.0f) acc += (double)l * (weight != nullptr ? weight[r] : 1.0f);  // (a row out of play has any weight)
  }
  part[threadIdx.x] = acc;
  for (int n = kTotalThreads / 2; n > 0; n /= 2) {
    __syncthreads();
    if ((int)threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
  }
  if (threadIdx.x == 0) *total = (float)(part[0] * scale);
}

template <typename T, bool DISTILL>
hipError_t launch_t(const LossArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.R);
  if (a.G != nullptr)
    hipLaunchKernelGGL((k_row_loss<T, DISTILL, true>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_row_loss<T, DISTILL, false>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_row_loss(const LossArgs& a, bool bf16, hipStream_t s) {
  if (a.val != nullptr) return bf16 ? launch_t<bf16_t, true>(a, s) : launch_t<float, true>(a, s);
  return bf16 ? launch_t<bf16_t, false>(a, s) : launch_t<float, false>(a, s);
}

hipError_t launch_row_total(const float* loss, const float* weight, int64_t R, float scale, float* total,
                            hipStream_t s) {
  hipLaunchKernelGGL(k_row_total, dim3(1), dim3(kTotalThreads), 0, s, loss, weight, R, scale, total);
  return hipGetLastError();
}

}  // namespace vsd
