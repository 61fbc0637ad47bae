// The base losses of draft training on materialised logits, and their total.
//
//   cross entropy  l = log sum_v exp(x_v / T) - x_y / T
//   distillation   l = sum_k p_k (log p_k - log q(i_k)),  q = softmax(x / T)
//   gradient       g_v = scale w / T (P q_v - sum_{k: i_k = v} p_k)
// (the cross entropy is P = 1 with one member, the label).
//
// One workgroup per row.  With the gradient the row stays in registers (kNch
// groups of eight columns per thread, all loads in flight at once) while its
// log-sum-exp is formed, so the logits are read once and g is written once; of
// rows longer than 1024 threads hold the rest is read twice (kMore).  With kNch = 0
// nothing is kept: the loss alone, and rows too many for wide workgroups, which are
// read twice.  A row out of play is not read.
//
// Bound by those bytes: 20 480 rows of 32 000 (bf16, a quarter out of play) with
// gradient in 440 us, 5.2 TB/s; 8192 of 128 256 in 786 us, 5.1 TB/s (a large copy:
// 4.7); the loss alone of 4099 rows of 32 003 (float32) in 92 us, 5.7 TB/s.
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"
#include "vsd_loss.hpp"

namespace vsd {

namespace {

constexpr int kMembersFirstRows = 8192, kMembersFirstCols = 512 * 64 / 8 * 7;
template <typename T, bool DISTILL, bool GRAD, int kThreads, int kNch, bool kMore>
__device__ __forceinline__ void row_loss(const LossArgs& a) {
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
  const int first = threadIdx.x * 8;

  // the row's members: every wavefront has the label, or whether there are any (the
  // teacher's probabilities are formed while the logits are on their way)
  Member e{-1, 1.0f, 0.0f};
  float mass = 1.0f;
  if (DISTILL) {
    e.id = member_id(a, r, lane);
    mass = __ballot(e.id >= 0) != 0ull ? 1.0f : 0.0f;
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
  MemberValue value{-INFINITY, 0.0f};
  if (wave == 0 && live) {
    if (DISTILL) value = load_value(a, r, lane, e.id);
    if (e.id >= 0) x_mine = load1(X + e.id);
  }

  float m = kNegBig, s = 0.0f;
  Raw8<T> row[kNch > 0 ? kNch : 1];
  auto members = [&]() {
    if (!DISTILL || wave != 0) return;
    e = member_of(a, e.id, value);
    const float total = wave_sum(e.p);
    sid[lane] = e.id;
    sp[lane] = e.p;
    if (lane == 0) sum_p = total;
  };
  // The first wavefront's probabilities: while the row is on its way, but for many rows
  // that fill at least 7/8 of 512 threads x 64 columns before it is asked for (us, before /
  // meanwhile, bf16: 16 384 rows of 32 000, 4, 16 and 32 members, 390 / 410, 397 / 416 and
  // 412 / 423; 16 384 of 28 672, 16, 355 / 372; 8192 of 32 768, 16, 217 / 227; 8192 of
  // 29 500, 16, 201 / 204; but 4096 of 30 522, 16, 117 / 116; 96 of 32 000, 10, 20.2 / 19.4;
  // 16 384 of 17 000 and 24 000, 32, 283 / 258 and 330 / 313; other threads and columns:
  // 4096 of 128 256, 64, 499 / 471; 9930 of 4673, 46, 68 / 66; 4000 of 9000 float32, 90 / 85).
  constexpr bool kMaybeFirst = DISTILL && kThreads == 512 && kNch == 8;
  const bool members_first = kMaybeFirst && a.R >= kMembersFirstRows && a.V >= kMembersFirstCols;
  if (live) {
    if (members_first) {
      members();
      __syncthreads();
    }
    if constexpr (kNch > 0) {
#pragma unroll
      for (int j = 0; j < kNch; ++j) load_cols(row[j], X, first + j * kStep, a.V);
    }
    if (!members_first) members();
    if constexpr (kNch > 0) {
#pragma unroll
      for (int j = 0; j < kNch; ++j) {
        float x[8];
        row[j].get(x);
        lse_add8(x, m, s, a.c);
      }
    }
    if constexpr (kMore) {  // what does not fit the registers
      constexpr int U = 4;  // loads of a step; the next one's are in flight
      Raw8<T> q[2][U];
      const int from = kNch * kStep, whole = (a.V - from) / (U * kStep);
      auto load = [&](Raw8<T>(&c)[U], int it) {
#pragma unroll
        for (int u = 0; u < U; ++u) c[u].load(X + from + first + (it * U + u) * kStep);
      };
      auto take = [&](const Raw8<T>(&c)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float x[8];
          c[u].get(x);
          lse_add8(x, m, s, a.c);
        }
      };
      if (whole > 0) load(q[0], 0);
      for (int it = 0; it < whole; it += 2) {  // (no load depends on a branch)
        load(q[1], min(it + 1, whole - 1));
        take(q[0]);
        if (it + 1 == whole) break;
        load(q[0], min(it + 2, whole - 1));
        take(q[1]);
      }
      for (int base = from + whole * U * kStep + first; base < a.V; base += kStep) {
        Raw8<T> c;
        float x[8];
        load_cols(c, X, base, a.V);
        c.get(x);
        lse_add8(x, m, s, a.c);
      }
    }
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
    if (DISTILL) mass = sum_p;
  }
  live = live && mass != 0.0f;
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
      // (with the total in this launch, another XCD's workgroup reads it)
      __hip_atomic_store(a.loss + r, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (a.lse != nullptr) a.lse[r] = live ? m * a.inv_t + tail : empty ? -INFINITY : 0.0f;
    }
  }
  if (!GRAD) return;

  if (!live) {
    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    int base = first;
    for (; base + 8 <= a.V; base += kStep) store8(G + base, zero);
    for (int v = base; v < min(a.V, base + 8); ++v) store1(G + v, 0.0f);
    return;
  }
  const float k = a.scale * w * a.inv_t, kq = k * mass / s;
  auto grad_of = [&](float x) { return kq * lse_term(x, m, a.c); };
  const int label = DISTILL ? -1 : e.id;
  auto write = [&](const Raw8<T>& q, int base) {
    float x[8], g[8];
    q.get(x);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = grad_of(x[j]);
    if ((uint32_t)(label - base) < 8u) {
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] -= base + j == label ? k : 0.0f;
    }
    if (base + 8 <= a.V) {
      store8(G + base, g);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (base + j < a.V) store1(G + base + j, g[j]);
    }
  };
  if constexpr (kNch > 0) {
#pragma unroll
    for (int j = 0; j < kNch; ++j)
      if (first + j * kStep < a.V) write(row[j], first + j * kStep);
  }
  if constexpr (kMore) {
    constexpr int U = 2;
    int base = first + kNch * kStep;
    for (; base + (U - 1) * kStep + 8 <= a.V; base += U * kStep) {
      Raw8<T> q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u].load(X + base + u * kStep);
#pragma unroll
      for (int u = 0; u < U; ++u) write(q[u], base + u * kStep);
    }
    for (; base < a.V; base += kStep) {
      Raw8<T> q;
      load_cols(q, X, base, a.V);
      write(q, base);
    }
  }
  if (!DISTILL) return;
  // the members' columns again, each from its own logit and by the first of
  // the members that name it, so that every element is rounded once
  __syncthreads();
  if (wave != 0 || e.id < 0) return;
  float p = 0.0f;
  bool mine = true;
  for (int j = 0; j < a.K; ++j) {
    const bool same = sid[j] == e.id;
    p += same ? sp[j] : 0.0f;
    mine = mine && !(same && j < lane);
  }
  if (mine) store1(G + e.id, grad_of(x_mine) - k * p);
}

__global__ __launch_bounds__(kTotalThreads) void k_row_total(const float* loss, const float* weight, int64_t R,
                                                             float scale, float* total) {
  row_total<kTotalThreads>(loss, weight, R, scale, total);
}

template <typename T, bool DISTILL, bool GRAD, int kThreads, int kNch, bool kMore>
__global__ __launch_bounds__(kThreads) void k_row_loss(LossArgs a) {
  row_loss<T, DISTILL, GRAD, kThreads, kNch, kMore>(a);
  total_by_last<kThreads>(a);
}

template <typename T, bool DISTILL, bool GRAD>
hipError_t launch_t(const LossArgs& a, hipStream_t s) {
  const RowThreads t = row_loss_threads(a.R, a.V, sizeof(T) == 4, GRAD);
  void (*kernel)(LossArgs) = nullptr;
  auto use = [&](int threads, int chunks, bool more, void (*k)(LossArgs)) {
    if (t.threads == threads && t.chunks == chunks && t.more == more) kernel = k;
  };
  if constexpr (!GRAD) {
    use(64, 0, true, k_row_loss<T, DISTILL, false, 64, 0, true>);
    use(256, 0, true, k_row_loss<T, DISTILL, false, 256, 0, true>);
    use(1024, 0, true, k_row_loss<T, DISTILL, false, 1024, 0, true>);
  } else {
    use(64, 4, false, k_row_loss<T, DISTILL, true, 64, 4, false>);
    use(256, 0, true, k_row_loss<T, DISTILL, true, 256, 0, true>);
    use(1024, 8, false, k_row_loss<T, DISTILL, true, 1024, 8, false>);
    if constexpr (sizeof(T) == 4) {
      use(256, 2, false, k_row_loss<T, DISTILL, true, 256, 2, false>);
      use(512, 2, false, k_row_loss<T, DISTILL, true, 512, 2, false>);
      use(1024, 2, false, k_row_loss<T, DISTILL, true, 1024, 2, false>);
      use(1024, 4, false, k_row_loss<T, DISTILL, true, 1024, 4, false>);
      use(1024, 8, true, k_row_loss<T, DISTILL, true, 1024, 8, true>);
    } else {
      use(128, 4, false, k_row_loss<T, DISTILL, true, 128, 4, false>);
      use(256, 4, false, k_row_loss<T, DISTILL, true, 256, 4, false>);
      use(512, 4, false, k_row_loss<T, DISTILL, true, 512, 4, false>);
      use(512, 8, false, k_row_loss<T, DISTILL, true, 512, 8, false>);
      use(1024, 16, false, k_row_loss<T, DISTILL, true, 1024, 16, false>);
      use(1024, 16, true, k_row_loss<T, DISTILL, true, 1024, 16, true>);
    }
  }
  if (kernel == nullptr) return hipErrorInvalidConfiguration;  // (row_loss_threads names one of these)
  hipLaunchKernelGGL(kernel, dim3((unsigned)a.R), dim3((unsigned)t.threads), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool DISTILL>
hipError_t launch_d(const LossArgs& a, hipStream_t s) {
  return a.G != nullptr ? launch_t<T, DISTILL, true>(a, s) : launch_t<T, DISTILL, false>(a, s);
}

}  // namespace

hipError_t launch_row_loss(const LossArgs& a, bool bf16, hipStream_t s) {
  hipError_t e;
  if (a.val != nullptr)
    e = bf16 ? launch_d<bf16_t, true>(a, s) : launch_d<float, true>(a, s);
  else
    e = bf16 ? launch_d<bf16_t, false>(a, s) : launch_d<float, false>(a, s);
  if (e != hipSuccess || a.total == nullptr || a.counter != nullptr) return e;
  return launch_row_total(a, s);
}

hipError_t launch_row_total(const LossArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_row_total, dim3(1), dim3(kTotalThreads), 0, s, a.loss, a.weight, a.R, a.scale, a.total);
  return hipGetLastError();
}

}  // namespace vsd
