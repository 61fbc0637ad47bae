// The K largest logits of a row, their indices and the row's log-sum-exp.
//
// One workgroup per row.  The first sweep forms the log-sum-exp and every
// thread's largest entry.  The K-th largest of some threads' maxima is a lower
// bound of the row's K-th entry, so the second sweep lists the entries that
// reach it (few more than K) in LDS, and each listed entry's place is the
// number of entries that beat it.  Order: the larger value first, equal values
// by the smaller index.  A row with more entries at the bound than the list
// holds (long runs of equal logits) gets its K-th entry by bisection instead.
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"
#include "vsd_loss.hpp"

namespace vsd {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kCap = 2048;   // listed entries
constexpr int kMostTop = kMaxMembers;
// maxima that each wavefront contributes to the bound: together more than K
__device__ __forceinline__ int maxima_of(int K) { return (K + kWaves - 1) / kWaves + 1; }
constexpr int kMaxima = kWaves * ((kMostTop + kWaves - 1) / kWaves + 1);

__device__ __forceinline__ bool beats(float v, int i, float ov, int oi) { return v > ov || (v == ov && i < oi); }

// A value as an integer in the same order (-0 = +0).
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int block_sum(int v, int* red) {
  const int s = wave_sum_int(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[wave_id()] = s;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) t += red[k];
  return t;
}

template <typename T, bool MAP>
__global__ __launch_bounds__(kThreads) void k_top_logits(TopArgs a) {
  constexpr int kStep = kThreads * 8;
  __shared__ float red_m[kWaves], red_s[kWaves];
  __shared__ int red_i[kWaves];
  __shared__ float maxima[kMaxima];
  __shared__ float bound;
  __shared__ float cv[kCap];
  __shared__ int ci[kCap];
  __shared__ int count;
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t r = blockIdx.x;
  const T* Y = static_cast<const T*>(a.Y) + r * a.ld;
  // every entry that may be a member (finite, its column mapped), by f(value, column)
  auto sweep = [&](auto&& f) {
    int base = threadIdx.x * 8;
    for (; base + 8 <= a.V; base += kStep) {
      float x[8];
      load8(Y + base, x);
      const uint32_t in = MAP ? a.mapped[base >> 3] : 0xFFu;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (((in >> k) & 1u) != 0u && x[k] > -INFINITY) f(x[k], base + k);
    }
    for (int v = base; v < min(a.V, base + 8); ++v) {
      const float x = load1(Y + v);
      if ((!MAP || (a.mapped[v >> 3] >> (v & 7) & 1) != 0) && x > -INFINITY) f(x, v);
    }
  };
  auto index_of = [&](int col) { return MAP ? a.inv[col] : col; };

  float m = kNegBig, s = 0.0f, best = -INFINITY;
  {
    int base = threadIdx.x * 8;
    for (; base + 8 <= a.V; base += kStep) {
      float x[8];
      load8(Y + base, x);
      lse_add8(x, m, s, a.c);
    }
    for (int v = base; v < min(a.V, base + 8); ++v) lse_join(m, s, load1(Y + v), 1.0f, a.c);
  }
  sweep([&](float x, int) { best = fmaxf(best, x); });
  wave_lse(m, s, a.c);
  const int per = maxima_of(a.K);
  for (int t = 0; t < per; ++t) {
    const float top = wave_max(best);
    const uint64_t has = __ballot(best == top);
    if (lane == (int)__builtin_ctzll(has)) best = -INFINITY;
    if (lane == 0) maxima[wave * per + t] = top;
  }
  if (lane == 0) {
    red_m[wave] = m;
    red_s[wave] = s;
  }
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  if (wave == 0) {
    if (a.lse != nullptr) {
      m = red_m[0];
      s = red_s[0];
#pragma unroll
      for (int k = 1; k < kWaves; ++k) lse_join(m, s, red_m[k], red_s[k], a.c);
      if (lane == 0) a.lse[r] = s == 0.0f ? -INFINITY : m * a.inv_t + logf(s);
    }
    const int n = kWaves * per;
    for (int i = lane; i < n; i += kWave) {
      const float v = maxima[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += beats(maxima[j], j, v, i) ? 1 : 0;
      if (rank == a.K - 1) bound = v;
    }
  }
  __syncthreads();
  const float least = bound;
  sweep([&](float x, int col) {
    if (x >= least) {
      const int at = atomicAdd(&count, 1);
      if (at < kCap) {
        cv[at] = x;
        ci[at] = index_of(col);
      }
    }
  });
  __syncthreads();
  int n = count;
  if (n > kCap) {
    // the K-th entry's value, bit by bit, then the index up to which entries of
    // that value are members
    auto counted = [&](auto&& f) {
      int c = 0;
      sweep([&](float x, int col) { c += f(x, col) ? 1 : 0; });
      return block_sum(c, red_i);
    };
    uint32_t kth = 0;
    for (int b = 31; b >= 0; --b) {
      const uint32_t t = kth | (1u << b);
      if (counted([&](float x, int) { return order_of(x) >= t; }) >= a.K) kth = t;
    }
    const int need = a.K - counted([&](float x, int) { return order_of(x) > kth; });
    int last = 0x7FFFFFFF;  // the smallest index with `need` entries of that value up to it
    for (int b = 30; b >= 0; --b) {
      const int t = last & ~(1 << b);
      if (counted([&](float x, int col) { return order_of(x) == kth && index_of(col) <= t; }) >= need) last = t;
    }
    __syncthreads();
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    sweep([&](float x, int col) {
      const uint32_t o = order_of(x);
      if (o > kth || (o == kth && index_of(col) <= last)) {
        const int at = atomicAdd(&count, 1);
        if (at < kCap) {
          cv[at] = x;
          ci[at] = index_of(col);
        }
      }
    });
    __syncthreads();
    n = min(count, kCap);
  }
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const float v = cv[i];
    const int id = ci[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += beats(cv[j], ci[j], v, id) ? 1 : 0;
    if (rank < a.K) {
      a.idx[r * a.K + rank] = id;
      a.val[r * a.K + rank] = v;
    }
  }
  if ((int)threadIdx.x >= n && (int)threadIdx.x < a.K) {
    a.idx[r * a.K + threadIdx.x] = -1;
    a.val[r * a.K + threadIdx.x] = -INFINITY;
  }
}

__global__ __launch_bounds__(256) void k_top_bits(const int32_t* inv, int V, uint8_t* mapped) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= (V + 7) / 8) return;
  uint32_t bits = 0;
  for (int k = 0; k < 8; ++k)
    if (b * 8 + k < V && inv[b * 8 + k] >= 0) bits |= 1u << k;
  mapped[b] = (uint8_t)bits;
}

template <typename T>
hipError_t launch_t(const TopArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.R);
  if (a.inv != nullptr)
    hipLaunchKernelGGL((k_top_logits<T, true>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_top_logits<T, false>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_top_bits(const int32_t* inv, int V, uint8_t* mapped, hipStream_t s) {
  const int n = (V + 7) / 8;
  hipLaunchKernelGGL(k_top_bits, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, inv, V, mapped);
  return hipGetLastError();
}

hipError_t launch_top_logits(const TopArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace vsd
