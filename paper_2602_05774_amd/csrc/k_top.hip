// The K largest logits of a row, their indices and the row's log-sum-exp.
//
// One workgroup per row, one sweep: it forms the log-sum-exp and, per thread, the
// largest entry of each of up to 16 groups of its columns.  The K-th largest of
// some threads' maxima is a lower bound of the row's K-th entry, so the members
// are among the entries that reach it, in the groups whose maximum does (few
// more than K): those groups are read again, the entries listed in LDS, and an
// entry's place is the number of entries that beat it.  Order: the larger value
// first, equal values by the smaller index.  A row with more groups or entries
// at the bound than the lists hold (long runs of equal logits) gets its K-th
// entry by bisection instead.  (Few long rows in segments of at least 4096 columns, a
// workgroup each, and a second launch that joined them: 24 rows of 128 256 in 23.5
// instead of 25.4 us, 24 rows of 32 000 in 22.1 instead of 18.0: not kept.)
//
// Bound by reading the row once: 8192 rows of 128 256 (bf16, mapped, K = 16) in 384
// us, 5.5 TB/s; 2049 of 32 003 (float32, K = 10) in 45 us, 5.8 TB/s.  Few rows take
// the latency of one row's sweep: 24 of 128 256 (K = 64) in 21 us.
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"
#include "vsd_loss.hpp"

namespace vsd {

namespace {

constexpr int kU = 4;  // loads of 8 columns in flight per thread
// LDS lists.  Short rows (one wavefront, one group a thread) have short ones, so
// that eight of their wavefronts fit a SIMD.
template <int kThreads>
struct Lists {
  static constexpr bool kShort = kThreads == kWave;
  static constexpr int kGroups = kShort ? 1 : 16;      // per thread
  static constexpr int kGroupCap = kShort ? 64 : 1024; // listed groups
  static constexpr int kCap = kShort ? 512 : 2048;     // listed entries
};
// Rows for one wavefront: with more members the K-th of its 64 maxima is far below
// the row's (us, one wavefront / four: 65 536 x 1000 K = 10 83 / 248, K = 32
// 113 / 399, K = 64 686 / 485; 8192 x 4000 K = 16 33 / 45, K = 32 40 / 65;
// 8192 x 8000 K = 16 50 / 48; 16 384 x 32 000 367 / 195).
constexpr int kShortCols = 4096, kShortK = 32;
// Members up to which four wavefronts' bound comes from rounds of wavefront maxima
// instead of a count over all threads' (us, rounds / count: 8192 x 4000, K = 16,
// 46.5 / 62.1; 8192 x 32 000 108 / 115; one wavefront, 65 536 x 1000, K = 10, 93 / 86).
constexpr int kRoundsK = 16;
// maxima that each of W wavefronts contributes to it: together more than K
__host__ __device__ constexpr int maxima_of(int K, int W) { return (K + W - 1) / W + 1; }

// A value as an integer in the same order (-0 = +0), and back.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) != 0u ? o & 0x7FFFFFFFu : ~o);
}
// An entry as one integer: the larger value, then the smaller index, is the
// larger key.  0 is below every entry.
__device__ __forceinline__ uint64_t key_of(float x, int index) {
  return (uint64_t)order_of(x) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int index_in(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float value_in(uint64_t key) { return value_of((uint32_t)(key >> 32)); }
// How many of keys[0 .. n) (n even, 16-byte aligned) are larger.
__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t* keys, int n) {
  int rank = 0;
  for (int j = 0; j < n; j += 2) {
    const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(keys + j);
    rank += (k.x > key ? 1 : 0) + (k.y > key ? 1 : 0);
  }
  return rank;
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, (uint32_t)dpp_i<kDppQuad1>((int)v));
  v = max(v, (uint32_t)dpp_i<kDppQuad2>((int)v));
  v = max(v, (uint32_t)dpp_i<kDppHalfMirror>((int)v));
  v = max(v, (uint32_t)dpp_i<kDppMirror>((int)v));
  return max(max((uint32_t)lane_i((int)v, 0), (uint32_t)lane_i((int)v, 16)),
             max((uint32_t)lane_i((int)v, 32), (uint32_t)lane_i((int)v, 48)));
}

template <int kWaves>
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

template <typename T, bool MAP, int kThreads>
__global__ __launch_bounds__(kThreads) void k_top_logits(TopArgs a) {
  constexpr int kWaves = kThreads / kWave, kStep = kThreads * 8;
  constexpr int kGroups = Lists<kThreads>::kGroups, kGroupCap = Lists<kThreads>::kGroupCap,
                kCap = Lists<kThreads>::kCap;
  constexpr int kShared = kGroups * kThreads > 2 * kCap ? kGroups * kThreads : 2 * kCap;
  __shared__ float red_m[kWaves], red_s[kWaves];
  __shared__ int red_i[kWaves];
  __shared__ __align__(16) uint32_t maxima[kThreads];
  __shared__ float bound;
  __shared__ __align__(16) float shared[kShared];  // the groups' maxima, later the listed entries' keys
  __shared__ int groups[kGroupCap];
  __shared__ int ngroups, count;
  uint64_t* const keys = reinterpret_cast<uint64_t*>(shared);
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t r = blockIdx.x;
  const int V = a.V;
  const T* Y = static_cast<const T*>(a.Y) + r * a.ld;
  const int first = threadIdx.x * 8;
  auto index_of = [&](int col) { return MAP ? a.inv[col] : col; };
  auto mask_of = [&](int base) { return MAP ? (uint32_t)a.mapped[base >> 3] : 0xFFu; };
  // every entry of eight columns that may be a member (above -inf, its column mapped), by f(value, column)
  auto entries = [&](int base, auto&& f) {
    if (base >= V) return;
    Raw8<T> q;
    float x[8];
    load_cols(q, Y, base, V);
    q.get(x);
    const uint32_t in = mask_of(base);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (((in >> k) & 1u) != 0u && x[k] > -INFINITY) f(x[k], base + k);
  };
  auto sweep = [&](auto&& f) {
    for (int base = first; base < V; base += kStep) entries(base, f);
  };

  // the sweep: kU * kStep columns an iteration, the next one's loads in flight
  // (whole iterations: no load depends on a branch), `per_group` iterations a group
  const int iters = (V + kU * kStep - 1) / (kU * kStep), whole = V / (kU * kStep);
  const int per_group = (iters + kGroups - 1) / kGroups;
  float m = kNegBig, s = 0.0f, best = -INFINITY, top = -INFINITY;
  int group = 0, in_group = 0;
  struct Cols {
    Raw8<T> q[kU];
    uint32_t in[kU];
  } cols[2];
  auto load = [&](Cols& c, int it) {
    const int base = first + it * kU * kStep;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      c.q[u].load(Y + base + u * kStep);
      if (MAP) c.in[u] = mask_of(base + u * kStep);
    }
  };
  auto take = [&](const Cols& c) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float x[8];
      c.q[u].get(x);
      lse_add8(x, m, s, a.c);
      if (MAP) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = ((c.in[u] >> k) & 1u) != 0u ? x[k] : -INFINITY;
      }
      top = fmaxf(top, max8(x));
    }
    if (++in_group == per_group) {
      shared[group * kThreads + threadIdx.x] = top;
      best = fmaxf(best, top);
      top = -INFINITY;
      in_group = 0;
      ++group;
    }
  };
  if (whole > 0) load(cols[0], 0);
  for (int it = 0; it < whole; it += 2) {
    load(cols[1], min(it + 1, whole - 1));
    take(cols[0]);
    if (it + 1 == whole) break;
    load(cols[0], min(it + 2, whole - 1));
    take(cols[1]);
  }
  if (whole < iters) {
    const int base = first + whole * kU * kStep;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      load_cols(cols[0].q[u], Y, base + u * kStep, V);
      cols[0].in[u] = MAP && base + u * kStep < V ? mask_of(base + u * kStep) : 0u;
    }
    take(cols[0]);
  }
  if (in_group > 0) {
    shared[group * kThreads + threadIdx.x] = top;
    best = fmaxf(best, top);
  }
  const int used = (iters + per_group - 1) / per_group;
  wave_lse(m, s, a.c);
  // the bound: the K-th largest of the threads' maxima (many members: counted
  // over all of them), or of some per wavefront that has columns.  Equal maxima
  // are told apart by the low byte, which gives way to the thread: the bound is
  // at most that much lower (not at all for bf16 logits).
  const bool rounds = kWaves > 1 && a.K <= kRoundsK;
  const int per = rounds ? maxima_of(a.K, min(kWaves, (V + kWave * 8 - 1) / (kWave * 8))) : kWave;
  static_assert(maxima_of(kRoundsK, 1) <= kWave && kThreads <= 256, "a wavefront has that many, a byte names a thread");
  uint32_t left = (order_of(best) & ~0xFFu) | threadIdx.x;
  if (rounds) {
    for (int t = 0; t < per; ++t) {
      const uint32_t top = wave_max_u32(left);
      if (left == top) left = 0u;
      if (lane == 0) maxima[wave * per + t] = top;
    }
  } else {
    maxima[threadIdx.x] = left;
  }
  if (lane == 0) {
    red_m[wave] = m;
    red_s[wave] = s;
  }
  if (threadIdx.x == 0) ngroups = count = 0;
  __syncthreads();
  const int nmax = kWaves * per;
  if ((int)threadIdx.x < nmax) {
    const uint32_t mine = maxima[threadIdx.x];
    int rank = 0;
    if (rounds) {
      for (int j = 0; j < nmax; ++j) rank += maxima[j] > mine ? 1 : 0;
    } else {
#pragma unroll 4
      for (int j = 0; j < kThreads; j += 4) {
        const uint4 o = *reinterpret_cast<const uint4*>(maxima + j);
        rank += (o.x > mine ? 1 : 0) + (o.y > mine ? 1 : 0) + (o.z > mine ? 1 : 0) + (o.w > mine ? 1 : 0);
      }
    }
    if (rank == a.K - 1) {
      const float v = value_of(mine & ~0xFFu);
      bound = v == v ? v : -INFINITY;  // (a thread without an entry: -inf without its low byte is no number)
    }
  }
  if (wave == 0) {
    m = red_m[0];
    s = red_s[0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) lse_join(m, s, red_m[k], red_s[k], a.c);
    if (lane == 0 && a.lse != nullptr) a.lse[r] = s == 0.0f ? -INFINITY : m * a.inv_t + logf(s);
  }
  __syncthreads();
  const float least = bound;
  if (best >= least && best > -INFINITY)
    for (int g = 0; g < used; ++g)
      if (shared[g * kThreads + threadIdx.x] >= least) {
        const int at = atomicAdd(&ngroups, 1);
        if (at < kGroupCap) groups[at] = g * kThreads + threadIdx.x;
      }
  __syncthreads();
  const bool crowded = ngroups > kGroupCap;
  auto list = [&](float x, int col) {
    const int at = atomicAdd(&count, 1);
    if (at < kCap) keys[at] = key_of(x, index_of(col));
  };
  if (!crowded) {
    const int chunks = per_group * kU, items = ngroups * chunks;
    for (int i = threadIdx.x; i < items; i += kThreads) {
      const int id = groups[i / chunks], g = id / kThreads, t = id % kThreads;
      entries((g * chunks + i % chunks) * kStep + t * 8, [&](float x, int col) {
        if (x >= least) list(x, col);
      });
    }
  }
  __syncthreads();
  int n = count;
  if (crowded || n > kCap) {
    // the K-th entry's value, bit by bit, then the index up to which entries of
    // that value are members
    auto counted = [&](auto&& f) {
      int c = 0;
      sweep([&](float x, int col) { c += f(x, col) ? 1 : 0; });
      return block_sum<kWaves>(c, red_i);
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
      if (o > kth || (o == kth && index_of(col) <= last)) list(x, col);
    });
    __syncthreads();
    n = min(count, kCap);
  }
  if (threadIdx.x == 0 && (n & 1) != 0) keys[n] = 0;  // (kCap is even)
  __syncthreads();
  int32_t* const idx = a.idx + r * a.K;
  float* const val = a.val + r * a.K;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t key = keys[i];
    const int rank = rank_of(key, keys, (n + 1) & ~1);
    if (rank < a.K) {
      idx[rank] = index_in(key);
      val[rank] = value_in(key);
    }
  }
  for (int i = n + (int)threadIdx.x; i < a.K; i += kThreads) {
    idx[i] = -1;
    val[i] = -INFINITY;
  }
}

// Rows of up to 512 kNch columns, one wavefront each: the row stays in registers as
// integers in the values' order (bf16: 16 bits of them; 0: no entry) and the K-th
// largest is found bit by bit, a count of all entries per bit, until exactly K are
// at or above it.  Bound by those counts (ballots): the lists' bound is worth little
// where K is near the number of groups.
// us, lists / this, by columns and K: 65 536 rows of 300 bf16, 4 79 / 69, 40 1065 / 87;
// of 500 float32, 20 106 / 76; of 1000 bf16, 10 85 / 143, 64 483 / 151; of 2000, 64
// 480 / 280; 10 rows of 400, 10 17.8 / 17.7, of 1000, 64 19.4 / 19.7, of 2000, 40 17.9 /
// 26.7 (four chunks' counts one after another: only many rows hide them).
constexpr int kManyShort = 1024;
constexpr int kShortRows = 4;  // per workgroup
template <typename T, bool MAP, int kNch>
__global__ __launch_bounds__(kShortRows * kWave) void k_top_short(TopArgs a) {
  constexpr int kBits = sizeof(T) == 2 ? 16 : 32, kDown = 32 - kBits;
  __shared__ __align__(16) uint64_t all_keys[kShortRows][VSD_MAX_TOP];
  const int lane = threadIdx.x & 63, V = a.V, K = a.K;
  const int64_t r = (int64_t)blockIdx.x * kShortRows + wave_id();
  if (r >= a.R) return;
  uint64_t* const keys = all_keys[wave_id()];
  const T* Y = static_cast<const T*>(a.Y) + r * a.ld;
  auto col_of = [&](int j) { return (j >> 3) * 512 + lane * 8 + (j & 7); };
  Raw8<T> q[kNch];
  uint32_t in[kNch];
#pragma unroll
  for (int u = 0; u < kNch; ++u) {
    const int base = u * 512 + lane * 8;
    load_cols(q[u], Y, base, V);
    in[u] = !MAP ? 0xFFu : base < V ? (uint32_t)a.mapped[base >> 3] : 0u;
  }
  uint32_t o[kNch * 8];
  float m = kNegBig, s = 0.0f;
#pragma unroll
  for (int u = 0; u < kNch; ++u) {
    float x[8];
    q[u].get(x);
    lse_add8(x, m, s, a.c);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      o[u * 8 + k] = ((in[u] >> k) & 1u) != 0u && x[k] > -INFINITY ? order_of(x[k]) >> kDown : 0u;
  }
  wave_lse(m, s, a.c);
  if (lane == 0 && a.lse != nullptr) a.lse[r] = s == 0.0f ? -INFINITY : m * a.inv_t + logf(s);
  auto counted = [&](auto&& f) {
    int c = 0;
#pragma unroll
    for (int j = 0; j < kNch * 8; ++j) c += __builtin_popcountll(__ballot(f(j)));
    return c;
  };
  uint32_t kth = 1;
  bool exact = counted([&](int j) { return o[j] >= 1u; }) <= K;
  if (!exact) {
    kth = 0;
    for (int b = kBits - 1; b >= 0 && !exact; --b) {
      const uint32_t t = kth | (1u << b);
      const int c = counted([&](int j) { return o[j] >= t; });
      if (c >= K) kth = t;
      exact = c == K;
    }
  }
  // more entries of the K-th's value than places: the smallest index with enough of
  // them up to it
  int last = 0x7FFFFFFF;
  if (!exact) {
    const int need = K - counted([&](int j) { return o[j] > kth; }), bits = 32 - __builtin_clz(V);
    auto index_if = [&](int j) { return o[j] != kth ? 0x7FFFFFFF : MAP ? a.inv[col_of(j)] : col_of(j); };
    last = (1 << bits) - 1;  // (every index is below V)
    for (int b = bits - 1; b >= 0; --b) {
      const int t = last & ~(1 << b);
      if (counted([&](int j) { return index_if(j) <= t; }) >= need) last = t;
    }
  }
  int n = 0;
#pragma unroll
  for (int j = 0; j < kNch * 8; ++j) {
    bool member = o[j] >= kth;
    const uint64_t maybe = __ballot(member);
    if (maybe == 0ull) continue;
    const int index = !member ? 0 : MAP ? a.inv[col_of(j)] : col_of(j);
    member = member && (o[j] > kth || index <= last);
    const uint64_t who = __ballot(member);
    // (bf16: the value's lower half is zeros below the order's, ones where it is negative)
    const uint32_t order = kDown == 0 || o[j] >= 0x8000u ? o[j] << kDown : o[j] << kDown | 0xFFFFu;
    if (member) keys[n + __builtin_popcountll(who & ((1ull << lane) - 1))] = (uint64_t)order << 32 | (uint32_t)~index;
    n += __builtin_popcountll(who);
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  if (lane >= K) return;
  if (lane >= n) {
    a.idx[r * K + lane] = -1;
    a.val[r * K + lane] = -INFINITY;
    return;
  }
  const uint64_t key = keys[lane];
  int rank = 0;
  for (int j = 0; j < n; ++j) rank += keys[j] > key ? 1 : 0;
  a.idx[r * K + rank] = index_in(key);
  a.val[r * K + rank] = value_in(key);
}

__global__ __launch_bounds__(256) void k_top_bits(const int32_t* inv, int V, uint8_t* mapped) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= (V + 7) / 8) return;
  uint32_t bits = 0;
  for (int k = 0; k < 8; ++k)
    if (b * 8 + k < V && inv[b * 8 + k] >= 0) bits |= 1u << k;
  mapped[b] = (uint8_t)bits;
}

template <typename T, int kThreads>
hipError_t launch_n(const TopArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.R);
  if (a.inv != nullptr)
    hipLaunchKernelGGL((k_top_logits<T, true, kThreads>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_top_logits<T, false, kThreads>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename T, int kNch>
hipError_t launch_short(const TopArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.R + kShortRows - 1) / kShortRows));
  if (a.inv != nullptr)
    hipLaunchKernelGGL((k_top_short<T, true, kNch>), grid, dim3(kShortRows * kWave), 0, s, a);
  else
    hipLaunchKernelGGL((k_top_short<T, false, kNch>), grid, dim3(kShortRows * kWave), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const TopArgs& a, hipStream_t s) {
  if (a.V <= 512) return launch_short<T, 1>(a, s);
  if (a.V <= 1024 && a.K > kShortK) return launch_short<T, 2>(a, s);
  if (a.V <= 2048 && a.K > kShortK && a.R >= kManyShort) return launch_short<T, 4>(a, s);
  if (a.V <= kShortCols && a.K <= kShortK) return launch_n<T, kWave>(a, s);
  return launch_n<T, 256>(a, s);
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
