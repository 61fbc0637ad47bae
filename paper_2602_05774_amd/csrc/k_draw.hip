// One token per row under the deployed rule: temperature, top-k, top-p, min-p and
// a given random number (vsd_sample_rows).
//
// The sweep (k_draw_sweep) reads the row once, a wavefront per span of 2048 columns:
// the largest logit of every 128 columns and, where the rule needs it, the span's sum
// of weights in double precision.  k_draw_finish, a wavefront per row, ends most rows
// from these records and a few reads more:
//  * greedy: the first group that holds the maximum;
//  * no filter: the span in which the cumulative sum passes u Z, read again;
//  * filters: a bound below which no kept entry lies (the K-th largest of the groups'
//    maxima; the largest value such that the maxima from it on already weigh p Z;
//    min-p's own), the groups that reach it read again, their entries listed in LDS
//    in index order, and the borders of top-k and top-p found bit by bit.
// k_draw_left takes the rows whose lists do not fit: flat ones by draw_flat, others (k
// above 2048, long runs of equal logits) by draw_row, which also takes rows of more
// than 262 144 columns (k_draw_row): one workgroup per row, sweeping it several times: the largest entry; the
// sum of the weights, which sets their integer scale; for top-k and top-p the entry
// where the count or the mass reaches its target, 8 bits of its value a sweep from
// histograms of integers in LDS, and among equal entries by index; the kept entries'
// mass; and the index where the mass up to it passes u Z.
#include "vsd_draw64.hpp"
#include "vsd_loss.hpp"

namespace vsd {

namespace {

template <typename T, int kThreads>
struct RowDraw {
  static constexpr int kWaves = kThreads / kWave, kStep = kThreads * 8, kParts = 256;
  static constexpr int kBits = sizeof(T) == 2 ? 16 : 32, kDown = 32 - kBits;
  struct Shared {
    uint64_t sums[kParts];
    uint64_t red[kWaves];
    double redd[kWaves];
    float redf[kWaves];
    uint64_t found[3];
    int at;
  };
  Shared& sh;
  const T* Y;
  int V;
  float m;
  double c, scale;

  // f(value, column) for the entries of columns [lo, hi) that thread t of n threads
  // visits, lo a multiple of 8
  template <class F>
  __device__ __forceinline__ void visit(int lo, int hi, int t, int n, F&& f) const {
    for (int64_t b = lo + (int64_t)t * 8; b < hi; b += n * 8) {
      const int base = (int)b;
      Raw8<T> q;
      float x[8];
      load_cols(q, Y, base, V);
      q.get(x);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (base + k < hi && !(x[k] == -INFINITY)) f(x[k], base + k);
    }
  }
  template <class F>
  __device__ __forceinline__ void sweep(F&& f) const {
    visit(0, V, threadIdx.x, kThreads, f);
  }
  __device__ __forceinline__ static uint32_t key(float x) { return draw_order(x) >> kDown; }
  __device__ __forceinline__ static float value(uint32_t k) {
    // (16 bits: the lower half is ones below zero, zeros above)
    return draw_value(kDown == 0 || k >= 0x8000u ? k << kDown : k << kDown | 0xFFFFu);
  }
  __device__ __forceinline__ uint64_t weight(float x) const { return (uint64_t)(draw_weight(x, m, c) * scale + 0.5); }

  template <typename N>
  __device__ __forceinline__ static N wave_total(N v) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
    return v;
  }
  template <typename N>
  __device__ __forceinline__ N total(N v, N* red) const {
    v = wave_total(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[wave_id()] = v;
    __syncthreads();
    N t = red[0];
    for (int k = 1; k < kWaves; ++k) t += red[k];
    return t;
  }
  __device__ __forceinline__ uint64_t total(uint64_t v) const { return total(v, sh.red); }

  // The smallest index up to which measure(x, column) sums to more than target
  // (which its sum over the row exceeds).
  template <class M>
  __device__ __forceinline__ int find_index(M&& measure, uint64_t target) const {
    const int lane = threadIdx.x & 63, w = wave_id();
    int lo = 0, hi = V;
    while (hi - lo > kStep) {
      const int part = (int)((((int64_t)hi - lo + kParts - 1) / kParts + 511) / 512 * 512);
      const int parts = (hi - lo + part - 1) / part;
      __syncthreads();
      for (int p = w; p < parts; p += kWaves) {
        const int from = lo + p * part;
        uint64_t s = 0;
        visit(from, min((int64_t)from + part, (int64_t)hi), lane, kWave, [&](float x, int col) { s += measure(x, col); });
        s = wave_total(s);
        if (lane == 0) sh.sums[p] = s;
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        uint64_t before = 0;
        int p = 0;
        while (p + 1 < parts && before + sh.sums[p] <= target) before += sh.sums[p++];
        sh.at = p;
        sh.found[0] = before;
      }
      __syncthreads();
      target -= sh.found[0];
      lo += sh.at * part;
      hi = (int)min((int64_t)lo + part, (int64_t)hi);
    }
    uint64_t s = 0;
    visit(lo, hi, threadIdx.x, kThreads, [&](float x, int col) { s += measure(x, col); });
    uint64_t upto = s;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const uint64_t o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 63) sh.red[w] = upto;
    if (threadIdx.x == 0) sh.at = hi - 1;
    __syncthreads();
    uint64_t before = upto - s;
    for (int k = 0; k < w; ++k) before += sh.red[k];
    if (before <= target && target < before + s) {
      uint64_t run = before;
      int at = -1;
      visit(lo, hi, threadIdx.x, kThreads, [&](float x, int col) {
        run += measure(x, col);
        if (at < 0 && run > target) at = col;
      });
      sh.at = at;
    }
    __syncthreads();
    return sh.at;
  }

  // The largest key such that measure over the entries with at least that key
  // reaches target (1 .. the row's total); `above`: over the larger ones, `here`:
  // over the entries of that key.
  template <class M>
  __device__ __forceinline__ uint32_t select(M&& measure, uint64_t target, uint64_t& above, uint64_t& here) const {
    uint32_t prefix = 0;
    above = 0;
    for (int shift = kBits - 8; shift >= 0; shift -= 8) {
      __syncthreads();
      for (int i = threadIdx.x; i < 256; i += kThreads) sh.sums[i] = 0;
      __syncthreads();
      sweep([&](float x, int col) {
        const uint32_t k = key(x);
        if ((uint64_t)k >> (shift + 8) == (uint64_t)prefix >> (shift + 8)) {
          const uint64_t v = measure(x, col);
          if (v != 0) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.sums[(k >> shift) & 255u]), (unsigned long long)v);
        }
      });
      __syncthreads();
      if (threadIdx.x < kWave) {  // lane l: digits 255 - 4 l down to 252 - 4 l
        const int lane = threadIdx.x;
        uint64_t s[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) mine += s[j] = sh.sums[255 - 4 * lane - j];
        uint64_t upto = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
          const uint64_t o = __shfl_up(upto, d);
          if (lane >= d) upto += o;
        }
        uint64_t before = above + upto - mine;
        if (before < target && (target <= before + mine || lane == kWave - 1)) {
          int j = 0;
          while (j < 3 && before + s[j] < target) before += s[j++];
          sh.found[0] = before;
          sh.found[1] = s[j];
          sh.at = 255 - 4 * lane - j;
        }
      }
      __syncthreads();
      above = sh.found[0];
      here = sh.found[1];
      prefix |= (uint32_t)sh.at << shift;
    }
    return prefix;
  }
};

template <typename T, int kThreads>
__device__ __forceinline__ void draw_row(const DrawArgs& a, int64_t r, typename RowDraw<T, kThreads>::Shared& sh) {
  using Row = RowDraw<T, kThreads>;
  const DrawSettings d = draw_settings(a, r);
  if (!draw_valid(d)) {
    if (threadIdx.x == 0) {
      report_error(a.err, VSD_DEVERR_SETTING_RANGE);
      draw_result(a, r, -1, 0.0f, 0);
    }
    return;
  }
  Row row{sh, static_cast<const T*>(a.Y) + r * a.ld, a.V, -INFINITY, 0.0, 1.0};
  float m = -INFINITY;
  uint64_t n = 0;  // entries, and (upper half) NaNs
  row.sweep([&](float x, int) {
    m = fmaxf(m, x);
    n += x == x ? 1ull : 1ull << 32;
  });
  n = row.total(n);
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) sh.redf[wave_id()] = m;
  __syncthreads();
  m = sh.redf[0];
  for (int k = 1; k < Row::kWaves; ++k) m = fmaxf(m, sh.redf[k]);
  if (n >> 32 != 0 || n == 0) {
    if (threadIdx.x == 0) draw_result(a, r, -1, n == 0 ? 0.0f : __builtin_nanf(""), 0);
    return;
  }
  row.m = m;
  if (d.temp == 0.0f) {
    const int tok = row.find_index([&](float x, int) { return x == m ? 1ull : 0ull; }, 0);
    if (threadIdx.x == 0) draw_result(a, r, tok, 0.0f, 1);
    return;
  }
  row.c = 1.4426950408889634074 / (double)d.temp;
  double z = 0.0;
  row.sweep([&](float x, int) { z += draw_weight(x, m, row.c); });
  z = row.total(z, sh.redd);
  const int e = 62 - (ilogb(z) + 1);
  row.scale = __builtin_ldexp(1.0, e);

  // the entries in play: larger than `least`, or equal to it up to index `last`
  uint32_t least = 0;
  int last = 0x7FFFFFFF;
  uint64_t above, here;
  auto in = [&](float x, int col) {
    const uint32_t k = Row::key(x);
    return k > least || (k == least && col <= last);
  };
  if (d.top_k > 0 && (uint64_t)d.top_k < n) {
    const uint32_t at = row.select([](float, int) { return 1ull; }, d.top_k, above, here);
    const uint64_t need = d.top_k - above;
    if (need < here)
      last = row.find_index([&](float x, int) { return Row::key(x) == at ? 1ull : 0ull; }, need - 1);
    least = at;
  }
  if (d.top_p < 1.0f) {
    uint64_t mass = 0;
    row.sweep([&](float x, int col) { mass += in(x, col) ? row.weight(x) : 0ull; });
    mass = row.total(mass);
    const uint64_t target = (uint64_t)__builtin_ceil((double)d.top_p * (double)mass);
    const uint32_t at = row.select([&](float x, int col) { return in(x, col) ? row.weight(x) : 0ull; }, target, above, here);
    const uint64_t each = row.weight(Row::value(at)), need = (target - above + each - 1) / each;
    if (need * each < here)
      last = row.find_index([&](float x, int col) { return Row::key(x) == at && in(x, col) ? 1ull : 0ull; }, need - 1);
    else if (at != least)
      last = 0x7FFFFFFF;
    least = at;
  }
  const double min_p = d.min_p;
  auto kept = [&](float x, int col) { return in(x, col) && draw_weight(x, m, row.c) >= min_p; };
  uint64_t mass = 0, count = 0;
  row.sweep([&](float x, int col) {
    if (kept(x, col)) {
      mass += row.weight(x);
      ++count;
    }
  });
  mass = row.total(mass);
  count = row.total(count);
  const int tok = row.find_index([&](float x, int col) { return kept(x, col) ? row.weight(x) : 0ull; },
                                 (uint64_t)((double)d.u * (double)mass));
  if (threadIdx.x == 0) {
    const float x = load1(row.Y + tok);
    const double lz = log((double)mass * __builtin_ldexp(1.0, -e));
    draw_result(a, r, tok, (float)((x == m ? 0.0 : ((double)x - (double)m) / (double)d.temp) - lz), (int32_t)count);
  }
}

template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void k_draw_row(DrawArgs a) {
  __shared__ typename RowDraw<T, kThreads>::Shared sh;
  draw_row<T, kThreads>(a, blockIdx.x, sh);
}

// ------------------------------------------------------------------ sweep ---
__device__ __forceinline__ float min3f(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float min8(const float (&v)[8]) {
  return min3f(min3f(v[0], v[1], v[2]), min3f(v[3], v[4], v[5]), min3f(v[6], v[7], v[7]));
}
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = (uint32_t)dpp_i<CTRL>((int)(uint32_t)u), hi = (uint32_t)dpp_i<CTRL>((int)(u >> 32));
  return __builtin_bit_cast(double, hi << 32 | lo);
}
__device__ __forceinline__ double lane_d(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = (uint32_t)lane_i((int)(uint32_t)u, l), hi = (uint32_t)lane_i((int)(u >> 32), l);
  return __builtin_bit_cast(double, hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum_d(double v) {
  v += dpp_d<kDppQuad1>(v);
  v += dpp_d<kDppQuad2>(v);
  v += dpp_d<kDppHalfMirror>(v);
  v += dpp_d<kDppMirror>(v);
  return (lane_d(v, 0) + lane_d(v, 16)) + (lane_d(v, 32) + lane_d(v, 48));
}
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp_f<kDppQuad1>(v));
  v = fmaxf(v, dpp_f<kDppQuad2>(v));
  v = fmaxf(v, dpp_f<kDppHalfMirror>(v));
  return fmaxf(v, dpp_f<kDppMirror>(v));
}

// Whether the rule needs the sum over all of the row's weights: the whole softmax, or
// top-p of it.  (With top-k the sum is over the kept entries, which are listed.)
__device__ __forceinline__ bool needs_sum(const DrawSettings& d) {
  return d.temp > 0.0f && d.top_k == 0 && (d.top_p < 1.0f || d.min_p == 0.0f);
}

constexpr int kLoads = kDrawSpan / 512;  // of 8 columns a lane

// (without sums 262 MB of fp32 rows in 40 us, 6.6 TB/s; with them 4096 x 128 256 bf16 in
// 395, which the weights' double-precision instructions take: the VALU issues in 95 % of the
// cycles, in 19 without them)
template <typename T>
__global__ __launch_bounds__(256) void k_draw_sweep(DrawArgs a) {
  const int lane = threadIdx.x & 63, tasks = (a.S + a.per - 1) / a.per;
  const int64_t task = (int64_t)blockIdx.x * 4 + wave_id();
  const int64_t r = task / tasks;
  if (task == 0 && lane == 0) *a.ntodo = 0;
  if (r >= a.R) return;
  const int first = (int)(task - r * tasks) * a.per, last = min(first + a.per, a.S);
  const DrawSettings d = draw_settings(a, r);
  const bool sums = needs_sum(d);
  const double c = sums ? 1.4426950408889634074 / (double)d.temp : 0.0;
  const T* Y = static_cast<const T*>(a.Y) + r * a.ld;
  auto load = [&](Raw8<T> (&q)[kLoads], int span) {
    const int base = span * kDrawSpan + lane * 8;
    if (span * kDrawSpan + kDrawSpan <= a.V) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) q[u].load(Y + base + u * 512);
    } else {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) load_cols(q[u], Y, base + u * 512, a.V);
    }
  };
  auto take = [&](const Raw8<T> (&q)[kLoads], int span) {
    float top = -INFINITY, low = INFINITY, gm = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      float x[8];
      q[u].get(x);
      const float t = max8(x);
      top = fmaxf(top, t);
      low = fminf(low, min8(x));
#pragma unroll
      for (int k = 0; k < 8; k += 2) nan |= __builtin_isunordered(x[k], x[k + 1]);
      const float g = row16_max(t);
      if ((lane & 15) == u) gm = g;
    }
    const float m = wave_max(top);
    int count = kDrawSpan;
    if (__any(low == -INFINITY)) {
      count = 0;
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float x[8];
        q[u].get(x);
#pragma unroll
        for (int k = 0; k < 8; ++k) count += __builtin_popcountll(__ballot(x[k] > -INFINITY));
      }
    }
    if (__any(nan)) count = -1;
    double s = 0.0;
    if (sums && m > -INFINITY) {
      const double md = m;
      auto sum = [&](auto&& weight) {
        double s2[2] = {0.0, 0.0};
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
          float x[8];
          q[u].get(x);
#pragma unroll
          for (int k = 0; k < 8; ++k) s2[k & 1] += weight(x[k]);
        }
        s = s2[0] + s2[1];
      };
      if (m == INFINITY)
        sum([&](float x) { return x == m ? 1.0 : 0.0; });
      else if (__all(((double)low - md) * c > -1000.0))
        sum([&](float x) { return exp2_64_near(((double)x - md) * c); });
      else
        sum([&](float x) { return exp2_64(((double)x - md) * c); });
      s = wave_sum_d(s);
    }
    const int64_t at = r * a.S + span;
    if ((lane & 15) < kLoads) a.group_max[at * 16 + (lane & 15) * 4 + (lane >> 4)] = gm;
    if (lane == 0) {
      a.span_max[at] = m;
      a.span_count[at] = count;
      a.span_sum[at] = s;
    }
  };
  static_assert(kDrawSpan / kDrawGroup == 16 && kLoads * 4 == 16, "sixteen groups of a span");
  Raw8<T> q[2][kLoads];
  load(q[0], first);
  for (int s = first; s < last; s += 2) {
    if (s + 1 < last) load(q[1], s + 1);
    take(q[0], s);
    if (s + 1 == last) break;
    if (s + 2 < last) load(q[0], s + 2);
    take(q[1], s + 1);
  }
}

// ----------------------------------------------------------------- finish ---
constexpr int kFinish = 256, kFinishWaves = kFinish / kWave;
// Listed entries.  Rows of 513 to 1024 columns, whose few groups bound little, are listed
// whole (us, 512 / 1024: 8192 rows of 1000 at T = 1.3, p = 0.99 548 / 137, later 101; 65 536 of 500
// 698 / 835, later 487).
constexpr int kCap = 512, kCapShort = 1024;
constexpr int kGroups = kDrawSpans * 16;
constexpr double kListScale = 4503599627370496.0;     // 2^52: a list's weights sum to at most 2^62
static_assert(kCapShort <= 1024 && kGroups <= 65536 && kDrawSpans == 2 * kWave, "");

template <int CTRL>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t u) {
  const uint64_t lo = (uint32_t)dpp_i<CTRL>((int)(uint32_t)u), hi = (uint32_t)dpp_i<CTRL>((int)(u >> 32));
  return hi << 32 | lo;
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t u, int l) {
  return (uint64_t)(uint32_t)lane_i((int)(u >> 32), l) << 32 | (uint32_t)lane_i((int)(uint32_t)u, l);
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
  v += dpp_u64<kDppQuad1>(v);
  v += dpp_u64<kDppQuad2>(v);
  v += dpp_u64<kDppHalfMirror>(v);
  v += dpp_u64<kDppMirror>(v);
  return (lane_u64(v, 0) + lane_u64(v, 16)) + (lane_u64(v, 32) + lane_u64(v, 48));
}

// Over a wavefront, by DPP (an LDS permute's latency six times over is what a chain of
// them would cost): the least, and sums of the lanes before (row_shr 1, 2, 4, 8, then the
// last lanes of the rows before).
__device__ __forceinline__ uint32_t wave_least(uint32_t v) {
  v = min(v, (uint32_t)dpp_i<kDppQuad1>((int)v));
  v = min(v, (uint32_t)dpp_i<kDppQuad2>((int)v));
  v = min(v, (uint32_t)dpp_i<kDppHalfMirror>((int)v));
  v = min(v, (uint32_t)dpp_i<kDppMirror>((int)v));
  return min(min((uint32_t)lane_i((int)v, 0), (uint32_t)lane_i((int)v, 16)),
             min((uint32_t)lane_i((int)v, 32), (uint32_t)lane_i((int)v, 48)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_zero(uint64_t u) {  // 0 where no lane is named
  const uint64_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
  const uint64_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xF, false);
  return hi << 32 | lo;
}
template <int CTRL, int ROWS, typename N>
__device__ __forceinline__ N dpp_add(N v) {
  return v + __builtin_bit_cast(N, dpp_zero<CTRL, ROWS>(__builtin_bit_cast(uint64_t, v)));
}
template <typename N>
__device__ __forceinline__ N wave_before(N v, N& all) {
  static_assert(sizeof(N) == 8, "");
  v = dpp_add<0x111, 0xF>(v);
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);  // row_bcast15 to rows 1 and 3
  v = dpp_add<0x143, 0xC>(v);  // row_bcast31 to rows 2 and 3
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  all = __builtin_bit_cast(N, lane_u64(u, 63));
  return __builtin_bit_cast(N, dpp_zero<0x138, 0xF>(u));  // wave_shr 1
}
// Sums and scans over a workgroup of kW wavefronts; `turn` alternates between two sets
// of words, so that one barrier a sum is enough.
template <int kW>
struct Block {
  uint64_t (*red)[3][kW];
  int turn;
  template <int N>
  __device__ __forceinline__ void sums(uint64_t (&v)[N]) {
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = wave_sum_u64(v[i]);
      if ((threadIdx.x & 63) == 0) red[turn][i][wave_id()] = v[i];
    }
    __syncthreads();
    // (a lane per wavefront: every wavefront reading all words held up the LDS)
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum_u64(lane < kW ? red[turn][i][lane] : 0ull);
  }
  __device__ __forceinline__ uint64_t sum(uint64_t v) {
    uint64_t s[1] = {v};
    sums(s);
    return s[0];
  }
  template <typename N>
  __device__ __forceinline__ N before(N v, N& all) {  // the sum over the threads before this one
    N mine;
    const N prev = wave_before(v, mine);
    const int lane = threadIdx.x & 63;
    turn ^= 1;
    N* const r = reinterpret_cast<N*>(red[turn][0]);
    if (lane == 0) r[wave_id()] = mine;
    __syncthreads();
    const N first = wave_before(lane < kW ? r[lane] : N(0), all);
    return __builtin_bit_cast(N, lane_u64(__builtin_bit_cast(uint64_t, first), wave_id())) + prev;
  }
  __device__ __forceinline__ uint32_t least(uint32_t v) {
    uint32_t lo = v, hi = 0;
    range(lo, hi);
    return lo;
  }
  // The smallest and the largest key (32 bits) of the threads' [lo, hi].
  __device__ __forceinline__ void range(uint32_t& lo, uint32_t& hi) {
    lo = wave_least(lo);
    uint32_t nhi = wave_least(~hi);
    const int lane = threadIdx.x & 63;
    turn ^= 1;
    if (lane == 0) red[turn][0][wave_id()] = (uint64_t)nhi << 32 | lo;
    __syncthreads();
    const uint64_t u = lane < kW ? red[turn][0][lane] : ~0ull;
    lo = wave_least((uint32_t)u);
    hi = ~wave_least((uint32_t)(u >> 32));
  }
  // The largest key in [lo, hi] such that measure(key), the sum over entries of at least
  // that key, reaches target (that of lo does): two bits of it a round.
  template <class M>
  __device__ __forceinline__ uint32_t largest(uint32_t lo, uint32_t hi, uint64_t target, M&& measure) {
    int bits = lo == hi ? 0 : 32 - __builtin_clz(lo ^ hi);
    uint32_t key = bits == 32 ? 0u : hi >> bits << bits;
    while (bits > 0) {
      bits = bits > 2 ? bits - 2 : 0;
      uint64_t s[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) s[i] = measure(key | (uint32_t)(i + 1) << bits);
      sums(s);
      key |= (uint32_t)(s[2] >= target ? 3 : s[1] >= target ? 2 : s[0] >= target ? 1 : 0) << bits;
    }
    return key;
  }
};

// A row's list: its columns in order, and the groups that they lie in.
template <int kCap>
struct FinishShared {
  int32_t col[kCap];
  uint16_t groups[kGroups];
};

// The largest key in [lo, hi] that reaches(key) (lo's does), bit by bit.
template <class F>
__device__ __forceinline__ uint32_t wave_largest(uint32_t lo, uint32_t hi, F&& reaches) {
  int bits = lo == hi ? 0 : 32 - __builtin_clz(lo ^ hi);
  uint32_t key = bits == 32 ? 0u : hi >> bits << bits;
#pragma unroll 1
  while (--bits >= 0) {
    const uint32_t t = key | 1u << bits;
    if (reaches(t)) key = t;
  }
  return key;
}

// One row by one wavefront (no barrier: what bounds it is how long the chain of its
// instructions takes); kPer groups a lane.  A workgroup of four wavefronts a row, its
// sums through LDS, took 24 us for 8 rows of 128 256 (k = 50, p = 0.9) and 119 for 4096 (p =
// 0.95); this 19 and 73 (8 rows of 256 000: 23; 32 groups a lane take 144 bytes of scratch).
template <typename T, int kPer, int kCap>
__global__ __launch_bounds__(kFinish) void k_draw_finish(DrawArgs a) {
  constexpr int kDown = sizeof(T) == 2 ? 16 : 0;  // (bf16: 16 bits of order)
  __shared__ FinishShared<kCap> all_rows[kFinishWaves];
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * kFinishWaves + wave_id();
  if (r >= a.R) return;
  FinishShared<kCap>& sh = all_rows[wave_id()];
  const T* Y = static_cast<const T*>(a.Y) + r * a.ld;
  const DrawSettings d = draw_settings(a, r);
  if (!draw_valid(d)) {
    if (lane == 0) {
      report_error(a.err, VSD_DEVERR_SETTING_RANGE);
      draw_result(a, r, -1, 0.0f, 0);
    }
    return;
  }
  auto key_of = [](float x) { return draw_order(x) >> kDown; };
  auto value_of = [](uint32_t k) {
    return draw_value(kDown == 0 || k >= 0x8000u ? k << kDown : k << kDown | 0xFFFFu);
  };
  // LDS written by some lanes is read by others of the wavefront
  auto settle = []() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  const int G = a.S * 16;
  // lane l: groups kPer l .. (keys; 0: no entry), spans 2 l and 2 l + 1
  uint32_t g[kPer];
  uint32_t low = 0xFFFFFFFFu, high = 0;
#pragma unroll
  for (int k = 0; k < kPer; k += 4) {
    const int at = lane * kPer + k;
    float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (at < G) v = *reinterpret_cast<const float4*>(a.group_max + r * G + at);
    const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g[k + i] = x[i] > -INFINITY ? key_of(x[i]) : 0u;
      low = min(low, g[k + i] - 1u);  // (none: the largest)
      high = max(high, g[k + i]);
    }
  }
  float span_max[2];
  uint64_t counts = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = 2 * lane + i;
    span_max[i] = s < a.S ? a.span_max[r * a.S + s] : -INFINITY;
    const int count = s < a.S ? a.span_count[r * a.S + s] : 0;
    counts += count < 0 ? 1ull << 40 : (uint64_t)count;
  }
  counts = wave_sum_u64(counts);
  const int n = (int)counts;
  if (counts == 0 || counts >> 40 != 0) {
    if (lane == 0) draw_result(a, r, -1, counts == 0 ? 0.0f : __builtin_nanf(""), 0);
    return;
  }
  low = wave_least(low) + 1u;
  high = ~wave_least(~high);
  const float m = value_of(high);
  if (d.temp == 0.0f) {
    uint32_t at = 0xFFFFFFFFu;
#pragma unroll
    for (int k = kPer - 1; k >= 0; --k)
      if (g[k] == high) at = (uint32_t)(lane * kPer + k);
    at = wave_least(at);
    uint32_t col = 0xFFFFFFFFu;
    if (lane < kDrawGroup / 8) {
      Raw8<T> q;
      float x[8];
      const int base = (int)at * kDrawGroup + lane * 8;
      load_cols(q, Y, base, a.V);
      q.get(x);
#pragma unroll
      for (int k = 7; k >= 0; --k)
        if (x[k] == m) col = (uint32_t)(base + k);
    }
    col = wave_least(col);
    if (lane == 0) draw_result(a, r, (int32_t)col, 0.0f, 1);
    return;
  }
  const double c = 1.4426950408889634074 / (double)d.temp, temp = d.temp;
  auto log_weight = [&](float x) { return x == m ? 0.0 : ((double)x - (double)m) / temp; };
  const bool by_k = d.top_k > 0 && d.top_k < n, by_p = d.top_p < 1.0f, by_m = d.min_p > 0.0f;
  double z = 0.0;  // the sum of all weights, where it is needed
  if (needs_sum(d)) {
    double mine[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      mine[i] = span_max[i] > -INFINITY ? a.span_sum[r * a.S + 2 * lane + i] * draw_weight(span_max[i], m, c) : 0.0;
    const double before = wave_before(mine[0] + mine[1], z);
    if (!by_p && !by_m) {
      // the whole softmax: the span, then its four rounds of 512 columns, then the column
      const double target = (double)d.u * z;
      const int which = draw_span(before, mine[0], mine[1], target);
      const uint32_t at = wave_least(which < 0 ? 0xFFFFFFFFu : (uint32_t)(2 * lane + which));
      double want = target - before - ((at & 1u) != 0u ? mine[0] : 0.0);
      want = lane_d(want, (int)(at >> 1));
      double passed = 0.0;
      int tok = -1, positive = -1;  // (positive: the last column of any weight, should roundings pass the span)
#pragma unroll 1
      for (int u = 0; u < kLoads && tok < 0; ++u) {
        const int base = (int)at * kDrawSpan + u * 512 + lane * 8;
        Raw8<T> q;
        float x[8];
        load_cols(q, Y, base, a.V);
        q.get(x);
        double w[8], sum = 0.0, all;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += w[k] = x[k] > -INFINITY ? draw_weight(x[k], m, c) : 0.0;
        double run = passed + wave_before(sum, all);
        uint32_t col = 0xFFFFFFFFu, some = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          run += w[k];
          if (w[k] > 0.0) {
            some = (uint32_t)(base + k) + 1u;
            if (col == 0xFFFFFFFFu && run > want) col = (uint32_t)(base + k);
          }
        }
        tok = (int)wave_least(col);
        some = ~wave_least(~some);
        if (some > 0) positive = (int)some - 1;
        passed += all;
      }
      if (tok < 0) tok = positive;
      if (lane == 0) {
        const float xt = load1(Y + tok);
        draw_result(a, r, tok, (float)(log_weight(xt) - log(z)), n);
      }
      return;
    }
  }
  // the bound of the list
  auto leave = [&]() {
    if (lane == 0) a.todo[atomicAdd(a.ntodo, 1)] = (int32_t)r;
  };
  float least = -INFINITY;
  bool min_bound = false;  // everything that min-p keeps is listed, maybe not all that top-p keeps
  if (n > kCap) {
    if (by_k) {
      if (d.top_k > kCap) return leave();
      auto count = [&](uint32_t at) {
        int s = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) s += __builtin_popcountll(__ballot(g[k] >= at));
        return s;
      };
      if (count(1u) < d.top_k) return leave();
      const uint32_t key = wave_largest(low, high, [&](uint32_t at) { return count(at) >= d.top_k; });
      least = value_of(key);
    } else if (by_p) {
      // (with d.top_k > 0, at least n, the sum was not formed)
      if (d.top_k > 0) return leave();
      // fp32 weights of the maxima, a little too small: enough for a bound
      uint32_t w[kPer];
      uint64_t all = 0;
      const float c32 = (float)c;
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const float x = value_of(g[k]);
        w[k] = g[k] > 0u ? (uint32_t)((x == m ? 1.0f : __builtin_amdgcn_exp2f((x - m) * c32)) * 0.9999f * 1073741824.0f) : 0u;
        all += w[k];
      }
      all = wave_sum_u64(all);
      const double goal = (double)d.top_p * z * 1073741824.0 + 1.0;
      if ((double)all < goal) {
        if (!by_m) return leave();
      } else {
        const uint64_t target = (uint64_t)goal;
        least = value_of(wave_largest(low, high, [&](uint32_t at) {
          uint64_t s = 0;
#pragma unroll
          for (int k = 0; k < kPer; ++k) s += g[k] >= at ? w[k] : 0u;
          return wave_sum_u64(s) >= target;
        }));
      }
    } else if (!by_m) {
      return leave();  // (top-k of at least n entries and nothing else)
    }
    if (by_m && !(by_k && by_p)) {
      // w >= min_p: x >= m + T log(min_p), less what the roundings may be off by
      const double at = (double)m + temp * log((double)d.min_p);
      const float bound = (float)(at - 1e-6 * (fabs((double)m) + fabs(at)) - 1e-30);
      if (m < INFINITY && bound > least) {
        least = bound;
        min_bound = true;
      }
    }
  }
  // the groups that reach it, and their entries, both in index order
  const uint32_t least_key = least > -INFINITY ? key_of(least) : 1u;
  int ngroups;
  {
    uint64_t mine = 0, all;
#pragma unroll
    for (int k = 0; k < kPer; ++k) mine += g[k] >= least_key ? 1 : 0;
    int at = (int)wave_before(mine, all);
    ngroups = (int)all;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (g[k] >= least_key) sh.groups[at++] = (uint16_t)(lane * kPer + k);
    settle();
  }
  constexpr int kSets = 8, kSet = kWave / 16;  // a set: 4 groups, a lane eight columns
  int listed = 0;
#pragma unroll 1
  for (int first = 0; first < ngroups; first += kSets * kSet) {
    Raw8<T> q[kSets];
    int base[kSets];
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      const int i = first + s * kSet + (lane >> 4);
      base[s] = i < ngroups ? (int)sh.groups[i] * kDrawGroup + (lane & 15) * 8 : a.V;
      load_cols(q[s], Y, base[s], a.V);
    }
    uint64_t reach = 0, counts[2] = {0, 0}, all[2], before[2];  // a bit per entry; 16 bits a set
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      float x[8];
      q[s].get(x);
      uint32_t bits = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) bits |= x[k] >= least && x[k] > -INFINITY ? 1u << k : 0u;
      reach |= (uint64_t)bits << (8 * s);
      counts[s >> 2] |= (uint64_t)__builtin_popcount(bits) << (16 * (s & 3));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) before[i] = wave_before(counts[i], all[i]);
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      int at = listed + (int)((before[s >> 2] >> (16 * (s & 3))) & 0xFFFFu);
      uint32_t bits = (uint32_t)(reach >> (8 * s)) & 0xFFu;
      while (bits != 0u) {
        if (at < kCap) sh.col[at] = base[s] + __builtin_ctz(bits);
        ++at;
        bits &= bits - 1u;
      }
      listed += (int)((all[s >> 2] >> (16 * (s & 3))) & 0xFFFFu);
    }
    if (listed > kCap) return leave();
  }
  settle();
  // entry 64 j + lane of the list: column, key, weight; `in`: in play, a bit each
  constexpr int kMine = kCap / kWave;
  int32_t col[kMine];
  uint32_t key[kMine], in = 0, enough = 0;
  uint64_t w[kMine];
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = j * kWave + lane;
    key[j] = 0;
    w[j] = 0;
    if (j * kWave >= listed) continue;  // (of the whole wavefront, here and below)
    if (i < listed) {
      col[j] = sh.col[i];
      key[j] = key_of(load1(Y + col[j]));
      in |= 1u << j;
    }
  }
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    if (j * kWave >= listed) continue;
    if ((in >> j & 1u) == 0u) continue;
    const double v = draw_weight(value_of(key[j]), m, c);
    w[j] = (uint64_t)(v * kListScale + 0.5);
    enough |= v >= (double)d.min_p ? 1u << j : 0u;
    kmin = min(kmin, key[j]);
    kmax = max(kmax, key[j]);
  }
  kmin = wave_least(kmin);
  kmax = ~wave_least(~kmax);
  auto mass_of = [&](uint32_t at) {  // of the entries in play of at least that key
    uint64_t s = 0;
#pragma unroll
    for (int j = 0; j < kMine; ++j)
      if (j * kWave < listed) s += (in >> j & 1u) != 0u && key[j] >= at ? w[j] : 0;
    return wave_sum_u64(s);
  };
  auto count_of = [&](uint32_t at) {
    int s = 0;
#pragma unroll
    for (int j = 0; j < kMine; ++j)
      if (j * kWave < listed) s += __builtin_popcountll(__ballot((in >> j & 1u) != 0u && key[j] >= at));
    return s;
  };
  // keeps of the entries in play those above `at`, and the first `ties` of that key
  auto cut = [&](uint32_t at, uint64_t ties) {
    uint64_t seen = 0;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      if (j * kWave >= listed) continue;
      const bool mine = (in >> j & 1u) != 0u, equal = mine && key[j] == at;
      const uint64_t who = __ballot(equal);
      const uint64_t rank = seen + (uint64_t)__builtin_popcountll(who & ((1ull << lane) - 1));
      if (mine && !(key[j] > at || (equal && rank < ties))) in &= ~(1u << j);
      seen += (uint64_t)__builtin_popcountll(who);
    }
  };
  if (by_k && listed > d.top_k) {
    const uint32_t at = wave_largest(kmin, kmax, [&](uint32_t b) { return count_of(b) >= d.top_k; });
    cut(at, (uint64_t)(d.top_k - count_of(at + 1u)));
  }
  if (by_p) {
    const uint64_t all = mass_of(0u);
    const double whole = by_k || n <= kCap ? (double)all : z * kListScale;
    const double goal = __builtin_ceil((double)d.top_p * whole);
    if (goal <= (double)all) {
      const uint64_t target = (uint64_t)goal;
      const uint32_t at = wave_largest(kmin, kmax, [&](uint32_t b) { return mass_of(b) >= target; });
      const uint64_t each = (uint64_t)(draw_weight(value_of(at), m, c) * kListScale + 0.5);
      cut(at, (target - mass_of(at + 1u) + each - 1) / each);
    } else if (!min_bound) {
      return leave();
    }
  }
  in &= enough;
  const int kept = count_of(0u);
  const uint64_t mass = mass_of(0u);
  // the entry in which the mass passes u of it
  const uint64_t target = (uint64_t)((double)d.u * (double)mass);
  uint64_t passed = 0;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    if (j * kWave >= listed) continue;
    const uint64_t mine = (in >> j & 1u) != 0u ? w[j] : 0;
    uint64_t all;
    const uint64_t before = passed + wave_before(mine, all);
    if (before <= target && target < before + mine)
      draw_result(a, r, col[j], (float)(log_weight(value_of(key[j])) - log((double)mass / kListScale)), kept);
    passed += all;
  }
}

// ------------------------------------------------------------- flat rows ---
// A row whose kept entries do not fit a wavefront's list: two sweeps by a workgroup.  The
// first (top-p) sums fp32 weights, as integers, in 2048 bins of equal width between the
// largest logit and one below which less than 1 - p of the mass can lie; the bins within
// 1e-4 of p Z are taken for the border's.  Each weight is rounded to an integer, so they
// may be off by n / 2^30 of Z (2.4e-4 at 262 144 columns, were all rounded one way): a
// border elsewhere is noticed from the exact sums, and the row left to draw_row.  (Top-k up
// to 2048: counts, and the bins of the first k entries.)  The second sweep forms the
// weights in 64 bits: of the entries above those bins per 512 columns, and the entries in
// them go to a list, where the border is found as in k_draw_finish.
constexpr int kBins = 2048, kFlatCap = 2048, kPieces = kDrawSpans * kDrawSpan / 512;
template <int kThreads>
struct FlatShared {
  union {
    uint32_t bins[kBins];
    struct {
      float x[kFlatCap];
      int32_t col[kFlatCap];
    } list;
  };
  uint64_t pieces[kPieces];  // kept mass of every 512 columns
  uint64_t red[2][3][kThreads / kWave];
  uint64_t target;
  int32_t n, at;
};

// False: left to draw_row.
template <typename T, int kThreads>
__device__ __forceinline__ bool draw_flat(const DrawArgs& a, int64_t r, FlatShared<kThreads>& sh) {
  constexpr int kFlatWaves = kThreads / kWave, kFlatMine = kFlatCap / kThreads, kMyBins = kBins / kThreads;
  constexpr int kDown = sizeof(T) == 2 ? 16 : 0;
  const DrawSettings d = draw_settings(a, r);
  Block<kFlatWaves> blk{sh.red, 0};
  const int t = threadIdx.x, lane = t & 63, wave = wave_id(), V = a.V;
  const T* Y = static_cast<const T*>(a.Y) + r * a.ld;
  auto key_of = [](float x) { return draw_order(x) >> kDown; };
  const bool span = t < a.S;
  const float span_max = span ? a.span_max[r * a.S + t] : -INFINITY;
  uint32_t lo = draw_order(span_max), hi = lo;
  if (!span) lo = 0xFFFFFFFFu, hi = 0;
  blk.range(lo, hi);
  const float m = draw_value(hi);
  const double c = 1.4426950408889634074 / (double)d.temp, temp = d.temp;
  const uint64_t n = blk.sum(span ? (uint64_t)a.span_count[r * a.S + t] : 0);
  const bool by_p = d.top_p < 1.0f, by_k = d.top_k > 0;
  if (by_k && ((uint64_t)d.top_k >= n || d.top_k > kFlatCap)) return false;
  double z = by_k ? (double)kFlatCap : (double)n;  // (at least the mass of what may be kept: sets the integers' scale)
  if (by_p && !by_k) (void)blk.before(span && span_max > -INFINITY ? a.span_sum[r * a.S + t] * draw_weight(span_max, m, c) : 0.0, z);
  const int e = 62 - (ilogb(z) + 1);
  const double scale = __builtin_ldexp(1.0, e), min_p = d.min_p;
  const double goal = __builtin_ceil((double)d.top_p * z * scale);

  float inv = 0.0f;  // bins: (m - x) inv
  const float c32 = (float)c;
  auto bin_of = [&](float x) {  // (the largest's difference to itself is 0 also where it is infinite)
    return x == m ? 0u : (uint32_t)fminf((m - x) * inv, (float)(kBins - 1));
  };
  int first = kBins, last = -1;  // the bins whose entries are listed
  for (int i = t; i < kPieces; i += kThreads) sh.pieces[i] = 0;
  if (t == 0) sh.n = 0;
  if (by_p || by_k) {
    // depth: top-p, as above; top-k, to as far below the least of the groups' maxima as
    // that lies below the largest logit (a border further down is draw_row's)
    double depth;
    if (by_k) {
      float low = INFINITY;
      for (int i = t; i < a.S * 16; i += kThreads) {
        const float g = a.group_max[r * a.S * 16 + i];
        if (g > -INFINITY) low = fminf(low, g);
      }
      uint32_t low_key = draw_order(low), high_key = 0;
      blk.range(low_key, high_key);
      depth = fmax(2.0 * ((double)m - (double)draw_value(low_key)), 1e-30);
    } else {
      depth = fmax(-temp * log((1.0 - (double)d.top_p) * z / (double)n), 1e-30);
    }
    inv = (float)fmin((kBins - 1) / depth, 3e38);
    const float bin_scale = by_k ? 1.0f : __builtin_ldexpf(1.0f, 30 - (ilogb(z) + 1));  // (weights together: below 2^31)
    for (int i = t; i < kBins; i += kThreads) sh.bins[i] = 0u;
    __syncthreads();
    Raw8<T> q;
    load_cols(q, Y, t * 8, V);
#pragma unroll 1
    for (int base = t * 8; base < V; base += kThreads * 8) {
      float x[8];
      q.get(x);
      load_cols(q, Y, min(base + kThreads * 8, V), V);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t b = bin_of(x[k]);  // (the last one holds all the rest: not needed, and one address for most lanes)
        const float w = by_k || x[k] == m ? 1.0f : __builtin_amdgcn_exp2f((x[k] - m) * c32);
        if (b < kBins - 1) atomicAdd(&sh.bins[b], (uint32_t)fmaf(w, bin_scale, 0.5f));
      }
    }
    __syncthreads();
    double mine[kMyBins], sum = 0.0, all;
#pragma unroll
    for (int i = 0; i < kMyBins; ++i) sum += mine[i] = (double)sh.bins[kMyBins * t + i];
    double run = blk.before(sum, all);
    // (top-k: every entry from the largest to the bin that completes the k)
    const double want = by_k ? (double)d.top_k : (double)d.top_p * z * (double)bin_scale;
    uint32_t b1 = 0xFFFFFFFFu, b2 = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < kMyBins; ++i) {
      run += mine[i];
      if (b1 == 0xFFFFFFFFu && run >= want * (by_k ? 1.0 : 1.0 - 1e-4)) b1 = (uint32_t)(kMyBins * t + i);
      if (b2 == 0xFFFFFFFFu && run >= want * (by_k ? 1.0 : 1.0 + 1e-4)) b2 = (uint32_t)(kMyBins * t + i);
    }
    b1 = blk.least(b1);
    b2 = blk.least(b2);
    if (b2 >= kBins - 1) return false;
    first = by_k ? 0 : (int)b1;
    last = (int)b2;
  }
  // min-p: entries far below the bound are not weighed
  const float bound = min_p > 0.0 && m < INFINITY
                          ? (float)((double)m + temp * log(min_p) -
                                    1e-6 * (fabs((double)m) + fabs((double)m + temp * log(min_p))) - 1e-30)
                          : -INFINITY;
  auto weigh = [&](float x, double& w) {
    w = draw_weight(x, m, c);
    return (uint64_t)(w * scale + 0.5);
  };
  __syncthreads();
  uint64_t above = 0, count = 0;
  const int pieces = (V + 511) / 512;
  Raw8<T> q;
  load_cols(q, Y, wave * 512 + lane * 8, V);
#pragma unroll 1
  for (int p = wave; p < pieces; p += kFlatWaves) {
    float x[8];
    q.get(x);
    const int base = p * 512 + lane * 8;
    load_cols(q, Y, min(base + kFlatWaves * 512, V), V);
    uint32_t over = 0, at_border = 0;  // entries above the border's bins, and in them
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      bool is_over = x[k] > -INFINITY && x[k] >= bound, is_at = false;
      if (by_p || by_k) {
        const int b = (int)bin_of(x[k]);
        is_at = x[k] > -INFINITY && b >= first && b <= last;
        is_over = x[k] > -INFINITY && b < first;
      }
      over |= is_over ? 1u << k : 0u;
      at_border |= is_at ? 1u << k : 0u;
    }
    uint64_t mass = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (!__any((over >> k & 1u) != 0u)) continue;
      double w;
      const uint64_t W = (over >> k & 1u) != 0u ? weigh(x[k], w) : 0;
      above += W;
      const bool keeps = (over >> k & 1u) != 0u && w >= min_p;
      mass += keeps ? W : 0;
      count += keeps ? 1 : 0;
    }
    if (__any(at_border != 0u)) {
      uint64_t all;
      int at = (int)wave_before((uint64_t)__builtin_popcount(at_border), all);
      int from = 0;
      if (lane == 0) from = atomicAdd(&sh.n, (int)all);
      at += __builtin_amdgcn_readfirstlane(from);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if ((at_border >> k & 1u) != 0u) {
          if (at < kFlatCap) {
            sh.list.x[at] = x[k];
            sh.list.col[at] = base + k;
          }
          ++at;
        }
    }
    mass = wave_sum_u64(mass);
    if (lane == 0) sh.pieces[p] = mass;
  }
  __syncthreads();
  const int listed = sh.n;
  if (listed > kFlatCap) return false;
  uint32_t least = 0;  // the smallest kept key of the list, and the last column with it
  int limit = 0x7FFFFFFF;
  if (by_p || by_k) {
    above = blk.sum(above);
    float x[kFlatMine];
    uint32_t key[kFlatMine];
    int col[kFlatMine];
    uint64_t w[kFlatMine];
    bool enough[kFlatMine], in[kFlatMine];
    uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
#pragma unroll
    for (int k = 0; k < kFlatMine; ++k) {
      const int i = t * kFlatMine + k;
      in[k] = i < listed;
      x[k] = in[k] ? sh.list.x[i] : -INFINITY;
      col[k] = in[k] ? sh.list.col[i] : 0;
      key[k] = key_of(x[k]);
      double v = 0.0;
      w[k] = in[k] ? weigh(x[k], v) : 0;
      enough[k] = v >= min_p;
      if (in[k]) {
        kmin = min(kmin, key[k]);
        kmax = max(kmax, key[k]);
      }
    }
    blk.range(kmin, kmax);
    auto over = [&](auto&& g) {
      uint64_t s = 0;
#pragma unroll
      for (int k = 0; k < kFlatMine; ++k) s += in[k] ? g(k) : 0ull;
      return s;
    };
    // keeps the entries above `least` and the first `ties` of that key (of `have`)
    auto cut = [&](uint64_t ties, uint64_t have) {
      limit = 0x7FFFFFFF;
      if (ties < have) {  // their columns: the largest of reversed ones
        const uint32_t top = (uint32_t)V;
        limit = (int)(top - blk.largest(0, top, ties, [&](uint32_t b) {
                        return over([&](int k) { return key[k] == least && top - (uint32_t)col[k] >= b ? 1ull : 0ull; });
                      }));
      }
#pragma unroll
      for (int k = 0; k < kFlatMine; ++k) in[k] = in[k] && (key[k] > least || (key[k] == least && col[k] <= limit));
    };
    if (by_k) {
      auto count_of = [&](uint32_t b) { return over([&](int k) { return key[k] >= b ? 1ull : 0ull; }); };
      least = blk.largest(kmin, kmax, d.top_k, count_of);
      uint64_t s[2] = {count_of(least + 1u), count_of(least)};
      blk.sums(s);
      cut((uint64_t)d.top_k - s[0], s[1] - s[0]);
    }
    if (by_p) {
      const uint64_t listed_mass = blk.sum(over([&](int k) { return w[k]; }));
      const uint64_t target = (uint64_t)(by_k ? __builtin_ceil((double)d.top_p * (double)listed_mass) : goal);
      if (above >= target || above + listed_mass < target) return false;  // (the border is elsewhere)
      const uint64_t need = target - above;
      auto mass_of = [&](uint32_t b) { return over([&](int k) { return key[k] >= b ? w[k] : 0ull; }); };
      const uint32_t before = least;
      const int limit_before = limit;
      least = blk.largest(kmin, kmax, need, mass_of);
      uint64_t s[2] = {mass_of(least + 1u), mass_of(least)};
      blk.sums(s);
      double v;
      const uint64_t each = weigh(draw_value(kDown == 0 || least >= 0x8000u ? least << kDown : least << kDown | 0xFFFFu), v);
      cut((need - s[0] + each - 1) / each, (s[1] - s[0]) / each);
      if (least == before) limit = min(limit, limit_before);
    }
#pragma unroll
    for (int k = 0; k < kFlatMine; ++k)
      if (in[k] && enough[k]) {
        atomicAdd(reinterpret_cast<unsigned long long*>(&sh.pieces[col[k] >> 9]), (unsigned long long)w[k]);
        ++count;
      }
    __syncthreads();
  }
  count = blk.sum(count);
  const uint64_t mine = t < pieces ? sh.pieces[t] : 0;
  uint64_t mass;
  const uint64_t before = blk.before(mine, mass);
  const uint64_t target = (uint64_t)((double)d.u * (double)mass);
  if (before <= target && target < before + mine) {
    sh.at = t;
    sh.target = target - before;
  }
  __syncthreads();
  if (wave > 0) return true;
  float x[8];
  const int base = sh.at * 512 + lane * 8;
  load_cols(q, Y, base, V);
  q.get(x);
  uint64_t w[8], sum = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    w[k] = 0;
    if (!(x[k] > -INFINITY)) continue;
    if (by_p || by_k) {
      const int b = (int)bin_of(x[k]);
      const uint32_t key = key_of(x[k]);
      if (b > last || (b >= first && !(key > least || (key == least && base + k <= limit)))) continue;
    } else if (x[k] < bound) {
      continue;
    }
    double v;
    const uint64_t W = weigh(x[k], v);
    if (v >= min_p) sum += w[k] = W;
  }
  uint64_t run = sum;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const uint64_t o = __shfl_up(run, s);
    if (lane >= s) run += o;
  }
  run -= sum;
  const uint64_t want = sh.target;
  bool found = false;
  if (run <= want && want < run + sum) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      run += w[k];
      if (!found && run > want) {
        found = true;
        const double lw = x[k] == m ? 0.0 : ((double)x[k] - (double)m) / temp;
        draw_result(a, r, base + k, (float)(lw - log((double)mass * __builtin_ldexp(1.0, -e))), (int32_t)count);
      }
    }
  }
  return true;
}

// The rows that were left.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void k_draw_left(DrawArgs a) {
  __shared__ union {
    FlatShared<kThreads> flat;
    typename RowDraw<T, kThreads>::Shared row;
  } sh;
  const int64_t n = *a.ntodo;
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int64_t r = a.todo[i];
    if (!draw_flat<T, kThreads>(a, r, sh.flat)) {
      __syncthreads();
      draw_row<T, kThreads>(a, r, sh.row);
    }
    __syncthreads();
  }
}
// Columns up to which 256 threads take such a row, several rows to a CU (us, 1024 / 256
// threads, p = 0.99 at T = 1.3: 8192 rows of 3000 1070 / 571, 4000 of 12 000 640 / 383).
constexpr int kLeftShort = 16384;

template <typename T>
hipError_t launch_t(DrawArgs a, hipStream_t s) {
  if (a.todo == nullptr) {  // (more columns than the records are for)
    hipLaunchKernelGGL((k_draw_row<T, 1024>), dim3((unsigned)a.R), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  const int64_t waves = a.R * ((a.S + a.per - 1) / a.per);
  hipLaunchKernelGGL((k_draw_sweep<T>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a);
  const dim3 rows((unsigned)((a.R + kFinishWaves - 1) / kFinishWaves));
  if (a.V > kCap && a.V <= kCapShort)
    hipLaunchKernelGGL((k_draw_finish<T, 4, kCapShort>), rows, dim3(kFinish), 0, s, a);
  else if (a.S <= 16)
    hipLaunchKernelGGL((k_draw_finish<T, 4, kCap>), rows, dim3(kFinish), 0, s, a);
  else if (a.S <= 64)
    hipLaunchKernelGGL((k_draw_finish<T, 16, kCap>), rows, dim3(kFinish), 0, s, a);
  else
    hipLaunchKernelGGL((k_draw_finish<T, 32, kCap>), rows, dim3(kFinish), 0, s, a);
  // (a row of kCapShort columns at most fits its list)
  if (a.V > kLeftShort)
    hipLaunchKernelGGL((k_draw_left<T, 1024>), dim3((unsigned)(a.R < 512 ? a.R : 512)), dim3(1024), 0, s, a);
  else if (a.V > kCapShort)
    hipLaunchKernelGGL((k_draw_left<T, 256>), dim3((unsigned)(a.R < 2048 ? a.R : 2048)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_draw(DrawArgs a, bool bf16, hipStream_t s) {
  if (a.todo != nullptr) {
    // spans a wavefront sweeps: one until the chip is full several times over
    a.per = 1;
    while (a.per < 16 && a.R * ((a.S + a.per - 1) / a.per) > 32768) a.per *= 2;
  }
  return bf16 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace vsd
