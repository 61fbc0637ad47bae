// One token per row under the deployed rule: temperature, top-k, top-p, min-p and
// a given random number (vsd_sample_rows).
//
// One workgroup per row, sweeping it several times: the largest entry; the sum of
// the weights, which sets their integer scale; for top-k and top-p the entry where
// the count or the mass reaches its target, 8 bits of its value a sweep from
// histograms of integers in LDS, and among equal entries by index; the kept
// entries' mass; and the index where the mass up to it passes u Z.
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
__global__ __launch_bounds__(kThreads) void k_draw_row(DrawArgs a) {
  using Row = RowDraw<T, kThreads>;
  __shared__ typename Row::Shared sh;
  const int64_t r = blockIdx.x;
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

template <typename T>
hipError_t launch_t(const DrawArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.R);
  if (a.V <= 4096)
    hipLaunchKernelGGL((k_draw_row<T, 256>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_draw_row<T, 1024>), grid, dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_draw(const DrawArgs& a, bool bf16, hipStream_t s) {
  return bf16 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
}

}  // namespace vsd
