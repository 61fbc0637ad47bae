// Weights of the filtered draws (vsd_sample_rows) in 64 bits.
//
// A weight w = exp((x - M) / T) <= 1 is formed in double precision (relative error 2e-14,
// in a whole row's sum 1e-12: what a border can be off by) and then held as an integer W =
// round(w 2^e), e such that a row's total stays below 2^63: sums of integers do
// not depend on their order, so neither the number of threads nor the order of
// atomics reaches a result.
#pragma once

#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

// 2^t for t <= 0: t = n + f with |f| <= 1/2, 2^f by the polynomial of degree 9 with
// constant term 1 (equal logits' sums are exact) whose largest relative error there is
// least, 1.5e-14.  (double FMAs issue at the rate of fp32 ones on this chip.)
__device__ __forceinline__ double exp2_64(double t) {
  t = __builtin_fmax(t, -1100.0);  // (2^-1100 is 0 here: u = 0 draws no finite logit of a row with +inf)
  const double n = __builtin_rint(t), f = t - n;
  double p = 0x1.b3de2fe9dfa6cp-24;
  p = __builtin_fma(p, f, 0x1.63e6965b042a6p-20);
  p = __builtin_fma(p, f, 0x1.ffce2fc22b257p-17);
  p = __builtin_fma(p, f, 0x1.430897f3391fap-13);
  p = __builtin_fma(p, f, 0x1.5d87fd93880d1p-10);
  p = __builtin_fma(p, f, 0x1.3b2ab72412209p-7);
  p = __builtin_fma(p, f, 0x1.c6b08d70c8812p-5);
  p = __builtin_fma(p, f, 0x1.ebfbdff81be06p-3);
  p = __builtin_fma(p, f, 0x1.62e42fefa37d1p-1);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)n);
}
// The same for -1000 < t <= 0 in five operations less: the rounding and the exponent by
// adding 1.5 2^52 (whose low word then is n), degree 8 (8.2e-13).
__device__ __forceinline__ double exp2_64_near(double t) {
  constexpr double kRound = 6755399441055744.0;
  const double r = t + kRound, f = t - (r - kRound);
  double p = 0x1.61c4f0e0d4891p-20;
  p = __builtin_fma(p, f, 0x1.00d85347934b4p-16);
  p = __builtin_fma(p, f, 0x1.430aa882d82b1p-13);
  p = __builtin_fma(p, f, 0x1.5d874d06f3adfp-10);
  p = __builtin_fma(p, f, 0x1.3b2ab5ed6f95bp-7);
  p = __builtin_fma(p, f, 0x1.c6b08dced3617p-5);
  p = __builtin_fma(p, f, 0x1.ebfbdff8ede89p-3);
  p = __builtin_fma(p, f, 0x1.62e42fef89d1ep-1);
  p = __builtin_fma(p, f, 1.0);
  const uint64_t u = __builtin_bit_cast(uint64_t, p);
  uint32_t hi;  // (written in C++ the shift and the addition become four 64-bit operations)
  asm("v_lshl_add_u32 %0, %1, 20, %2" : "=v"(hi) : "v"((uint32_t)__builtin_bit_cast(uint64_t, r)), "v"((uint32_t)(u >> 32)));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)u);
}

// The weight of logit x in a row whose largest is m (c = log2(e) / T); equal
// logits weigh 1 also where both are infinite.
__device__ __forceinline__ double draw_weight(float x, float m, double c) {
  return x == m ? 1.0 : exp2_64(((double)x - (double)m) * c);
}

// A value as an integer in the same order (-0 = +0), and back.
__device__ __forceinline__ uint32_t draw_order(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u & 0x80000000u) != 0u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float draw_value(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) != 0u ? o & 0x7FFFFFFFu : ~o);
}

struct DrawSettings {
  float temp, top_p, min_p, u;
  int32_t top_k;
};
__device__ __forceinline__ DrawSettings draw_settings(const DrawArgs& a, int64_t r) {
  DrawSettings d;
  d.temp = a.row_temp != nullptr ? a.row_temp[r] : a.temp;
  d.top_k = a.row_top_k != nullptr ? a.row_top_k[r] : a.top_k;
  d.top_p = a.row_top_p != nullptr ? a.row_top_p[r] : a.top_p;
  d.min_p = a.row_min_p != nullptr ? a.row_min_p[r] : a.min_p;
  d.u = a.u[r];
  return d;
}
__device__ __forceinline__ bool draw_valid(const DrawSettings& d) {
  return (d.temp == 0.0f || (d.temp >= 1e-30f && d.temp <= 1e30f)) && d.top_k >= 0 && d.top_p > 0.0f &&
         d.top_p <= 1.0f && d.min_p >= 0.0f && d.min_p <= 1.0f && d.u >= 0.0f && d.u < 1.0f;
}
__device__ __forceinline__ void draw_result(const DrawArgs& a, int64_t r, int32_t tok, float log_prob, int32_t kept) {
  a.tok[r] = tok;
  if (a.log_prob != nullptr) a.log_prob[r] = log_prob;
  if (a.kept != nullptr) a.kept[r] = kept;
}

}  // namespace vsd
