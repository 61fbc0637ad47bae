// Weights of the filtered draws (vsd_sample_rows) in 64 bits.
//
// A weight w = exp((x - M) / T) <= 1 is formed in double precision (relative error
// about 1e-14: what a border can be off by) and then held as an integer W =
// round(w 2^e), e such that a row's total stays below 2^63: sums of integers do
// not depend on their order, so neither the number of threads nor the order of
// atomics reaches a result.
#pragma once

#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

// 2^t for t <= 0: t = n + f with |f| <= 1/2, 2^f by the exponential's series in f
// ln 2 through the 11th power (the next term is below 7e-15).  (double FMAs issue at
// the rate of fp32 ones on this chip.)
__device__ __forceinline__ double exp2_64(double t) {
  t = __builtin_fmax(t, -1060.0);
  const double n = __builtin_rint(t), f = t - n;
  double p = 4.4455382718708114976e-10;                 // ln2^11 / 11!
  p = __builtin_fma(p, f, 7.0549116208011233299e-09);
  p = __builtin_fma(p, f, 1.0178086009239699728e-07);
  p = __builtin_fma(p, f, 1.3215486790144309488e-06);
  p = __builtin_fma(p, f, 1.5252733804059840280e-05);
  p = __builtin_fma(p, f, 1.5403530393381609954e-04);
  p = __builtin_fma(p, f, 1.3333558146428443423e-03);
  p = __builtin_fma(p, f, 9.6181291076284771619e-03);
  p = __builtin_fma(p, f, 5.5504108664821579953e-02);
  p = __builtin_fma(p, f, 2.4022650695910071233e-01);
  p = __builtin_fma(p, f, 6.9314718055994530942e-01);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)n);
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
