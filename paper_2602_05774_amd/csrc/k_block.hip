// Products of 8-bit block matrices (vsd_block_product): out = a b^T, a scale per
// row and 128 columns of a, per 1 or 128 rows and 128 columns of b.
//
// The matrix instructions on 8-bit values align eight products at a time to the
// largest of their exponents and cut them 13 bits below it (measured: 448 x 448 + 18
// x 18 gives 201 024, not 201 028), in every shape that they have: sums of random
// values are off by some 1e-5 of themselves.  That is nothing next to a bf16
// result's rounding (2^-8), but fp32 results would lose half their bits.  So bf16
// results come from these instructions and fp32 results from the bf16 ones, which
// sum in fp32, at half the rate: an e4m3 value is a bf16 value exactly.
//
// A wavefront owns a 32 x 32 tile and walks the blocks: each block's product is
// formed on the matrix cores from zero and added, times its scales, in fp32.
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Eight of the type's values (two words) in bf16.
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// sum_k a[m][k] b[n][k] over 64 values of k; lane l holds 32 of row l % 32 of both
// operands, the same ones of each (the order of a sum's terms is free), and
// column l % 32, rows 8 (e / 4) + 4 (l / 32) + e % 4 of the result.  (Constant zeros
// as scales select the form without them.)
__device__ __forceinline__ f32x16 mfma8(const i32x8& a, const i32x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}
// The same with fp32's accuracy.
__device__ __forceinline__ f32x16 mfma8_exact(const i32x8& a, const i32x8& b, f32x16 c) {
#pragma unroll
  for (int k = 0; k < 8; k += 2)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(a[k], a[k + 1]), widen(b[k], b[k + 1]), c, 0, 0, 0);
  return c;
}
template <bool EXACT>
__device__ __forceinline__ f32x16 block_step(const i32x8& a, const i32x8& b, const f32x16& c) {
  if constexpr (EXACT)
    return mfma8_exact(a, b, c);
  else
    return mfma8(a, b, c);
}

__device__ __forceinline__ i32x8 load32(const uint8_t* p) {
  const int4 u = reinterpret_cast<const int4*>(p)[0], v = reinterpret_cast<const int4*>(p)[1];
  return i32x8{u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
}

template <typename O, int kGroup>
__global__ __launch_bounds__(kWave) void k_block_product(BlockArgs a) {
  const int lane = threadIdx.x;
  const int64_t m0 = (int64_t)(blockIdx.x % a.mt) * 32, n0 = (int64_t)(blockIdx.x / a.mt) * 32;
  const int64_t m = min(m0 + (lane & 31), a.M - 1), n = min(n0 + (lane & 31), a.N - 1);
  const uint8_t* pa = a.a + m * a.lda + (lane >> 5) * 32;
  const uint8_t* pb = a.b + n * a.ldb + (lane >> 5) * 32;
  f32x16 acc{};
  for (int64_t j = 0; j < a.blocks; ++j) {
    // (rows of the result are rows of a)
    constexpr bool kExact = sizeof(O) == 4;
    f32x16 c = block_step<kExact>(load32(pa + j * 128), load32(pb + j * 128), f32x16{});
    c = block_step<kExact>(load32(pa + j * 128 + 64), load32(pb + j * 128 + 64), c);
    const float sb = a.sb[j * a.ldsb + n / kGroup];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t row = min(m0 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3), a.M - 1);
      acc[e] = fmaf(c[e], a.sa[j * a.ldsa + row] * sb, acc[e]);
    }
  }
  if (n0 + (lane & 31) >= a.N) return;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int64_t row = m0 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
    if (row < a.M) store1(static_cast<O*>(a.out) + row * a.ldo + n, acc[e]);
  }
}

template <typename O>
hipError_t launch_t(const BlockArgs& a, int group, hipStream_t s) {
  const dim3 grid((unsigned)(a.mt * ((a.N + 31) / 32)));
  if (group == 1)
    hipLaunchKernelGGL((k_block_product<O, 1>), grid, dim3(kWave), 0, s, a);
  else
    hipLaunchKernelGGL((k_block_product<O, 128>), grid, dim3(kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_product(BlockArgs a, int group, bool bf16, hipStream_t s) {
  a.mt = (a.M + 31) / 32;
  return bf16 ? launch_t<bf16_t>(a, group, s) : launch_t<float>(a, group, s);
}

}  // namespace vsd
