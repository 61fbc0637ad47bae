// Quantising to 8-bit values with a scale per block of 1 x 128 or 128 x 128, of a
// matrix or of its transpose (vsd_quantize_blocks).
//
// Every element is read once and every quotient is one IEEE division; bytes bound it.
// Blocks of 1 x 128 of the matrix itself: 16 lanes a block, no LDS (k_quantize_rows).
// Otherwise a workgroup owns a tile of 128 x 128 elements, a thread 8 x 8 of them, and
// the magnitudes' maxima, and a transpose, meet in LDS (k_quantize: the transpose of
// 32 003 x 2048 fp32 in 64 us, 5.1 TB/s).
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

namespace {

constexpr int kThreads = 256;

// Magnitudes as integers: the larger number is the larger integer, a NaN above
// infinity, so a maximum keeps it.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ __forceinline__ float scale_of(uint32_t amax) {
  return amax >= 0x7F800000u ? __builtin_nanf("") : fmaxf(__uint_as_float(amax) / 448.0f, 1.17549435e-38f);
}
// What a block's elements are divided by: its scale, or 1 where that is NaN (its
// values then mean nothing, but padding stays zero).
__device__ __forceinline__ float divisor(float scale) { return scale == scale ? scale : 1.0f; }

// Two values, rounded to the nearest, ties to even (v_cvt_pk_fp8_f32): |x / s| <=
// 448 up to a rounding that the conversion takes back.
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return (uint32_t)v;
}

// Eight values from an address of any alignment: the compiler's own wide loads, which
// take one (rows of odd lengths by single elements: 6144 x 4099 bf16 42 us, so 23).
template <typename T>
__device__ __forceinline__ void load8_any(const T* p, float (&v)[8]) {
  T q[8] __attribute__((aligned(16)));
  __builtin_memcpy(q, p, sizeof(q));
  load8(q, v);
}

// 16 rows x 4 blocks a workgroup (a block's 16 scales are one line), a lane 8 columns.
// (us, by tiles of 128 x 128 / this: 1 x 4096 bf16 8.1 / 5.2, 6144 x 4096 23.3 / 21.4, 2000
// x 33 000 54 / 45, 20 000 x 4096 fp32 79 / 70.)
constexpr int kRowBlocks = 4;
template <typename T>
__device__ __forceinline__ void row_blocks(const QuantArgs& a, int64_t r, int b0) {
  const int tc = threadIdx.x & 15;
  const T* X = static_cast<const T*>(a.x) + r * a.ld;
  float x[kRowBlocks][8];
#pragma unroll
  for (int b = 0; b < kRowBlocks; ++b) {
    const int64_t c = (int64_t)(b0 + b) * 128 + tc * 8;
    if (r < a.rows && c + 8 <= a.cols) {
      load8_any(X + c, x[b]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[b][k] = r < a.rows && c + k < a.cols ? load1(X + c + k) : 0.0f;
    }
  }
#pragma unroll
  for (int b = 0; b < kRowBlocks; ++b) {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, magnitude(x[b][k]));
    top = max(top, (uint32_t)dpp_i<kDppQuad1>((int)top));
    top = max(top, (uint32_t)dpp_i<kDppQuad2>((int)top));
    top = max(top, (uint32_t)dpp_i<kDppHalfMirror>((int)top));
    top = max(top, (uint32_t)dpp_i<kDppMirror>((int)top));
    if (r >= a.rows || b0 + b >= a.col_tiles) continue;
    const float scale = scale_of(top), s = divisor(scale);
    if (tc == 0) a.scales[(b0 + b) * a.scale_ld + r] = scale;
    float q[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = x[b][k] / s;
    *reinterpret_cast<uint2*>(a.values + r * a.out_ld + (int64_t)(b0 + b) * 128 + tc * 8) =
        make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
  }
}
template <typename T>
__global__ __launch_bounds__(kThreads) void k_quantize_rows(QuantArgs a) {
  const int groups = (a.col_tiles + kRowBlocks - 1) / kRowBlocks;
  const int64_t n = (a.rows + 15) / 16 * groups;
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int64_t q = i / groups;
    row_blocks<T>(a, q * 16 + (threadIdx.x >> 4), (int)(i - q * groups) * kRowBlocks);
  }
}

// TRANS: the result's rows are x's columns.
template <typename T, int kGroup, bool TRANS>
__global__ __launch_bounds__(kThreads) void k_quantize(QuantArgs a) {
  static_assert(kGroup == 128 || TRANS, "rows' blocks are k_quantize_rows's");
  __shared__ uint32_t part[16][128];
  __shared__ __align__(16) uint32_t out[TRANS ? 128 * 33 : 1];
  const int t = threadIdx.x, tr = t >> 4, tc = t & 15;
  const int64_t row0 = (int64_t)(blockIdx.x / a.col_tiles) * 128, col0 = (int64_t)(blockIdx.x % a.col_tiles) * 128;
  const T* X = static_cast<const T*>(a.x);
  float x[8][8];  // rows row0 + tr * 8 + i, columns col0 + tc * 8 + k
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = row0 + tr * 8 + i, c = col0 + tc * 8;
    if (r < a.rows && c + 8 <= a.cols) {
      load8_any(X + r * a.ld + c, x[i]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[i][k] = r < a.rows && c + k < a.cols ? load1(X + r * a.ld + c + k) : 0.0f;
    }
  }
  uint32_t amax[8];  // of a row (TRANS: of a column) of the thread's
#pragma unroll
  for (int i = 0; i < 8; ++i) amax[i] = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = TRANS ? k : i;
      amax[at] = max(amax[at], magnitude(x[i][k]));
    }
  const int mine = TRANS ? tc : tr, other = TRANS ? tr : tc;
#pragma unroll
  for (int i = 0; i < 8; ++i) part[other][mine * 8 + i] = amax[i];
  __syncthreads();
  if (t < 128) {
    uint32_t top = part[0][t];
    for (int k = 1; k < 16; ++k) top = max(top, part[k][t]);
    part[0][t] = top;
  }
  __syncthreads();
  if (kGroup == 128) {
    if (t < kWave) {
      uint32_t top = max(part[0][t], part[0][t + 64]);
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      part[0][t] = part[0][t + 64] = top;
    }
    __syncthreads();
  }
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = divisor(scale_of(part[0][mine * 8 + i]));
  // the tile of the result: rows out_row0 .., block b of the columns
  const int64_t out_row0 = TRANS ? col0 : row0, b = (TRANS ? row0 : col0) / 128;
  const int64_t out_rows = TRANS ? a.cols : a.rows;
  if (t < 128 && (kGroup == 1 ? out_row0 + t < out_rows : t == 0))
    a.scales[b * a.scale_ld + out_row0 / kGroup + t] = scale_of(part[0][t]);
  if (!TRANS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = row0 + tr * 8 + i;
      float q[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) q[k] = x[i][k] / s[i];
      if (r < a.rows)
        *reinterpret_cast<uint2*>(a.values + r * a.out_ld + col0 + tc * 8) =
            make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = x[i][k] / s[k];
    uint32_t* const to = out + (tc * 8 + k) * 33 + tr * 2;
    to[0] = pack4(q[0], q[1], q[2], q[3]);
    to[1] = pack4(q[4], q[5], q[6], q[7]);
  }
  __syncthreads();
#pragma unroll
  for (int i = t; i < 128 * 8; i += kThreads) {
    const int c = i >> 3, w = (i & 7) * 4;
    const uint32_t* const from = out + c * 33 + w;
    if (col0 + c < a.cols)
      *reinterpret_cast<uint4*>(a.values + (col0 + c) * a.out_ld + row0 + w * 4) = make_uint4(from[0], from[1], from[2], from[3]);
  }
}

template <typename T>
hipError_t launch_t(const QuantArgs& a, int group, bool trans, hipStream_t s) {
  const dim3 grid((unsigned)a.tiles), block(kThreads);
  if (group == 1 && !trans) {
    const int64_t n = (a.rows + 15) / 16 * ((a.col_tiles + kRowBlocks - 1) / kRowBlocks);
    hipLaunchKernelGGL((k_quantize_rows<T>), dim3((unsigned)(n < 1 << 22 ? n : 1 << 22)), block, 0, s, a);
  }
  if (group == 1 && trans) hipLaunchKernelGGL((k_quantize<T, 1, true>), grid, block, 0, s, a);
  if (group != 1 && !trans) hipLaunchKernelGGL((k_quantize<T, 128, false>), grid, block, 0, s, a);
  if (group != 1 && trans) hipLaunchKernelGGL((k_quantize<T, 128, true>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantArgs& a, bool bf16, int group, bool trans, hipStream_t s) {
  return bf16 ? launch_t<bf16_t>(a, group, trans, s) : launch_t<float>(a, group, trans, s);
}

}  // namespace vsd
