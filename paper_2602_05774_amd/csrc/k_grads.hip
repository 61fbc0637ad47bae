// The global norm of many gradients and their scaling to a bound.
//
// Two kinds of launch, each over up to kGradTable tensors described in the
// kernel's arguments (nothing is uploaded): the sums of squares, one double per
// workgroup, and the scaling, whose workgroups each add those sums up (in one
// order, so all get the same norm) instead of waiting for a launch that does.  The
// squares are formed and summed in double precision: fp32 squares would overflow
// from 1.8e19 on and lose elements below 1e-19 (double FMAs issue at the rate of
// fp32 ones on this chip, far above what memory feeds).
//
// Bytes bound both: of 500 million bf16 elements in 150 tensors the squares run at 4.8
// TB/s of reads, the scaling at 5.2 of both (us a launch of a third: 69, 129).  Not kept:
// the scaling from the last chunk back, for what the caches still hold (150), chunks of
// 16 384 elements and 4096 workgroups (no faster).
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

namespace {

constexpr int kThreads = 256;

// f(chunk, tensor) for this workgroup's chunks of the table; lane k looks at tensor k
// (a search of the arguments would wait for one load after another).
template <class F>
__device__ __forceinline__ void chunks(const GradTable& t, F&& f) {
  static_assert(kGradTable <= kWave, "a lane per tensor");
  const int lane = threadIdx.x & 63;
  const int first = lane < kGradTable ? t.first[lane] : 0x7FFFFFFF;
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const int k = __builtin_popcountll(__ballot(first <= c)) - 1;
    f(c - lane_i(first, k), t.e[k]);
  }
}

// Elements by address: their number up to the next multiple of 16 bytes.
__device__ __forceinline__ int to_aligned(const void* p, int es) {
  return (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / es;
}

// A chunk of a tensor: one(i, o) for single elements (offsets into the source and
// the output), eight(i, o) for eight from a 16-byte boundary of both.
template <class One, class Eight>
__device__ __forceinline__ void elements(const GradEntry& e, int chunk, One&& one, Eight&& eight) {
  const int64_t n = e.rows * e.cols, lo = (int64_t)chunk * kGradChunk;
  const int len = (int)min((int64_t)kGradChunk, n - lo), t = threadIdx.x;
  if (e.rows > 1) {
    for (int i = t; i < len; i += kThreads) {
      const int64_t r = (lo + i) / e.cols, c = lo + i - r * e.cols;
      one(r * e.ld + c, r * e.out_ld + c);
    }
    return;
  }
  const int es = e.bf16 ? 2 : 4, out_es = e.out_bf16 ? 2 : 4;
  const int head = min(len, to_aligned(static_cast<const char*>(e.p) + lo * es, es));
  const bool both = ((reinterpret_cast<uintptr_t>(e.out) + (lo + head) * out_es) & 15u) == 0;
  const int body = both ? (len - head) / 8 : 0, tail = head + body * 8;
  if (t < head) one(lo + t, lo + t);
  if (body == kGradChunk / 8) {  // (the usual chunk: all its loads may be in flight)
#pragma unroll
    for (int k = 0; k < kGradChunk / 8 / kThreads; ++k) eight(lo + (k * kThreads + t) * 8, lo + (k * kThreads + t) * 8);
    return;
  }
  for (int i = t; i < body; i += kThreads) eight(lo + head + i * 8, lo + head + i * 8);
  for (int i = tail + t; i < len; i += kThreads) one(lo + i, lo + i);
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[wave_id()] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <typename T>
__device__ __forceinline__ void squares(const GradEntry& e, int chunk, double (&s)[4]) {
  const T* p = static_cast<const T*>(e.p);
  elements(
      e, chunk,
      [&](int64_t i, int64_t) {
        const double x = load1(p + i);
        s[0] = __builtin_fma(x, x, s[0]);
      },
      [&](int64_t i, int64_t) {
        float x[8];
        load8(p + i, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k & 3] = __builtin_fma((double)x[k], (double)x[k], s[k & 3]);
      });
}

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradTable t, double* part) {
  __shared__ double red[kThreads / kWave];
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  chunks(t, [&](int chunk, const GradEntry& e) {
    if (e.bf16)
      squares<bf16_t>(e, chunk, s);
    else
      squares<float>(e, chunk, s);
  });
  const double all = block_sum((s[0] + s[1]) + (s[2] + s[3]), red);
  if (threadIdx.x == 0) part[blockIdx.x] = all;
}

__device__ __forceinline__ double norm_of(const double* part, int n, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) s += part[i];
  return __builtin_sqrt(block_sum(s, red));
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(const double* part, int n, float* norm) {
  __shared__ double red[kThreads / kWave];
  const double v = norm_of(part, n, red);
  if (threadIdx.x == 0) *norm = (float)v;
}

template <typename T, typename O>
__device__ __forceinline__ void scaled(const GradEntry& e, int chunk, float scale) {
  const T* p = static_cast<const T*>(e.p);
  O* const out = static_cast<O*>(e.out);
  elements(
      e, chunk, [&](int64_t i, int64_t o) { store1(out + o, load1(p + i) * scale); },
      [&](int64_t i, int64_t o) {
        float x[8];
        load8(p + i, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= scale;
        store8(out + o, x);
      });
}

__global__ __launch_bounds__(kThreads) void k_grad_scale(GradTable t, GradScale g) {
  __shared__ double red[kThreads / kWave];
  const double norm = g.norm != nullptr ? (double)*g.norm : norm_of(g.part, g.parts, red);
  const bool finite = norm <= 1.7976931348623157e308;
  const float scale = !finite ? 1.0f : norm > (double)g.max_norm ? (float)((double)g.max_norm / norm) : 1.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0 && t.reports) {
    if (g.norm_out != nullptr) *g.norm_out = (float)norm;
    if (g.scale_out != nullptr) *g.scale_out = finite ? scale : __builtin_nanf("");
  }
  chunks(t, [&](int chunk, const GradEntry& e) {
    if (scale == 1.0f && e.out == e.p) return;
    if (e.bf16 && e.out_bf16)
      scaled<bf16_t, bf16_t>(e, chunk, scale);
    else if (e.bf16)
      scaled<bf16_t, float>(e, chunk, scale);
    else if (e.out_bf16)
      scaled<float, bf16_t>(e, chunk, scale);
    else
      scaled<float, float>(e, chunk, scale);
  });
}

}  // namespace

hipError_t launch_grad_squares(const GradTable& t, double* part, hipStream_t s) {
  hipLaunchKernelGGL(k_grad_squares, dim3(t.groups), dim3(kThreads), 0, s, t, part);
  return hipGetLastError();
}
hipError_t launch_grad_norm(const double* part, int n, float* norm, hipStream_t s) {
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(kThreads), 0, s, part, n, norm);
  return hipGetLastError();
}
hipError_t launch_grad_scale(const GradTable& t, const GradScale& g, hipStream_t s) {
  hipLaunchKernelGGL(k_grad_scale, dim3(t.groups), dim3(kThreads), 0, s, t, g);
  return hipGetLastError();
}

}  // namespace vsd
