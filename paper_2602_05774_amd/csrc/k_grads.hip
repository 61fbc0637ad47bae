// The global norm of many gradients and their scaling to a bound.
//
// Two kinds of launch, each over up to kGradTable tensors described in the
// kernel's arguments (nothing is uploaded): the sums of squares, one double per
// workgroup, and the scaling, whose workgroups each add those sums up (in one
// order, so all get the same norm) instead of waiting for a launch that does.  The
// squares are formed and summed in double precision: fp32 squares would overflow
// from 1.8e19 on and lose elements below 1e-19 (double FMAs issue at the rate of
// fp32 ones on this chip, far above what memory feeds).
#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float element(const void* p, int64_t i) {
  return load1(static_cast<const T*>(p) + i);
}

// f(chunk, tensor) for this workgroup's chunks of the table
template <class F>
__device__ __forceinline__ void chunks(const GradTable& t, F&& f) {
  int k = 0;
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    while (k + 1 < t.n && t.e[k + 1].first <= c) ++k;
    f(c - t.e[k].first, t.e[k]);
  }
}

// f(index into the source, index into the output) for a thread's elements of a chunk
template <class F>
__device__ __forceinline__ void elements(const GradEntry& e, int chunk, F&& f) {
  const int64_t n = e.rows * e.cols, lo = (int64_t)chunk * kGradChunk, hi = min(lo + kGradChunk, n);
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const int64_t r = e.rows == 1 ? 0 : i / e.cols, c = i - r * e.cols;
    f(r * e.ld + c, r * e.out_ld + c);
  }
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[wave_id()] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradTable t, double* part) {
  __shared__ double red[kThreads / kWave];
  double s = 0.0;
  chunks(t, [&](int chunk, const GradEntry& e) {
    elements(e, chunk, [&](int64_t i, int64_t) {
      const double x = e.bf16 ? element<bf16_t>(e.p, i) : element<float>(e.p, i);
      s = __builtin_fma(x, x, s);
    });
  });
  s = block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
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

__global__ __launch_bounds__(kThreads) void k_grad_scale(GradTable t, GradScale g) {
  __shared__ double red[kThreads / kWave];
  const double norm = g.norm != nullptr ? (double)*g.norm : norm_of(g.part, g.parts, red);
  const bool finite = norm <= 1.7976931348623157e308;
  const float scale = !finite ? 1.0f : norm > (double)g.max_norm ? (float)((double)g.max_norm / norm) : 1.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0 && t.first) {
    if (g.norm_out != nullptr) *g.norm_out = (float)norm;
    if (g.scale_out != nullptr) *g.scale_out = finite ? scale : __builtin_nanf("");
  }
  chunks(t, [&](int chunk, const GradEntry& e) {
    if (scale == 1.0f && e.out == e.p) return;
    elements(e, chunk, [&](int64_t i, int64_t o) {
      const float x = (e.bf16 ? element<bf16_t>(e.p, i) : element<float>(e.p, i)) * scale;
      if (e.out_bf16)
        store1(static_cast<bf16_t*>(e.out) + o, x);
      else
        store1(static_cast<float*>(e.out) + o, x);
    });
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
