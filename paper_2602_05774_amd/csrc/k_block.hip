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
// Many rows: 256 x 256 tiles (vsd_block_tiles.hpp), the sum in ranges where there are
// few tiles.
// Few rows: a stream of b (k_block_few).  Rows too long for the tiles' offsets: a
// wavefront per 32 x 32 tile that walks the blocks.  In all of them a block's product
// is formed on the matrix cores from zero and added, times its scales, in fp32.
#include "vsd_block_tiles.hpp"

namespace vsd {

namespace {

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

// Few rows (kTiles x 32 at most): a stream of b.  A workgroup owns 32 of b's rows; its
// wavefronts take the blocks of its range in turn, the next block's loads in flight
// (64 bytes of a row a lane, whole cache lines), and their sums meet in LDS in the
// wavefronts' order.  b's rows are the products' rows (registers) and a's their
// columns (lanes), so that a's scales are one load a block and b's, of 128 rows, one
// for all: with the factors the other way round each block took 16 loads of a's
// scales and one token (32 000 x 4096) 35 us, 48 rows (32 003 x 2048, fp32) 32.
template <typename O, bool EXACT, int kGroup, int kTiles, int kWaves>
__global__ __launch_bounds__(kWaves * kWave) void k_block_few(BlockArgs a) {
  __shared__ float sums[kWaves - 1][kTiles * 16][kWave];
  const int lane = threadIdx.x & 63, wave = wave_id(), half = lane >> 5;
  const int64_t n0 = (int64_t)blockIdx.x * 32;
  const int64_t begin = (int64_t)blockIdx.y * a.per, end = min(begin + a.per, a.blocks);
  const uint8_t* const pb = a.b + min(n0 + (lane & 31), a.N - 1) * a.ldb + half * 32;
  const uint8_t* pa[kTiles];
  const float* sa[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int64_t m = min((int64_t)(t * 32 + (lane & 31)), a.M - 1);
    pa[t] = a.a + m * a.lda + half * 32;
    sa[t] = a.sa + m;
  }
  // rows 8 q + 4 half .. + 3 of the tile are registers 4 q .. 4 q + 3
  constexpr int kSb = kGroup == 1 ? 16 : 1;
  struct Step {
    i32x8 b[2], a[kTiles][2];
    float sa[kTiles], sb[kSb];
  };
  auto load = [&](int64_t j) {
    Step s;
    s.b[0] = load32(pb + j * 128);
    s.b[1] = load32(pb + j * 128 + 64);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      s.a[t][0] = load32(pa[t] + j * 128);
      s.a[t][1] = load32(pa[t] + j * 128 + 64);
      s.sa[t] = sa[t][j * a.ldsa];
    }
    const float* const sb = a.sb + j * a.ldsb;
    if constexpr (kGroup == 1) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s.sb[e] = sb[min(n0 + 8 * (e >> 2) + 4 * half + (e & 3), a.N - 1)];
    } else {
      s.sb[0] = sb[n0 / kGroup];
    }
    return s;
  };
  f32x16 acc[kTiles] = {};
  int64_t j = begin + wave;
  Step next;
  if (j < end) next = load(j);
  for (; j < end; j += kWaves) {
    const Step s = next;
    next = load(min(j + kWaves, end - 1));
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      f32x16 c = block_step<EXACT>(s.b[0], s.a[t][0], f32x16{});
      c = block_step<EXACT>(s.b[1], s.a[t][1], c);
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[t][e] = fmaf(c[e], s.sa[t] * s.sb[kGroup == 1 ? e : 0], acc[t][e]);
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sums[wave - 1][t * 16 + e][lane] = acc[t][e];
  }
  __syncthreads();
  if (wave > 0) return;
  O* const out = static_cast<O*>(a.out) + (int64_t)blockIdx.y * a.range_stride;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int64_t m = t * 32 + (lane & 31);
    if (m >= a.M) return;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = acc[t][e];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w) v += sums[w][t * 16 + e][lane];
      const int64_t n = n0 + 8 * (e >> 2) + 4 * half + (e & 3);
      if (n < a.N) store1(out + m * a.ldo + n, v);
    }
  }
}

// The sum over the ranges, in their order.
template <typename O>
__global__ __launch_bounds__(256) void k_block_join(const float* part, int ranges, int64_t M, int64_t N, int64_t ldp, O* out,
                                                    int64_t ldo) {
  const int64_t per = ldp / 8, n = M * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / per, c = (i - m * per) * 8;
    float x[8], y[8];
    load8(part + m * ldp + c, x);
    for (int r = 1; r < ranges; ++r) {
      load8(part + (r * M + m) * ldp + c, y);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] += y[k];
    }
    O* const to = out + m * ldo + c;
    if (c + 8 <= N) {
      store8(to, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < N) store1(to + k, x[k]);
    }
  }
}

// The ranges' sums (in the workspace) to the result.
template <typename O>
void launch_join(const BlockArgs& a, int ranges, int64_t ldp, const char* ws, hipStream_t s) {
  const int64_t n = (a.M * ldp / 8 + 255) / 256;
  hipLaunchKernelGGL((k_block_join<O>), dim3((unsigned)(n < 4096 ? n : 4096)), dim3(256), 0, s,
                     reinterpret_cast<const float*>(ws), ranges, a.M, a.N, ldp, static_cast<O*>(a.out), a.ldo);
}

template <typename O, bool EXACT, int kGroup>
void launch_few_t(const BlockArgs& a, const BlockPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)((a.N + 31) / 32), (unsigned)p.ranges);
  if (a.M <= 32 && p.waves == 4)
    hipLaunchKernelGGL((k_block_few<O, EXACT, kGroup, 1, 4>), grid, dim3(256), 0, s, a);
  else if (a.M <= 32)
    hipLaunchKernelGGL((k_block_few<O, EXACT, kGroup, 1, 8>), grid, dim3(512), 0, s, a);
  else if (p.waves == 4)
    hipLaunchKernelGGL((k_block_few<O, EXACT, kGroup, 2, 4>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_block_few<O, EXACT, kGroup, 2, 8>), grid, dim3(512), 0, s, a);
}

template <typename O>
hipError_t launch_few(BlockArgs a, const BlockPlan& p, int group, char* ws, hipStream_t s) {
  constexpr bool kExact = sizeof(O) == 4;
  a.per = p.per;
  if (p.ranges == 1) {
    if (group == 1)
      launch_few_t<O, kExact, 1>(a, p, s);
    else
      launch_few_t<O, kExact, 128>(a, p, s);
    return hipGetLastError();
  }
  BlockArgs r = a;
  r.out = ws;
  r.ldo = (a.N + 7) / 8 * 8;
  r.range_stride = a.M * r.ldo;
  if (group == 1)
    launch_few_t<float, kExact, 1>(r, p, s);
  else
    launch_few_t<float, kExact, 128>(r, p, s);
  launch_join<O>(a, p.ranges, r.ldo, ws, s);
  return hipGetLastError();
}

template <bool F8, typename O>
void launch_tiles(const BlockTileArgs& t, int group, int ranges, hipStream_t s) {
  const dim3 grid((unsigned)(t.mt * t.runs), (unsigned)ranges), block(block_tiles::kThreads);
  if (group == 1)
    hipLaunchKernelGGL((block_tiles::k_block_tiles<F8, 1, O>), grid, block, 0, s, t);
  else
    hipLaunchKernelGGL((block_tiles::k_block_tiles<F8, 128, O>), grid, block, 0, s, t);
}

template <typename O>
hipError_t launch_by_tiles(const BlockArgs& a, const BlockPlan& p, int group, char* ws, hipStream_t s) {
  constexpr bool kF32 = sizeof(O) == 4;
  BlockTileArgs t{};
  t.a = a.a;
  t.b = a.b;
  t.sa = a.sa;
  t.sb = a.sb;
  t.M = a.M;
  t.N = a.N;
  t.lda = a.lda;
  t.ldb = a.ldb;
  t.ldsa = a.ldsa;
  t.ldsb = a.ldsb;
  t.mt = (int32_t)((a.M + 255) / 256);
  t.nt = (int32_t)((a.N + 255) / 256);
  t.run = p.run;
  t.runs = p.runs;
  t.stages = (int32_t)a.blocks;
  t.per = p.per;
  if (p.ranges == 1) {
    t.out = a.out;
    t.ldo = a.ldo;
    launch_tiles<!kF32, O>(t, group, 1, s);
    return hipGetLastError();
  }
  t.out = ws;
  t.ldo = (a.N + 7) / 8 * 8;
  t.range_stride = a.M * t.ldo;
  launch_tiles<!kF32, float>(t, group, p.ranges, s);
  launch_join<O>(a, p.ranges, t.ldo, ws, s);
  return hipGetLastError();
}

template <typename O>
hipError_t launch_t(const BlockArgs& a, const BlockPlan& p, int group, char* ws, hipStream_t s) {
  if (p.tiles) return launch_by_tiles<O>(a, p, group, ws, s);
  if (a.M <= kBlockFewRows) return launch_few<O>(a, p, group, ws, s);
  const dim3 grid((unsigned)(a.mt * ((a.N + 31) / 32)));
  if (group == 1)
    hipLaunchKernelGGL((k_block_product<O, 1>), grid, dim3(kWave), 0, s, a);
  else
    hipLaunchKernelGGL((k_block_product<O, 128>), grid, dim3(kWave), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_product(BlockArgs a, const BlockPlan& p, int group, bool bf16, void* workspace, hipStream_t s) {
  a.mt = (a.M + 31) / 32;
  char* const ws = static_cast<char*>(workspace);
  return bf16 ? launch_t<bf16_t>(a, p, group, ws, s) : launch_t<float>(a, p, group, ws, s);
}

}  // namespace vsd
