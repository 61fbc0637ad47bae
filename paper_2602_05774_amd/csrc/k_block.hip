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

// One block of a 16 x 16 tile, lane l holding 32 bytes of row l % 16 of both operands:
// the result's column l % 16, rows 4 (l / 16) .. + 3.
template <bool EXACT>
__device__ __forceinline__ f32x4 block16(const i32x8& a, const i32x8& b) {
  f32x4 c{};
  if constexpr (EXACT) {
#pragma unroll
    for (int k = 0; k < 8; k += 2)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a[k], a[k + 1]), widen(b[k], b[k + 1]), c, 0, 0, 0);
  } else {
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
  }
  return c;
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

// Few rows (16 kTiles at most): a stream of b.  A workgroup owns 32 of b's rows, as two
// tiles of 16; its wavefronts take the blocks of its range in turn, the next block of b
// in flight, and their sums meet in LDS in the wavefronts' order.  Four lanes read 64
// consecutive bytes of a row (a value's place in the sum is free, so the lanes of a
// row take neighbouring 16-byte chunks): with the 32 x 32 instructions and 16 bytes of
// 64 rows a load the chunks of a line were fetched by four loads.  Loads return in
// order, so a's (from L2) are asked for before b's next block (from HBM): the other way
// round took a quarter longer (36 us against 29 for 48 rows of 32 003 x 2048, 25 since).
// What bounds many of these rows is not arithmetic: 48 take 27.0 us to fp32 and 25.4 to
// bf16, VALU instructions in 18 and 10 % of the cycles, matrix ones in 8 and 4 %; a
// workgroup reads all of a (from L2: 1.5 bytes for each of b's) with one block ahead.
// b's rows are the products' rows (registers) and a's their columns (lanes), so that
// a's scales are one load a block and b's, of 128 rows, one for all.
template <typename O, bool EXACT, int kGroup, int kTiles, int kWaves>
__global__ __launch_bounds__(kWaves * kWave) void k_block_few(BlockArgs a) {
  __shared__ float sums[kWaves - 1][kTiles * 8][kWave];
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 32;
  const int64_t begin = (int64_t)blockIdx.y * a.per, end = min(begin + a.per, a.blocks);
  const uint8_t* pb[2];
  const uint8_t* pa[kTiles];
  const float* sa[kTiles];
#pragma unroll
  for (int u = 0; u < 2; ++u) pb[u] = a.b + min(n0 + u * 16 + (lane & 15), a.N - 1) * a.ldb + quarter * 16;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int64_t m = min((int64_t)(t * 16 + (lane & 15)), a.M - 1);
    pa[t] = a.a + m * a.lda + quarter * 16;
    sa[t] = a.sa + m;
  }
  auto load = [&](const uint8_t* p) {
    const int4 x = *reinterpret_cast<const int4*>(p), y = *reinterpret_cast<const int4*>(p + 64);
    return i32x8{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  };
  f32x4 acc[kTiles][2] = {};
  i32x8 next[2] = {};
  int64_t j = begin + wave;
  if (j < end) {
    next[0] = load(pb[0] + j * 128);
    next[1] = load(pb[1] + j * 128);
  }
  for (; j < end; j += kWaves) {
    const i32x8 b[2] = {next[0], next[1]};
    const float* const sbj = a.sb + j * a.ldsb;
    float sb[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (kGroup == 1)
          sb[u][e] = sbj[min(n0 + u * 16 + quarter * 4 + e, a.N - 1)];
        else
          sb[u][e] = sbj[n0 / kGroup];
      }
    i32x8 x[kTiles];
    float s[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      x[t] = load(pa[t] + j * 128);
      s[t] = sa[t][j * a.ldsa];
    }
    __builtin_amdgcn_sched_barrier(0);
    const int64_t ahead = min(j + kWaves, end - 1) * 128;
    next[0] = load(pb[0] + ahead);
    next[1] = load(pb[1] + ahead);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f32x4 c = block16<EXACT>(b[u], x[t]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][u][e] = fmaf(c[e], s[t] * sb[u][e], acc[t][u][e]);
      }
  }
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[wave - 1][t * 8 + e][lane] = acc[t][e >> 2][e & 3];
  }
  __syncthreads();
  if (wave > 0) return;
  O* const out = static_cast<O*>(a.out) + (int64_t)blockIdx.y * a.range_stride;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int64_t m = t * 16 + (lane & 15);
    if (m >= a.M) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = acc[t][e >> 2][e & 3];
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w) v += sums[w][t * 8 + e][lane];
      const int64_t n = n0 + (e >> 2) * 16 + quarter * 4 + (e & 3);
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

template <typename O, bool EXACT, int kGroup, int kTiles>
void launch_few_m(const BlockArgs& a, const BlockPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)((a.N + 31) / 32), (unsigned)p.ranges);
  if (p.waves == 4)
    hipLaunchKernelGGL((k_block_few<O, EXACT, kGroup, kTiles, 4>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_block_few<O, EXACT, kGroup, kTiles, 8>), grid, dim3(512), 0, s, a);
}

template <typename O, bool EXACT, int kGroup>
void launch_few_t(const BlockArgs& a, const BlockPlan& p, hipStream_t s) {
  if (a.M <= 16)
    launch_few_m<O, EXACT, kGroup, 1>(a, p, s);
  else if (a.M <= 32)
    launch_few_m<O, EXACT, kGroup, 2>(a, p, s);
  else if (a.M <= 48)
    launch_few_m<O, EXACT, kGroup, 3>(a, p, s);
  else
    launch_few_m<O, EXACT, kGroup, 4>(a, p, s);
}

template <typename O>
hipError_t launch_few(BlockArgs a, const BlockPlan& p, int group, char* ws, hipStream_t s) {
  constexpr bool kExact = sizeof(O) == 4;
  a.per = p.per;
  if (p.ranges == 1) {
    static_assert(kBlockFewCols % 128 == 0, "a launch starts with a block of 128 of b's rows");
    for (int64_t n0 = 0; n0 < a.N; n0 += kBlockFewCols) {
      BlockArgs c = a;
      c.b += n0 * a.ldb;
      c.sb += n0 / group;
      c.out = static_cast<O*>(a.out) + n0;
      c.N = a.N - n0 < kBlockFewCols ? a.N - n0 : kBlockFewCols;
      if (group == 1)
        launch_few_t<O, kExact, 1>(c, p, s);
      else
        launch_few_t<O, kExact, 128>(c, p, s);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
  if (p.few) return launch_few<O>(a, p, group, ws, s);
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
