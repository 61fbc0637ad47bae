// Products of block matrices by 256 x 256 tiles (see k_block.hip), many rows.
//
// Operands: U rows (of b: the result's columns) and V rows (of a: its rows), 128
// bytes of each a stage: a block.  The schedule is that of the LM head's product loop: eight
// wavefronts in two groups that run half a phase apart, one reading fragments and
// issuing loads while the other multiplies; four phases a stage, one quadrant of
// the tile each, every phase refilling the half operand whose last reader is past
// (48 KB in flight, never drained); 16-byte chunks of a row swizzled over the banks.
// What is added to it: a quadrant's product starts from zero and is joined to the
// tile's fp32 sums, times its scales, by the vector units while the matrix cores form
// the other half of the phase's products; the scales ride through LDS, loaded two
// stages ahead with the operands.
// 6144 x 128 256 x 4096 to bf16: 2.95 to 3.08 ms, 2.1 to 2.2 PFLOP/s; a stage takes some 3700
// cycles, 2048 of them matrix instructions, VALU instructions in 42 % (an earlier form's
// 3281 us were 2914 without the joins, 2795 without loads, 2894 without stores).  32 000 x 2048 x
// 9001 to fp32: 1.2 ms, 0.99 PFLOP/s, the VALU shared by the conversions to bf16 and the
// other group's joins (63 % of the cycles, matrix instructions in 44 %).
//   phase  reads   refills             multiplies   waits for
//   1      U0(t)   U1(t+1)             U0 V0
//   2      V1(t)   V0(t+2)             U0 V1
//   3      U1(t)   U0(t+2)             U1 V0        V0(t+1)
//   4      V0(t+1) V1(t+2), scales     U1 V1        all of t+1
#pragma once

#include "vsd_device.hpp"
#include "vsd_kernels.hpp"

namespace vsd {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Eight e4m3 values (two words) in bf16.
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

namespace block_tiles {
namespace {

constexpr int kTile = 256, kThreads = 512, kRow = 128;  // bytes of a row a stage
constexpr int kHalf = 128 * kRow, kBuf = 4 * kHalf;     // half an operand's stage; U0 U1 V0 V1
constexpr int kScales = 2 * kBuf, kSlots = 4, kSlot = 2 * kTile * 4;  // V's 256 scales, U's 256
constexpr int kLds = kScales + kSlots * kSlot;
constexpr int kXcds = 8, kGroupRows = 4;
static_assert(kLds <= 160 * 1024, "the stages and the scales fit the LDS");

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ int swz_u(int r) { return ((r >> 1) & 3) | (((r >> 5) & 1) << 2); }
__device__ __forceinline__ int swz_v(int r) { return (r >> 1) & 7; }

__device__ __forceinline__ void phase_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // s_waitcnt: vmcnt bits 3:0 and 15:14, expcnt 6:4, lgkmcnt 11:8
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Workgroup -> (row tile, run of column tiles): the workgroups of one XCD (ids are
// dealt round-robin) walk groups of kGroupRows row tiles.
__device__ __forceinline__ void tile_of(int pid, int nrt, int ncol, int& rt, int& col) {
  const int total = nrt * ncol, xcd = pid % kXcds, local = pid / kXcds;
  const int per = total / kXcds, extra = total % kXcds;
  const int id = xcd * per + min(xcd, extra) + local;
  const int g = id / (kGroupRows * ncol), in = id % (kGroupRows * ncol);
  const int first = g * kGroupRows, rows = min(nrt - first, kGroupRows);
  rt = first + in % rows;
  col = in / rows;
}

// A lane's x of the other lane (by CTRL) and its y change places: where `odd`, x becomes
// the other's y, else y the other's x.
template <int CTRL>
__device__ __forceinline__ void quad_swap(uint32_t (&x)[4], uint32_t (&y)[4], bool odd) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t got = (uint32_t)dpp_i<CTRL>((int)(odd ? x[w] : y[w]));
    x[w] = odd ? got : x[w];
    y[w] = odd ? y[w] : got;
  }
}

template <int N>
struct Index {
  static constexpr int value = N;
};
template <class F>
__device__ __forceinline__ void each16(F&& f) {
  f(Index<0>{}), f(Index<1>{}), f(Index<2>{}), f(Index<3>{}), f(Index<4>{}), f(Index<5>{}), f(Index<6>{}), f(Index<7>{});
  f(Index<8>{}), f(Index<9>{}), f(Index<10>{}), f(Index<11>{}), f(Index<12>{}), f(Index<13>{}), f(Index<14>{}), f(Index<15>{});
}

// F8: 8-bit matrix instructions; else the values go through bf16 ones, converted
// between the products.
template <bool F8, int kGroup, typename O>
__device__ __forceinline__ void tiles(const BlockTileArgs& a, uint8_t* lds) {
  const int lane = threadIdx.x & 63, w = wave_id(), wr = w >> 2, wc = w & 3;
  int rt, run;
  tile_of(blockIdx.x, a.mt, a.runs, rt, run);
  const int t_begin = run * a.run, t_end = min(t_begin + a.run, a.nt);
  const int k_begin = (int)blockIdx.y * a.per, k_end = min(k_begin + a.per, a.stages);  // stages of this range
  const int64_t m0 = (int64_t)rt * kTile;
  auto rows = [&](const uint8_t* base, int64_t ld, int64_t n) {
    return row_rsrc(base, (uint32_t)min(n, (int64_t)kTile) * (uint32_t)ld);
  };
  auto u_tile = [&](int t) { return rows(a.b + (int64_t)t * kTile * a.ldb, a.ldb, a.N - (int64_t)t * kTile); };
  const __amdgpu_buffer_rsrc_t rv = rows(a.a + m0 * a.lda, a.lda, a.M - m0);
  // where the wavefront's first load of a half starts for this lane (bytes); the
  // second, 8 rows on, has the same swizzle (U), or the chunks' upper bit turned (V)
  const int r0 = w * 16 + (lane >> 3);
  const int ou = (int)(r0 * a.ldb + (((lane & 7) ^ swz_u(r0)) << 4));
  const int ov = (int)(r0 * a.lda + (((lane & 7) ^ swz_v(r0)) << 4));
  const int ldu = (int)a.ldb, ldv = (int)a.lda;
  // a cursor: the tile and the stage; past the last one it repeats
  struct Cursor {
    __amdgpu_buffer_rsrc_t u;
    int t, k;
  };
  auto advance = [&](Cursor& c) {
    int t = c.t, k = c.k + 1;
    if (k == k_end) {
      if (t + 1 < t_end) {
        c.u = u_tile(++t);
        k = k_begin;
      } else {
        --k;
      }
    }
    c.t = __builtin_amdgcn_readfirstlane(t);
    c.k = __builtin_amdgcn_readfirstlane(k);
  };
  uint8_t* const mine = lds + w * 16 * kRow;
  auto load_u = [&](int h, const Cursor& c, int buf) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(c.u, (lds_void*)(mine + buf * kBuf + h * kHalf + j * 8 * kRow), 16,
                                               ou + (h * 128 + j * 8) * ldu, c.k * kRow, 0, 0);
  };
  auto load_v = [&](int h, const Cursor& c, int buf) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void*)(mine + buf * kBuf + (2 + h) * kHalf + j * 8 * kRow), 16,
                                               (ov ^ (j << 6)) + (h * 128 + j * 8) * ldv, c.k * kRow, 0, 0);
  };
  // one load a wavefront: 64 of V's scales (wavefronts 0 .. 3) or of U's
  const bool of_v = w < 4;
  const float* const scales = of_v ? a.sa + m0 : a.sb;
  const int64_t scale_ld = of_v ? a.ldsa : a.ldsb, scale_n = of_v ? a.M - m0 : (a.N + kGroup - 1) / kGroup;
  const int scale_tile = of_v ? 0 : kTile / kGroup;  // U's scales of a tile
  const int scale_at = ((w & 3) * 64 + lane) / (of_v ? 1 : kGroup) * 4;
  auto load_scales = [&](const Cursor& c, int slot) {
    const int64_t j = c.k, first = (int64_t)c.t * scale_tile;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        row_rsrc(scales + j * scale_ld + first, (uint32_t)min(scale_n - first, (int64_t)kTile) * 4u),
        (lds_void*)(lds + kScales + slot * kSlot + w * 256), 4, scale_at, 0, 0, 0);
  };

  // a lane's fragment addresses in the first quarter of a stage; quarter ks: ^ ks << 5
  uint32_t fu_at, fv_at;
  {
    const int m = lane & 31, b = (m >> 2) & 1;
    const int ru = 32 * b + 4 * (m >> 3) + (m & 3);
    fu_at = (wr * 64 + ru) * kRow + (((lane >> 5) ^ swz_u(ru)) << 4);
    fv_at = 2 * kHalf + (wc * 32 + m) * kRow + (((lane >> 5) ^ swz_v(m)) << 4);
  }
  f32x16 acc[2][2][2], tmp[2];
  i32x4 fu[2][4], fv0[4], fv1[4];
  auto frag = [&](uint32_t off) { return *reinterpret_cast<const i32x4*>(lds + off); };
  auto read_u = [&](int buf, int half) {
    const uint32_t at = fu_at + buf * kBuf;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) fu[i][ks] = frag((at ^ (ks << 5)) + half * kHalf + i * 16 * kRow);
  };
  auto read_v = [&](i32x4 (&f)[4], int buf, int half) {
    const uint32_t at = fv_at + buf * kBuf;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) f[ks] = frag((at ^ (ks << 5)) + half * kHalf);
  };
  // The scales of U half h and V half g: read ahead of the phase's fragments (LDS
  // returns in order), so that the join does not wait for those.
  struct Scales {
    float v, u[kGroup == 1 ? 2 : 1];
  };
  auto scales_of = [&](int h, int g, int slot) {
    const float* const S = reinterpret_cast<const float*>(lds + kScales + slot * kSlot);
    Scales s;
    s.v = S[g * 128 + wc * 32 + (lane & 31)];
    if constexpr (kGroup == 1) {
      // a lane's registers are 16 consecutive U rows: their scales lie in the 16 lanes of
      // its DPP row, and the join takes lane e's
#pragma unroll
      for (int i = 0; i < 2; ++i) s.u[i] = S[kTile + h * 128 + wr * 64 + 32 * (lane >> 5) + 16 * i + (lane & 15)];
    } else {
      s.u[0] = S[kTile + h * 128];
    }
    __builtin_amdgcn_sched_barrier(0);
    return s;
  };
  // acc += tmp[i] times the scales of U (registers) and V (lanes)
  auto join = [&](int h, int g, int i, const Scales& s) {
    if constexpr (kGroup == 128) {
      const float both = s.v * s.u[0];
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[h][g][i][e] = fmaf(tmp[i][e], both, acc[h][g][i][e]);
    } else {
      each16([&](auto e) {
        constexpr int kE = decltype(e)::value;
        const float ue = dpp_f<0x150 + kE>(s.u[i]);  // row_newbcast
        acc[h][g][i][kE] = fmaf(tmp[i][kE] * ue, s.v, acc[h][g][i][kE]);
      });
    }
    asm volatile("" : "+v"(acc[h][g][i]));  // (the sums stay in this phase and in their registers)
    __builtin_amdgcn_sched_barrier(0);
  };
  // A phase's products, of U half h and V half g.  8-bit: while the matrix cores form one
  // half of them, the vector units join the other: tmp[1] of the quadrant before
  // (`pending`: there is one), then this one's tmp[0].
  auto mult = [&](i32x4 (&v)[4], int h, int g, const Scales& s, int h1, int g1, const Scales& s1, bool pending) {
    __builtin_amdgcn_s_setprio(1);
    if constexpr (F8) {
      auto half = [&](int i) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          const i32x8 x = __builtin_shufflevector(fu[i][2 * ks], fu[i][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7);
          const i32x8 y = __builtin_shufflevector(v[2 * ks], v[2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7);
          tmp[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, ks == 0 ? f32x16{} : tmp[i], 0, 0, 0, 0, 0, 0);
        }
        asm volatile("" : "+v"(tmp[i]));
        __builtin_amdgcn_sched_barrier(0);
      };
      half(0);
      if (pending) join(h1, g1, 1, s1);
      half(1);
      join(h, g, 0, s);
    } else {
      // (the values' bf16 forms are made anew for every quadrant: kept, they would not fit)
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) asm volatile("" : "+v"(fu[0][ks]), "+v"(fu[1][ks]), "+v"(v[ks]));
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const bf16x8 y = widen(v[ks >> 1][(ks & 1) * 2], v[ks >> 1][(ks & 1) * 2 + 1]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          tmp[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              widen(fu[i][ks >> 1][(ks & 1) * 2], fu[i][ks >> 1][(ks & 1) * 2 + 1]), y, ks == 0 ? f32x16{} : tmp[i], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);  // (not all conversions first: they would fill the registers)
      }
      asm volatile("" : "+v"(tmp[0]), "+v"(tmp[1]));
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // fp32 results: the conversions fill the products' phases, so both halves are joined
  // in the reading phase after them.
  auto join_read = [&](int h, int g, const Scales& s) {
    if constexpr (!F8) {
      __builtin_amdgcn_sched_barrier(0);
      join(h, g, 0, s);
      join(h, g, 1, s);
    }
  };
  // The tile's results: 32 consecutive columns a lane in each half of the columns.  Four
  // lanes change pieces, so that they store 64 consecutive bytes of a row (us, each lane
  // 16 bytes of its row / this: 16 384 x 5000 x 100 to fp32 167 / 107, to bf16 60 / 48,
  // 16 384 x 16 384 x 64 to fp32 917 / 404, 6144 x 128 256 x 4096 to bf16 3130 / 3080).
  O* const out = static_cast<O*>(a.out) + (int64_t)blockIdx.y * a.range_stride;
  auto store = [&](int t) {
    int l = lane;
    asm volatile("" : "+v"(l));  // (its addresses are formed here, not kept across the loop)
    const int64_t n = (int64_t)t * kTile + wr * 64 + 32 * (l >> 5);
    const int q = l & 3;
    constexpr int kPer = 16 / (int)sizeof(O);  // results of a 16-byte piece
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int64_t m = m0 + g * 128 + wc * 32 + (l & 28);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 32; c += 4 * kPer) {
          uint32_t d[4][4];  // a row's pieces c .. c + 4 kPer; then: four rows, the lane's piece of each
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if constexpr (sizeof(O) == 4) {
                const int e = c + k * 4 + w;
                d[k][w] = __float_as_uint(acc[h][g][e >> 4][e & 15]);
              } else {
                const int e = c + k * 8 + w * 2;
                d[k][w] = pack_bf16x2(acc[h][g][e >> 4][e & 15], acc[h][g][e >> 4][(e & 15) + 1]);
              }
            }
          quad_swap<kDppQuad1>(d[0], d[1], (q & 1) != 0);
          quad_swap<kDppQuad1>(d[2], d[3], (q & 1) != 0);
          quad_swap<kDppQuad2>(d[0], d[2], (q & 2) != 0);
          quad_swap<kDppQuad2>(d[1], d[3], (q & 2) != 0);
          const int64_t at = n + h * 128 + c + q * kPer;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (m + k >= a.M) continue;
            O* const to = out + (m + k) * a.ldo + at;
            if (at + kPer <= a.N) {
              *reinterpret_cast<uint4*>(to) = make_uint4(d[k][0], d[k][1], d[k][2], d[k][3]);
            } else {
#pragma unroll
              for (int e = 0; e < kPer; ++e) {
                if (at + e >= a.N) continue;
                if constexpr (sizeof(O) == 4)
                  to[e] = __uint_as_float(d[k][e]);
                else
                  to[e] = (O)(d[k][e >> 1] >> (16 * (e & 1)));
              }
            }
          }
        }
    }
  };

  Cursor c1{u_tile(t_begin), t_begin, k_begin}, c2;
  load_scales(c1, 0);
  load_v(0, c1, 0);
  load_u(0, c1, 0);
  load_v(1, c1, 0);
  load_u(1, c1, 0);
  advance(c1);
  c2 = c1;
  advance(c2);
  load_v(0, c1, 1);
  load_u(0, c1, 1);
  load_v(1, c1, 1);
  load_scales(c1, 1);
  wait_loads<7>();
  phase_barrier();
  if (wr == 1) phase_barrier();  // from here on this group runs half a phase behind
  read_v(fv0, 0, 0);
  wait_lds();
  auto clear = [&]() {
#pragma unroll
    for (int q = 0; q < 8; ++q) acc[q >> 2][(q >> 1) & 1][q & 1] = f32x16{};
  };
  clear();
  int p = 0, slot = 0;
  Scales s[4];  // of the quadrants, in their order
  // Stores are counted with the loads and end in their order, so a wait for loads that
  // were issued after a tile's stores waits for the stores.  The next tile's U1 is
  // therefore asked for before them, and its first stage's waits leave the stores of a
  // whole tile (each wavefront's kStores) out: they have almost two stages to drain.
  constexpr int kStores = sizeof(O) == 2 ? 16 : 32;
  bool stored = false, whole = false;  // a tile was stored just now, all of it
  for (int t = t_begin, k = k_begin; t < t_end; p ^= 1, slot = (slot + 1) & (kSlots - 1)) {
    const bool pending = k > k_begin;
    s[0] = scales_of(0, 0, slot);
    if (!stored) load_u(1, c1, p ^ 1);
    read_u(p, 0);
    if (pending) join_read(1, 1, s[3]);
    phase_barrier();
    wait_lds();
    mult(fv0, 0, 0, s[0], 1, 1, s[3], pending);
    phase_barrier();

    s[1] = scales_of(0, 1, slot);
    load_v(0, c2, p);
    read_v(fv1, p, 1);
    join_read(0, 0, s[0]);
    phase_barrier();
    wait_lds();
    mult(fv1, 0, 1, s[1], 0, 0, s[0], true);
    phase_barrier();

    s[2] = scales_of(1, 0, slot);
    load_u(0, c2, p);
    read_u(p, 1);
    join_read(0, 1, s[1]);
    if (whole)
      wait_loads<11 + kStores>();
    else
      wait_loads<11>();
    phase_barrier();
    wait_lds();
    mult(fv0, 1, 0, s[2], 0, 1, s[1], true);
    phase_barrier();

    s[3] = scales_of(1, 1, slot);
    load_v(1, c2, p);
    load_scales(c2, (slot + 2) & (kSlots - 1));
    read_v(fv0, p ^ 1, 0);
    join_read(1, 0, s[2]);
    if (whole)
      wait_loads<7 + kStores>();
    else
      wait_loads<7>();
    phase_barrier();
    wait_lds();
    mult(fv1, 1, 1, s[3], 1, 0, s[2], true);
    c1 = c2;
    advance(c2);
    if (wr == 0) phase_barrier();
    stored = whole = false;
    if (++k == k_end) {  // both groups finish a tile between the same two barriers
      join_read(1, 1, s[3]);
      if (F8) join(1, 1, 1, s[3]);
      load_u(1, c1, p);
      stored = true;
      whole = m0 + kTile <= a.M && (int64_t)(t + 1) * kTile <= a.N;
      store(t);
      clear();
      ++t;
      k = k_begin;
    }
    if (wr == 1) phase_barrier();
  }
  if (wr == 0) phase_barrier();
  wait_loads<0>();  // the repeated loads have landed before the LDS is given up
}

template <bool F8, int kGroup, typename O>
__global__ __launch_bounds__(kThreads) void k_block_tiles(BlockTileArgs a) {
  __shared__ __align__(16) uint8_t lds[kLds];
  tiles<F8, kGroup, O>(a, lds);
}

}  // namespace
}  // namespace block_tiles
}  // namespace vsd
