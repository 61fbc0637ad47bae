// The base losses through an LM head: logits x = h W^T formed tile by tile by
// k_lmhead.hip's product loop (which includes this file after it) and consumed
// in the accumulators.  Neither they (but for few rows, and up to 8192 of a small
// vocabulary: lm_few_keeps) nor their gradient are kept: g is formed a piece of the
// vocabulary at a time, in bf16 (the operand type of the two products that read it:
// against 64 bits bf16 gradients are off by 0.0022 of their size, 0.0017 with g in
// fp32), and both add up in fp32.
//
//   rows     the rows that take part are listed and their hidden states copied
//            to consecutive rows, followed by zero rows up to a multiple of 64:
//            rows out of play then cost nothing and whatever they hold (padding)
//            reaches no sum, and the weight's gradient has whole stages of rows
//   forward  the rows' log-sum-exps over runs of vocabulary tiles; a combine
//            joins the runs and forms the loss
//   pieces   g of a piece, then dh += g W and dW = g^T h
//
// Bound by the matrix cores: 6144 rows (4608 in play) of 128 256 x 4096 take 4.0 ms
// forward, 4.2 for g, whose logits are formed again, and 8.2 for dh and dW: 1.14 to
// 1.2 PFLOP/s with the matrix cores busy 70 to 72 % of the time (a large library
// product: 1.46).  Everything else is 60 us of it.

// The distillation's members, one wavefront per row (a lane each); the latency of
// two reads (9001 rows of 16 in 6 us).
__global__ __launch_bounds__(256) void k_lm_loss_members(LmLossArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + wave_id();
  if (r >= a.l.R) return;
  const int id = member_id(a.l, r, lane);
  const Member e = member_of(a.l, id, load_value(a.l, r, lane, id));
  const float mass = wave_sum(e.p), plogp = wave_sum(e.plogp);
  if (lane < a.l.K) {
    a.mid[r * a.l.K + lane] = e.id;
    a.mp[r * a.l.K + lane] = e.p;
  }
  if (lane == 0) {
    a.mstat[r] = make_float2(mass, plogp);
    a.tag[r] = mass != 0.0f ? 0 : -1;
  }
}

// How the products of n rows in play are divided among the CUs, a workgroup on
// each at a time.  A lane tries one division; the cheapest (in 64-deep product
// stages, every workgroup costing a few more) wins.  One wavefront.
constexpr float kRunCost = 6.0f;  // stages' time of a workgroup's first loads and of its end
// Tiles per run, so that nrt row tiles x runs fill whole rounds.
__device__ int plan_runs(int nrt, int tiles, int stages, int lane) {
  const int most = min(tiles, max(1, kLmLossRuns / nrt));
  float best = -INFINITY;
  int at = 0x7FFFFFFF;
  for (int runs = lane + 1; runs <= most; runs += kWave) {
    const int rounds = (nrt * runs + kLmCus - 1) / kLmCus, run = (tiles + runs - 1) / runs;
    argmax_merge(best, at, -(float)rounds * ((float)run * stages + kRunCost), run);
  }
  wave_argmax(best, at);
  return at;
}
// Ranges of the depth (`stages`) of a product of so many tiles.  Next to another
// product's `beside` stages no range may take longer than all of them over all
// CUs; alone, whole rounds.
__device__ int plan_splits(int64_t tiles, int stages, float beside, int limit, int lane) {
  const int most = (int)min((int64_t)min(stages, kLmLossSplits), max((int64_t)1, limit / tiles));
  float best = -INFINITY;
  int at = 0x7FFFFFFF;
  const int splits = lane + 1;
  if (splits <= most) {
    const float each = (float)((stages + splits - 1) / splits) + kRunCost;
    const float cost = beside > 0.0f ? fmaxf(each, ((float)tiles * splits * each + beside) / kLmCus)
                                     : (float)((tiles * splits + kLmCus - 1) / kLmCus) * each;
    best = -cost;
    at = splits;
  }
  wave_argmax(best, at);
  return at;
}

// The plan of n rows in play, by one wavefront.
__device__ void make_plan(const LmLossArgs& a, int n, int lane) {
  LmLossPlan p{n, 0, 0, 0, 0, 1, 0, 1};
  if (n > 0) {
    const int nrt = (n + TM - 1) / TM, tiles = (a.l.V + TN - 1) / TN, stages = a.H / TK;
    p.fwd_run = plan_runs(nrt, tiles, stages, lane);
    p.fwd_runs = (tiles + p.fwd_run - 1) / p.fwd_run;
    if (a.dh != nullptr) {
      const int ct = (a.cols + TN - 1) / TN, ht = (a.H + TN - 1) / TN, deep = (a.cols + TK - 1) / TK;
      p.g_run = plan_runs(nrt, ct, stages, lane);
      const int wdeep = (n + TK - 1) / TK;  // (whole stages: the rows are padded)
      const float dh = (float)nrt * ht * ((float)deep + kRunCost);
      const float dw = a.dw != nullptr ? (float)ct * ht * ((float)wdeep + kRunCost) : 0.0f;
      const int splits = plan_splits((int64_t)nrt * ht, deep, dw, kLmLossDh, lane);
      p.per = (deep + splits - 1) / splits * TK;
      p.splits = (a.cols + p.per - 1) / p.per;  // (every range of the first piece has columns)
      if (a.wacc != nullptr) {
        const int wsplits = plan_splits((int64_t)ct * ht, wdeep, dh, kLmLossDw, lane);
        p.dw_per = (wdeep + wsplits - 1) / wsplits * TK;
        p.dw_splits = (wdeep * TK + p.dw_per - 1) / p.dw_per;
      }
    }
  }
  if (lane == 0) *a.plan = p;
}
__device__ __forceinline__ bool in_play(const LmLossArgs& a, int64_t r) {
  const int32_t t = a.tag[r];
  if ((uint32_t)t >= (uint32_t)a.l.V) {
    if (t != -1) report_error(a.l.err, VSD_DEVERR_TOKEN_RANGE);
    return false;
  }
  return row_weight(a.l, r) != 0.0f;
}
__device__ __forceinline__ void out_of_play(const LmLossArgs& a, int64_t r) {
  a.l.loss[r] = 0.0f;
  if (a.l.lse != nullptr) a.l.lse[r] = 0.0f;
}

// at[r] = row r's place among the rows in play, or -1; the rows in play and their
// plan.  Every workgroup counts the rows before its own 1024.
constexpr int kListRows = 1024;
__global__ __launch_bounds__(kListRows) void k_lm_loss_list(LmLossArgs a) {
  __shared__ int red[kListRows / kWave];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t first = (int64_t)blockIdx.x * kListRows, r = first + threadIdx.x;
  int before = 0;
  for (int64_t k = threadIdx.x; k < first; k += kListRows) before += in_play(a, k) ? 1 : 0;
  before = wave_sum_int(before);
  if (lane == 0) red[wave] = before;
  __syncthreads();
  int place = 0;
  for (int k = 0; k < kListRows / kWave; ++k) place += red[k];
  __syncthreads();
  const bool in = r < a.l.R && in_play(a, r);
  const uint64_t has = __ballot(in);
  if (lane == 0) red[wave] = __builtin_popcountll(has);
  __syncthreads();
  int total = place;
  for (int k = 0; k < kListRows / kWave; ++k) {
    if (k < wave) place += red[k];
    total += red[k];
  }
  place += (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0u));
  if (r < a.l.R) {
    a.at[r] = in ? place : -1;
    if (in)
      a.rows[place] = (int32_t)r;
    else
      out_of_play(a, r);
  }
  if (wave == 0 && blockIdx.x == gridDim.x - 1) make_plan(a, total, lane);
}

// The hidden states of the rows in play, consecutively; zero rows behind them; a
// zero gradient for the other rows.  One wavefront per row (6144 rows of 4096 in 18
// us, after 12 for the list; 48 with their list in 10).  LIST (at most 1024
// rows): every workgroup finds the rows in play itself, and the first one writes
// what the list would.
template <bool LIST>
__global__ __launch_bounds__(256) void k_lm_loss_pack(LmLossArgs a) {
  __shared__ uint64_t in[LIST ? kListRows / kWave : 1];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t r = (int64_t)blockIdx.x * 4 + wave;
  auto place_of = [&](int k, int& n) {  // row k's place or -1, the rows in play
    int place = 0;
    n = 0;
    for (int w = 0; w < kListRows / kWave; ++w) {
      const int c = __builtin_popcountll(in[w]);
      place += w < k / kWave ? c : 0;
      n += c;
    }
    if (k >= kListRows) return -1;
    const uint64_t mine = in[k / kWave], bit = 1ull << (k % kWave);
    return (mine & bit) != 0 ? place + __builtin_popcountll(mine & (bit - 1)) : -1;
  };
  if (LIST) {
    for (int k = threadIdx.x; k < kListRows; k += 256) {
      const uint64_t has = __ballot(k < a.l.R && in_play(a, k));
      if (lane == 0) in[k / kWave] = has;
    }
    __syncthreads();
    if (blockIdx.x == 0) {
      int n;
      for (int k = threadIdx.x; k < (int)a.l.R; k += 256) {
        const int place = place_of(k, n);
        if (place >= 0)
          a.rows[place] = k;
        else
          out_of_play(a, k);
      }
      place_of(0, n);
      if (wave == 0) make_plan(a, n, lane);
    }
  }
  int n = 0;
  const uint4* from = nullptr;
  uint4* to;
  if (r < a.l.R) {
    const int32_t place = LIST ? place_of((int)r, n) : a.at[r];
    if (place >= 0) {
      from = reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.h) + r * a.H);
      to = reinterpret_cast<uint4*>(a.hp + (int64_t)place * a.H);
    } else {
      if (a.dh == nullptr) return;
      to = reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.dh) + r * a.H);
    }
  } else {
    if (LIST)
      place_of(0, n);
    else
      n = a.plan->n;
    const int64_t place = n + (r - a.l.R);
    if (place >= lm_loss_pad(n)) return;
    to = reinterpret_cast<uint4*>(a.hp + place * a.H);
  }
  for (int k = lane; k < a.H / 8; k += kWave) to[k] = from != nullptr ? from[k] : make_uint4(0, 0, 0, 0);
}

// A run of vocabulary tiles against 256 rows: their log-sum-exps over the
// columns of each wavefront group.
__global__ __launch_bounds__(kThreads, 1) void k_lm_loss_fwd(LmLossArgs a) {
  __shared__ __align__(16) bf16_t lds[2 * kBufElems];
  const int64_t n = a.plan->n;
  const int nrt = (int)((n + TM - 1) / TM), runs = a.plan->fwd_runs, length = a.plan->fwd_run;
  if ((int64_t)blockIdx.x >= (int64_t)nrt * runs) return;
  int rt, run;
  tile_of(blockIdx.x, nrt, runs, rt, run);
  const int64_t row0 = (int64_t)rt * TM, i = row0 + nt_lane_row();
  const int tiles = (a.l.V + TN - 1) / TN, begin = run * length;
  float m = kNegBig, s = 0.0f;
  NtRows src{static_cast<const bf16_t*>(a.w), a.hp, a.l.V, row0, n, a.H, begin, min(tiles, begin + length)};
  nt_stream(lds, src, [&](int tile, NtAcc& acc) {
    nt_row_per_lane(acc);
    if (i >= n) return;
#pragma unroll 1
    for (int ch = 0; ch < 16; ++ch) {
      const int c = tile * TN + nt_chunk_col(ch);
      if (c >= a.l.V) break;
      float x[8];
      nt_chunk(acc, ch, x);
      if (c + 8 > a.l.V) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k >= a.l.V) x[k] = -INFINITY;
      }
      lse_add8(x, m, s, a.l.c);
    }
  });
  if (i < n) a.part[((int64_t)run * 2 + (wave_id() >> 2)) * n + i] = make_float2(m, s);
}

// Few rows: the products x = h W^T of 64 columns with 32 kG rows.
// Four wavefronts, each with 32 of the columns and half of a stage's depth (64).
// Bound by the stream of W: stages of W (8 KB) and of the rows (4 KB kG, from L2)
// are loaded straight into a ring in LDS, as nt_stream does (eight consecutive
// lanes a row's 128 bytes; operands loaded from memory in the matrix cores'
// layout, one row per lane, took the address unit a cycle per lane: 48 rows of
// 32 000 x 4096 in 86 us).  One barrier per stage: before it a wavefront
// has waited for its loads of the stage and finished reading the one before, whose
// place the next loads take.  Past the end the last stage is loaded again.
// take(g, c, x) consumes a lane's 16 logits of row 32 g + lane % 32: x[e] is
// column c + 8 (e / 4) + e % 4 (the first two wavefronts).
template <int kG>
struct Few {
  static constexpr int kRing = kG == 1 ? 6 : kG == 2 ? 4 : 3;
  static constexpr int kStage = (kLmFewCols + 32 * kG) * TK;  // elements
  static constexpr int kLds = kRing * kStage;
  static_assert(kLds * 2 >= 2 * kG * 16 * kWave * 4, "the halves' sums fit the ring");
  static_assert(kLds * 2 * 2 <= 160 * 1024, "two workgroups fit the LDS");
};
constexpr int kFewThreads = 256;
template <int kG, class Take>
__device__ __forceinline__ void lm_few_products(const bf16_t* h, int n, const bf16_t* W, int V, int H, bf16_t* lds,
                                                Take&& take) {
  constexpr int kRing = Few<kG>::kRing, kStage = Few<kG>::kStage, kLoads = 2 + kG;  // per wavefront and stage
  const int lane = threadIdx.x & 63, wave = wave_id(), half = wave >> 1;
  const int first = blockIdx.x * kLmFewCols, c0 = first + (wave & 1) * 32;
  const int cols = __builtin_amdgcn_readfirstlane(max(0, min(V - first, kLmFewCols)));  // (scalar, as a descriptor)
  const auto wr = row_rsrc(W + (int64_t)first * H, (uint32_t)cols * (uint32_t)H * 2u);
  const auto hr = row_rsrc(h, (uint32_t)n * (uint32_t)H * 2u);
  int wo[2], ho[kG];  // the lane's byte offset: eight rows per load
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = (wave * 2 + j) * 8 + (lane >> 3);
    wo[j] = (r * H + (((lane & 7) ^ swz_v(r)) << 3)) * 2;
  }
#pragma unroll
  for (int j = 0; j < kG; ++j) {
    const int r = (wave * kG + j) * 8 + (lane >> 3);
    ho[j] = (r * H + (((lane & 7) ^ swz_v(r)) << 3)) * 2;
  }
  const int stages = H / TK;
  auto load = [&](int stage, int slot) {
    const int k = __builtin_amdgcn_readfirstlane(min(stage, stages - 1) * TK * 2);
    bf16_t* const to = lds + slot * kStage;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)(to + (wave * 2 + j) * 8 * TK), 16, wo[j], k, 0, 0);
#pragma unroll
    for (int j = 0; j < kG; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(hr, (lds_void*)(to + (kLmFewCols + (wave * kG + j) * 8) * TK), 16, ho[j],
                                               k, 0, 0);
  };
  f32x16 acc[kG];
#pragma unroll
  for (int g = 0; g < kG; ++g) acc[g] = f32x16{};
  const int row = lane & 31;
  auto frag = [&](int slot, int r, int j) {  // 16 K values from step j of this wavefront's half
    const int c = half * 4 + j * 2 + (lane >> 5);
    return *reinterpret_cast<const bf16x8*>(lds + slot * kStage + r * TK + ((c ^ swz_v(r)) << 3));
  };
#pragma unroll
  for (int u = 0; u < kRing - 1; ++u) load(u, u);
  int slot = 0;
  for (int t = 0; t < stages; ++t) {
    wait_loads<(kRing - 2) * kLoads>();
    phase_barrier();
    load(t + kRing - 1, slot == 0 ? kRing - 1 : slot - 1);
    bf16x8 fw[2], fh[kG][2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      fw[j] = frag(slot, (wave & 1) * 32 + row, j);
#pragma unroll
      for (int g = 0; g < kG; ++g) fh[g][j] = frag(slot, kLmFewCols + g * 32 + row, j);
    }
    wait_lds();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int g = 0; g < kG; ++g) acc[g] = mfma(fw[j], fh[g][j], acc[g]);
    slot = slot + 1 == kRing ? 0 : slot + 1;
  }
  wait_loads<0>();  // the repeated loads have landed ...
  __syncthreads();  // ... in every wavefront: the ring is free
  // the two halves of the depth
  float* mine = reinterpret_cast<float*>(lds) + (wave & 1) * kG * 16 * kWave + lane;
  if (half == 1) {
#pragma unroll
    for (int g = 0; g < kG; ++g)
#pragma unroll
      for (int e = 0; e < 16; ++e) mine[(g * 16 + e) * kWave] = acc[g][e];
  }
  __syncthreads();
  if (half == 1) return;
#pragma unroll
  for (int g = 0; g < kG; ++g) {
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = acc[g][e] + mine[(g * 16 + e) * kWave];
    take(g, c0 + 4 * (lane >> 5), x);
  }
}

// (blockIdx.y: 32 kG rows; more than one of them only with kG = 4)
// With a gradient the logits are kept (lm_few_keeps), as its g needs them: W is the
// most that few rows read, and products again for g cost more than 8 bytes per logit
// (loss and dh of 16 rows of 128 256 x 4096: 631 us, so 435; 48 of 32 000 x 4096: 163
// and 127; with dW, 132 of 512 x 3456: 118 and 94).
template <int kG>
__global__ __launch_bounds__(kFewThreads, 2) void k_lm_loss_few(LmLossArgs a) {
  __shared__ __align__(16) bf16_t lds[Few<kG>::kLds];
  const int lane = threadIdx.x & 63, n = a.plan != nullptr ? a.plan->n : (int)a.l.R, row0 = blockIdx.y * 32 * kG;
  if (row0 >= n) return;
  const bf16_t* h = a.plan != nullptr ? a.hp : static_cast<const bf16_t*>(a.h);
  lm_few_products<kG>(h + (int64_t)row0 * a.H, min(n - row0, 32 * kG), static_cast<const bf16_t*>(a.w), a.l.V, a.H, lds,
                      [&](int g, int c, float (&x)[16]) {
                        const int i = row0 + g * 32 + (lane & 31);
                        if (a.x != nullptr && i < n) {
                          float* X = a.x + (int64_t)i * lm_few_ldx(a.l.V) + c;
#pragma unroll
                          for (int q = 0; q < 4; ++q)
                            *reinterpret_cast<float4*>(X + 8 * q) =
                                make_float4(x[q * 4], x[q * 4 + 1], x[q * 4 + 2], x[q * 4 + 3]);
                        }
                        float m = kNegBig, s = 0.0f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                          if (c + 8 * (e / 4) + e % 4 >= a.l.V) x[e] = -INFINITY;
                          m = fmaxf(m, x[e]);
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) s += lse_term(x[e], m, a.l.c);
                        lse_join(m, s, __shfl_xor(m, 32), __shfl_xor(s, 32), a.l.c);
                        if (lane < 32 && i < n)
                          a.part[(int64_t)i * 2 * lm_few_groups(a.l.V) + blockIdx.x * 2 + wave_id()] = make_float2(m, s);
                      });
}

// A row's loss and what its gradient needs, g_v = kq exp2((x_v - m) c) - k p_v, by
// all lanes of a wavefront from (m, s) and the logit of a lane's member (cross
// entropy: every lane the label's).
template <bool DISTILL>
__device__ __forceinline__ void lm_loss_finish(const LmLossArgs& a, int64_t i, int64_t r, float m, float s, float x) {
  const int lane = threadIdx.x & 63;
  const bool live = s != 0.0f;
  const float tail = logf(s);
  // a member's dot product, rounded in another order than the sums behind m, is not above
  // the row's largest logit (a NaN stays one)
  x = x > m ? m : x;
  float mass = 1.0f, loss;
  if (DISTILL) {
    const int K = a.l.K;
    const float p = lane < K ? a.mp[r * K + lane] : 0.0f;
    if (lane < K) a.mx[i * K + lane] = x;
    const float2 ms = a.mstat[r];
    mass = ms.x;
    loss = ms.y - wave_sum(p != 0.0f ? p * ((x - m) * a.l.inv_t - tail) : 0.0f);
  } else {
    loss = tail - (x - m) * a.l.inv_t;
  }
  if (lane == 0) {
    // (with the total in this launch, another XCD's workgroup reads it)
    __hip_atomic_store(a.l.loss + r, live ? loss : 0.0f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (a.l.lse != nullptr) a.l.lse[r] = live ? m * a.l.inv_t + tail : -INFINITY;
    const float k = live ? a.l.scale * row_weight(a.l, r) * a.l.inv_t : 0.0f;
    a.stat[i] = make_float4(m, live ? k * mass / s : 0.0f, k, 0.0f);
  }
}

// The logits of U members by a wavefront (v < 0: none, -inf), all on their way at
// once; each is wave_dot's sum.
template <int U>
__device__ __forceinline__ void wave_dots(const bf16_t* h, const bf16_t* W, const int (&v)[U], int H, int lane,
                                          float (&x)[U]) {
  float acc[U] = {};
  const bf16_t* w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = W + (int64_t)max(v[u], 0) * H;
#pragma unroll 2
  for (int k = lane * 8; k < H; k += kWave * 8) {
    float hv[8], wv[U][8];
    load8(h + k, hv);
#pragma unroll
    for (int u = 0; u < U; ++u) load8(w[u] + k, wv[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[u] = fmaf(hv[j], wv[u][j], acc[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = v[u] >= 0 ? wave_sum(acc[u]) : -INFINITY;
}

// The runs joined and the members' logits (dot products).  One wavefront per row.
// Bound by the members' rows of W, from the caches: 6300 rows of 16 members x 2048 in
// 76 us, 5.4 TB/s (one member after another: 114).  One label each, 4608
// rows of 4096: 16 us.
template <bool DISTILL>
__global__ __launch_bounds__(256) void k_lm_loss_combine(LmLossArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + wave_id(), n = a.plan->n;
  if (i >= n) return;
  const int64_t r = a.rows[i];
  float m = kNegBig, s = 0.0f;
  for (int e = lane; e < 2 * a.plan->fwd_runs; e += kWave) {
    const float2 p = a.part[(int64_t)e * n + i];
    lse_join(m, s, p.x, p.y, a.l.c);
  }
  wave_lse(m, s, a.l.c);
  const bf16_t* h = a.hp + i * a.H;
  const bf16_t* W = static_cast<const bf16_t*>(a.w);
  float x = -INFINITY;
  if (DISTILL) {
    const int K = a.l.K, id = lane < K ? a.mid[r * K + lane] : -1;
    constexpr int U = 4;
    for (int k = 0; k < K; k += U) {
      int v[U];
      float xk[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = lane_i(id, min(k + u, K - 1));
      wave_dots<U>(h, W, v, a.H, lane, xk);
#pragma unroll
      for (int u = 0; u < U; ++u) x = lane == k + u ? xk[u] : x;
    }
  } else {
    x = wave_dot(h, W + (int64_t)a.l.idx[r] * a.H, a.H, lane);
  }
  lm_loss_finish<DISTILL>(a, i, r, m, s, x);
}

// The same by a workgroup per row (lm_by_workgroup): few rows have two partial sums
// for every 64 columns one after another, and the distillation's dot products want many wavefronts (500
// rows of 32 000 x 2048 with 64 members: 174 -> 99.6 us).
// Without a plan every row is here, in play or not.
template <bool DISTILL, int kThreads>
__global__ __launch_bounds__(kThreads) void k_lm_loss_row_combine(LmLossArgs a) {
  constexpr int kWaves = kThreads / kWave;
  __shared__ float red_m[kWaves], red_s[kWaves], xs[DISTILL ? kMaxMembers : 1];
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int64_t i = blockIdx.x;
  bool in = i < (a.plan != nullptr ? a.plan->n : (int)a.l.R);
  const int64_t r = a.plan != nullptr && in ? a.rows[i] : i;
  if (a.plan == nullptr) {
    const int32_t t = a.tag[r];
    in = (uint32_t)t < (uint32_t)a.l.V && row_weight(a.l, r) != 0.0f;
    if (!in && threadIdx.x == 0) {
      if (t != -1 && (uint32_t)t >= (uint32_t)a.l.V) report_error(a.l.err, VSD_DEVERR_TOKEN_RANGE);
      __hip_atomic_store(a.l.loss + r, 0.0f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (a.l.lse != nullptr) a.l.lse[r] = 0.0f;
    }
  }
  if (in) {
    const bool few = lm_few_forward(a.l.R, a.l.V, a.dh != nullptr);
    const int parts = 2 * (few ? lm_few_groups(a.l.V) : a.plan->fwd_runs);
    const float2* part = a.part + i * (few ? parts : 1);
    const int64_t next = few ? 1 : a.plan->n;  // from one partial sum to the next
    const bf16_t* h = a.plan != nullptr ? a.hp + i * a.H : static_cast<const bf16_t*>(a.h) + r * a.H;
    const bf16_t* W = static_cast<const bf16_t*>(a.w);
    // the cross entropy's first wavefront has the label's logit meanwhile
    constexpr int kFirst = DISTILL ? 0 : 1, kSumming = kThreads - kFirst * kWave;
    float m = kNegBig, s = 0.0f;
    if (wave >= kFirst) {
      constexpr int U = 8;  // in flight per thread
      for (int e0 = threadIdx.x - kFirst * kWave; e0 < parts; e0 += U * kSumming) {
        float2 p[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          p[u] = e0 + u * kSumming < parts ? part[(e0 + u * kSumming) * next] : make_float2(kNegBig, 0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u) lse_join(m, s, p[u].x, p[u].y, a.l.c);
      }
      wave_lse(m, s, a.l.c);
    }
    if (lane == 0) {
      red_m[wave] = m;
      red_s[wave] = s;
    }
    if (DISTILL) {
      for (int k = wave; k < a.l.K; k += kWaves) {
        const int v = __builtin_amdgcn_readfirstlane(a.mid[r * a.l.K + k]);
        const float x = v >= 0 ? wave_dot(h, W + (int64_t)v * a.H, a.H, lane) : -INFINITY;
        if (lane == 0) xs[k] = x;
      }
    } else if (wave == 0) {
      const float x = wave_dot(h, W + (int64_t)a.l.idx[r] * a.H, a.H, lane);
      if (lane == 0) xs[0] = x;
    }
    __syncthreads();
    if (wave == 0) {
      m = red_m[0];
      s = red_s[0];
#pragma unroll
      for (int k = 1; k < kWaves; ++k) lse_join(m, s, red_m[k], red_s[k], a.l.c);
      lm_loss_finish<DISTILL>(a, i, r, m, s, !DISTILL ? xs[0] : lane < a.l.K ? xs[lane] : -INFINITY);
    }
  }
  total_by_last<kThreads>(a.l);
}

// g of one piece of the vocabulary (columns c0 .. c0 + cols - 1): a run of
// 256 x 256 tiles per workgroup, zeros past the columns and in the rows that pad
// the rows in play.
template <bool DISTILL>
__global__ __launch_bounds__(kThreads, 1) void k_lm_loss_g(LmLossArgs a) {
  __shared__ __align__(16) bf16_t lds[2 * kBufElems];
  const int64_t n = a.plan->n;
  const int nrt = (int)((n + TM - 1) / TM), nct = (a.cols + TN - 1) / TN;
  if (n == 0) return;
  const int length = a.plan->g_run, runs = (nct + length - 1) / length;
  if ((int64_t)blockIdx.x >= (int64_t)nrt * runs) return;
  int rt, run;
  tile_of(blockIdx.x, nrt, runs, rt, run);
  const int64_t row0 = (int64_t)rt * TM, i = row0 + nt_lane_row();
  NtRows src{static_cast<const bf16_t*>(a.w) + (int64_t)a.c0 * a.H, a.hp, a.cols, row0, n, a.H, run * length,
             min(nct, (run + 1) * length)};
  nt_stream(lds, src, [&](int tile, NtAcc& acc) {
    nt_row_per_lane(acc);
    if (i >= lm_loss_pad(n)) return;
    const uint32_t keep = i < n ? ~0u : 0u;  // (what lies behind the rows in play gives zeros, whatever x is)
    const float4 st = i < n ? a.stat[i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const int label = !DISTILL && i < n ? a.l.idx[a.rows[i]] - a.c0 : -1;
    // (x c - m c in one operation saved no time, 2961 and 2968 us for both gradients of 9001
    // rows of 32 000 x 2048, and is no number where m c or its rounding leaves float32's range)
    bf16_t* G = a.g + i * a.ldg;
#pragma unroll 1
    for (int ch = 0; ch < 16; ++ch) {
      const int col = tile * TN + nt_chunk_col(ch);
      float x[8], g[8];
      nt_chunk(acc, ch, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = st.y * lse_term(x[j], st.x, a.l.c);
      if (!DISTILL && (uint32_t)(label - col) < 8u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] -= col + j == label ? st.z : 0.0f;
      }
      if (col + 8 > a.cols) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j >= a.cols) g[j] = 0.0f;
      }
      *reinterpret_cast<uint4*>(G + col) =
          make_uint4(pack_bf16x2(g[0], g[1]) & keep, pack_bf16x2(g[2], g[3]) & keep, pack_bf16x2(g[4], g[5]) & keep,
                     pack_bf16x2(g[6], g[7]) & keep);
    }
  });
}

// A row's members in columns [lo, hi), each from its own logit and by the first of
// the members that name the column.  By a wavefront.
__device__ __forceinline__ void lm_loss_fix(const LmLossArgs& a, int64_t i, int lo, int hi) {
  const int lane = threadIdx.x & 63, K = a.l.K;
  const int64_t r = a.rows[i];
  const int id = lane < K ? a.mid[r * K + lane] : -1;
  const float p = lane < K ? a.mp[r * K + lane] : 0.0f;
  float sum = 0.0f;
  bool first = id >= lo && id < hi;
  for (int k = 0; k < K; ++k) {
    const bool same = lane_i(id, k) == id;
    sum += same ? lane_f(p, k) : 0.0f;
    first = first && !(same && k < lane);
  }
  if (!first) return;
  const float4 st = a.stat[i];
  store1(a.g + i * a.ldg + (id - a.c0), st.y * lse_term(a.mx[i * K + lane], st.x, a.l.c) - st.z * sum);
}

// The distillation's members of that piece.  One wavefront per row (6300 rows of 16
// in 9 us, the latency of its reads).
__global__ __launch_bounds__(256) void k_lm_loss_fix(LmLossArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 4 + wave_id();
  if (i < a.plan->n) lm_loss_fix(a, i, a.c0, a.c0 + a.cols);
}

// g of a piece from the logits that few rows' products left: 2048 columns of row
// blockIdx.y per workgroup.  Bound by 6 bytes per element (48 rows of 32 000 in 5 us).
constexpr int kFewGCols = 8 * 256;
template <bool DISTILL>
__global__ __launch_bounds__(256) void k_lm_loss_few_g(LmLossArgs a) {
  const int n = a.plan->n, i = blockIdx.y, first = blockIdx.x * kFewGCols, col = first + threadIdx.x * 8;
  if (i >= (int)lm_loss_pad(n)) return;
  if (col < (a.cols + kLmTile - 1) / kLmTile * kLmTile) {
    float g[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (i < n && col < a.cols) {
      const float4* X = reinterpret_cast<const float4*>(a.x + (int64_t)i * lm_few_ldx(a.l.V) + a.c0 + col);
      const float4 lo = X[0], hi = X[1], st = a.stat[i];
      const float x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      const int label = DISTILL ? -1 : a.l.idx[a.rows[i]] - a.c0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + j < a.cols) g[j] = st.y * lse_term(x[j], st.x, a.l.c) - (col + j == label ? st.z : 0.0f);
    }
    *reinterpret_cast<uint4*>(a.g + (int64_t)i * a.ldg + col) =
        make_uint4(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]), pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7]));
  }
  if (!DISTILL || i >= n) return;
  __syncthreads();  // (the row's stores before its members')
  if (wave_id() == 0) lm_loss_fix(a, i, a.c0 + first, a.c0 + min(first + kFewGCols, a.cols));
}

// dh of a piece: 256 x 256 tiles of g W, the piece's columns in `splits` ranges
// of `per`.  One piece and one range write the rounded result; otherwise
// acc[range] holds the fp32 sums, which the last piece (one range) or
// k_lm_loss_out turns into the result.
__device__ __forceinline__ void lm_loss_dh(const LmLossArgs& a, bf16_t* lds, int pid, int nrt) {
  const int lane = threadIdx.x & 63, w = wave_id();
  const int64_t n = a.plan->n;
  const int nct = (a.H + TN - 1) / TN, per = a.plan->per, tiles = nrt * nct;
  const int z = pid / tiles, k0 = z * per, K = min(per, a.cols - k0);
  if (K <= 0) return;  // (a short last piece)
  int rt, ct;
  tile_of(pid % tiles, nrt, nct, rt, ct);
  const int64_t row0 = (int64_t)rt * TM;
  const int n0 = ct * TN;
  const bool add = a.c0 > 0, out = a.plan->splits == 1 && a.c0 + a.cols == a.l.V;
  float* sums = a.acc + (int64_t)z * n * a.H;
  NtTile<KRows<false>, false> src{{static_cast<const bf16_t*>(a.w) + (int64_t)(a.c0 + k0) * a.H, a.H, a.H, n0, K},
                                  {a.g + k0, a.ldg, row0, n, K},
                                  K};
  nt_stream(lds, src, [&](int, NtAcc& acc) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int64_t i = row0 + g * 128 + (w & 3) * 32 + (lane & 31);
      if (i >= n) continue;
      bf16_t* D = static_cast<bf16_t*>(a.dh) + (int64_t)a.rows[i] * a.H;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = n0 + (q >> 1) * 128 + (w >> 2) * 64 + (lane >> 5) * 32 + (q & 1) * 16;
        if (col >= a.H) continue;  // H and col are multiples of 16
        const f32x16& c = acc[q >> 1][g][q & 1];
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          float v[8] = {c[e], c[e + 1], c[e + 2], c[e + 3], c[e + 4], c[e + 5], c[e + 6], c[e + 7]};
          if (add) {
            float o[8];
            load8(sums + i * a.H + col + e, o);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += o[j];
          }
          if (out)
            store8(D + col + e, v);
          else
            store8(sums + i * a.H + col + e, v);
        }
      }
    }
  });
}

// dW of a piece: 256 x 256 tiles of g^T h over the rows in play (whole stages:
// the rows behind them are zeros in both operands), the rows in `dw_splits` ranges
// where the tiles are few: their fp32 sums then go to wacc and k_lm_loss_out
// adds them.
template <typename T>
__device__ __forceinline__ void lm_loss_dw(const LmLossArgs& a, bf16_t* lds, int pid) {
  const int lane = threadIdx.x & 63, w = wave_id();
  const int all = (int)lm_loss_pad(a.plan->n), splits = a.plan->dw_splits;
  const int nrt = (a.cols + TM - 1) / TM, nct = (a.H + TN - 1) / TN;
  const int z = splits > 1 ? pid / (nrt * nct) : 0, k0 = z * a.plan->dw_per;
  const int K = splits > 1 ? min(a.plan->dw_per, all - k0) : all;
  int rt, ct;
  tile_of(splits > 1 ? pid % (nrt * nct) : pid, nrt, nct, rt, ct);
  const int row0 = rt * TM, n0 = ct * TN;
  auto write_to = [&](auto* D, const NtAcc& acc) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int row = row0 + g * 128 + (w & 3) * 32 + (lane & 31);
      if (row >= a.cols) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = n0 + (q >> 1) * 128 + (w >> 2) * 64 + (lane >> 5) * 32 + (q & 1) * 16;
        if (col >= a.H) continue;  // H and col are multiples of 16
        const f32x16& c = acc[q >> 1][g][q & 1];
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          const float v[8] = {c[e], c[e + 1], c[e + 2], c[e + 3], c[e + 4], c[e + 5], c[e + 6], c[e + 7]};
          store8(D + (int64_t)row * a.H + col + e, v);
        }
      }
    }
  };
  auto write = [&](const NtAcc& acc) {
    if (splits > 1)
      write_to(a.wacc + (int64_t)z * a.cols * a.H, acc);
    else
      write_to(static_cast<T*>(a.dw) + (int64_t)a.c0 * a.H, acc);
  };
  if (K == 0) {  // no row in play
    NtAcc acc;
#pragma unroll
    for (int q = 0; q < 8; ++q) acc[q >> 2][(q >> 1) & 1][q & 1] = f32x16{};
    write(acc);
    return;
  }
  NtTile<KMajor<false, false>, true> src{{a.hp + (int64_t)k0 * a.H, a.H, a.H, n0, K},
                                         {a.g + (int64_t)k0 * a.ldg, a.ldg, a.ldg, row0, K},
                                         K};
  nt_stream(lds, src, [&](int, NtAcc& acc) { write(acc); });
}

// The two products that read a piece's g in one launch: dh's few long ones
// first, dW's many short ones (T: its type; void: none) fill the CUs behind them.
template <typename T>
__global__ __launch_bounds__(kThreads, 1) void k_lm_loss_grads(LmLossArgs a) {
  __shared__ __align__(16) bf16_t lds[2 * kBufElems];
  const int nrt = (int)((a.plan->n + TM - 1) / TM), nht = (a.H + TN - 1) / TN;
  const int64_t ndh = (int64_t)nrt * nht * a.plan->splits, pid = blockIdx.x;
  if (pid < ndh) {
    lm_loss_dh(a, lds, (int)pid, nrt);
    return;
  }
  if constexpr (!std::is_void_v<T>) {
    if (pid - ndh < (int64_t)((a.cols + TM - 1) / TM) * nht * a.plan->dw_splits) lm_loss_dw<T>(a, lds, (int)(pid - ndh));
  }
}

// What is left after the products, eight columns per thread: the ranges' sums of dh
// (out_dh workgroups), those of a piece's dW (out_dw; T: its type), the total.
template <typename T>
__global__ __launch_bounds__(256) void k_lm_loss_out(LmLossArgs a) {
  const int64_t b = blockIdx.x;
  if (b >= a.out_dh + a.out_dw) {
    row_total<256>(a.l.loss, a.l.weight, a.l.R, a.l.scale, a.l.total);
    return;
  }
  const bool dh = b < a.out_dh;
  const int splits = dh ? a.plan->splits : a.plan->dw_splits;
  const int64_t at = ((b - (dh ? 0 : a.out_dh)) * 256 + threadIdx.x) * 8;
  const int64_t all = (dh ? (int64_t)a.plan->n : (int64_t)a.cols) * a.H;
  if (splits == 1 || at >= all) return;
  const float* sums = dh ? a.acc : a.wacc;
  float v[8];
  load8(sums + at, v);
#pragma unroll 4
  for (int z = 1; z < splits; ++z) {
    float o[8];
    load8(sums + z * all + at, o);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += o[j];
  }
  if (dh)
    store8(static_cast<bf16_t*>(a.dh) + (int64_t)a.rows[at / a.H] * a.H + at % a.H, v);
  else
    store8(static_cast<T*>(a.dw) + (int64_t)a.c0 * a.H + at, v);
}
