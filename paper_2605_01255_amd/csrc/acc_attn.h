// Attention over packed documents, forward and backward (the operator between a decoder layer's projections).
//
//   z_ij = f(scale q_i . k_j) - slope |i - j|,  f(x) = cap tanh(x / cap) or x;   P = softmax over the keys that i sees;   O = P V
//   dV = P^T dO;  dS = P o (dO V^T - delta) f',  delta_i = dO_i . O_i;  dQ = scale dS K;  dK = scale dS^T Q
//
// Every mask is an interval of keys per query, [lo_i, hi_i), and turned round an interval of queries per key: documents give both ends,
// causality and a document's prefix the upper, a window the lower.  A work-group has one document's rows only, and transfers rows of the
// interval it needs only, so what other documents and rows of no document hold reaches nothing.
//
// Blocks of 32 x 32 on the matrix pipe (bfloat16: 32x32x16, float: 32x32x2).  Scores are formed transposed, the contracted index of the
// product behind them in the registers and the other one in the lane: accumulator register r of lane l holds row 8 (r / 4) + 4 (l / 32) + r % 4
// of column l % 32, and the eight registers 8 u .. 8 u + 7 are, rounded, exactly the operand of that product's step of 16 rows if its other
// operand takes the rows in the same order.  So probabilities never pass through LDS, a row's softmax is a reduction within a lane and one
// exchange with lane l + 32, and the running factors are one value a lane.  The other operand is read from row-major tiles by transposing
// LDS reads.  Tiles come by direct global -> LDS transfers, one ahead.
#pragma once
#include "acc_tile32.h"

namespace acc {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnParams {
  const void *q, *k, *v, *dout;
  const void* o_in;
  void *o, *dq, *dk, *dv;
  float *lse, *delta;
  const int64_t *starts, *prefix;
  const float* slopes;
  int64_t ldq, ldk, ldv, ldo;   // elements
  int n, docs, seq;             // docs == 0: sequences of seq rows
  int heads, kv_heads, group, d;
  int tiles;                    // of one head, those that hold no row included
  int causal, window;
  float c2, scale;              // scale log2 e, scale
  float cap2, inv_cap;          // cap log2 e (0: none), scale / cap
};

// ---- which rows a work-group has -----------------------------------------------------------------------------
struct AttnRows {
  int head, first;     // its first row
  int begin, end;      // the document's rows
  int prefix_end;
  bool empty, dead;    // no row at all; rows of no document
};

// Work-group -> head and tile.  An XCD (work-groups are dealt round-robin to the eight) has a contiguous run of (head, tile), so that its
// L2 holds the few heads it is at; last tiles first, which have the most keys where the mask is causal.
// A document's tiles start at its first row.  Tile number t belongs to document e (0: the rows before the first, docs + 1: those behind the
// last) where e is the last with b_e / BM + e <= t, b_e its first row: these numbers rise by at least the document's tiles from one to the next.
template <int BM> __device__ __forceinline__ AttnRows attn_rows(const AttnParams& p, int heads, int lane, bool last_first) {
  AttnRows w{};
  const int64_t total = (int64_t)heads * p.tiles, per = (total + 7) >> 3;
  const int64_t id = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  w.empty = (int64_t)(blockIdx.x >> 3) >= per || id >= total;
  if (w.empty) return w;
  w.head = (int)(id / p.tiles);
  int t = (int)(id - (int64_t)w.head * p.tiles);
  if (last_first) t = p.tiles - 1 - t;
  int doc, tile;
  if (p.docs == 0) {
    const int per_seq = (p.seq + BM - 1) / BM;
    doc = t / per_seq;
    tile = t - doc * per_seq;
    w.begin = doc * p.seq;
    w.end = p.n - w.begin < p.seq ? p.n : w.begin + p.seq;
  } else {
    auto bound = [&](int e) {
      if (e <= 0) return 0;
      if (e > p.docs + 1) return p.n;
      const int64_t b = p.starts[e - 1];
      return b < 0 ? 0 : b > p.n ? p.n : (int)b;
    };
    int lo = 0, hi = p.docs + 2;   // the document is in [lo, hi)
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) >> 6, e = lo + lane * step;
      const bool before = e < hi && bound(e) / BM + e <= t;
      const int count = __popcll(__ballot(before));
      lo += (count > 1 ? count - 1 : 0) * step;
      hi = lo + step < hi ? lo + step : hi;
    }
    doc = __builtin_amdgcn_readfirstlane(lo);
    w.begin = __builtin_amdgcn_readfirstlane(bound(doc));
    w.end = __builtin_amdgcn_readfirstlane(bound(doc + 1));
    tile = t - (w.begin / BM + doc);
    w.dead = doc == 0 || doc == p.docs + 1;
    --doc;
  }
  w.first = w.begin + tile * BM;
  if (tile < 0 || w.first >= w.end) {
    w.empty = true;
    return w;
  }
  w.prefix_end = w.begin;
  if (p.prefix && !w.dead) {
    int64_t m = p.prefix[doc];
    if (m > w.end - w.begin) m = w.end - w.begin;
    if (m > 0) w.prefix_end = w.begin + __builtin_amdgcn_readfirstlane((int)m);
  }
  return w;
}

// Keys that query i sees.
__device__ __forceinline__ int keys_lo(const AttnParams& p, const AttnRows& w, int i) {
  if (!p.window) return w.begin;
  const int lo = i - p.window + 1;
  return lo > w.begin ? lo : w.begin;
}
__device__ __forceinline__ int keys_hi(const AttnParams& p, const AttnRows& w, int i) {
  if (!p.causal) return w.end;
  return i + 1 > w.prefix_end ? i + 1 : w.prefix_end;
}
// Queries that see key j.
__device__ __forceinline__ int queries_lo(const AttnParams& p, const AttnRows& w, int j) { return !p.causal || j < w.prefix_end ? w.begin : j; }
__device__ __forceinline__ int queries_hi(const AttnParams& p, const AttnRows& w, int j) {
  return p.window && p.window < w.end - j ? j + p.window : w.end;
}

// Scores of one block (S, row 4 h of it at `at`, this lane's own row `own`) to their logits in units of log 2, in place, and the cap's
// derivative; where there is neither cap nor bias they stay products, and the factor p.c2 is applied with the subtraction of the maximum.
template <typename T, bool GRAD>
__device__ __forceinline__ f32x16 shape_scores(const AttnParams& p, f32x16 s, float slope2, int at, int own, f32x16* slope_of_cap) {
  if (p.cap2 > 0.f) {
    f32x16 x = s * p.inv_cap, inv;
    for_regs([&](int r) { inv[r] = __builtin_amdgcn_rcpf(1.f + fast_exp2(x[r] * (2.f * kLog2e))); });   // (1 - tanh x) / 2
    if constexpr (sizeof(T) == 2) s = p.cap2 * (1.f - 2.f * inv);
    else for_regs([&](int r) { s[r] = p.cap2 * tanhf(x[r]); });
    if constexpr (GRAD) *slope_of_cap = 4.f * inv * (1.f - inv);
  } else {
    s *= p.c2;
  }
  if (slope2 != 0.f) {
    const float gap = (float)(at - own);
    for_regs([&](int r) { s[r] -= slope2 * fabsf(gap + (float)(8 * (r >> 2) + (r & 3))); });
  }
  return s;
}

// ---- forward -------------------------------------------------------------------------------------------------
// A work-group of NW waves has NW x 32 queries of one head; their rows stay in registers as operands.
template <typename T, int DB, int NW> __global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void attn_fwd_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, DB>;
  constexpr int BM = NW * 32, BN = Tile::BN, KB = BN / 32;
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AttnRows w = attn_rows<BM>(p, p.heads, lane, true);
  if (w.empty) return;
  const int kv = w.head / p.group;
  const int w0 = w.first + wave * 32;                        // this wave's rows
  const int w1 = w0 + 31 < w.end ? w0 + 31 : w.end - 1;
  const int mine = w0 + c < w.end ? w0 + c : w.end - 1;      // lanes behind the document's end repeat its last row
  const bool there = w0 + c < w.end;

  typename DirectFrag<T>::type qf[Tile::STEPS];
  load_row<T, DB>(qf, (const T*)p.q + (int64_t)w.head * p.d, mine, p.ldq, p.d, h, !w.dead);
  const T* kbase = (const T*)p.k + (int64_t)kv * p.d;
  const T* vbase = (const T*)p.v + (int64_t)kv * p.d;
  const int last = w.first + BM < w.end ? w.first + BM - 1 : w.end - 1;
  const int k_lo = keys_lo(p, w, w.first), k_hi = w.dead ? k_lo : keys_hi(p, w, last);
  const int lo = keys_lo(p, w, mine), span = keys_hi(p, w, mine) - lo;
  const int full_lo = keys_lo(p, w, w1), full_hi = keys_hi(p, w, w0);       // tiles inside are seen whole by the wave
  const int any_lo = keys_lo(p, w, w0), any_hi = keys_hi(p, w, w1);         // tiles outside not at all
  const bool shaped = p.cap2 > 0.f || p.slopes;
  const float slope2 = p.slopes ? p.slopes[w.head] * kLog2e : 0.f, c2 = shaped ? 1.f : p.c2;

  const Tile32Reads<T, DB> at(lane);
  const Tile32Loader<T, DB, NW> kload(lane, wave, p.ldk, p.d), vload(lane, wave, p.ldv, p.d);
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16{};
  float m = -INFINITY, l = 0.f;

  const int tiles = (k_hi - k_lo + BN - 1) / BN;
  auto issue = [&](int t) {
    const int row = k_lo + t * BN;
    const uint32_t stage = lds + (t & 1) * 2 * Tile::BYTES;
    kload.issue(kbase, row, k_hi - row, p.ldk, p.d, stage, wave);
    vload.issue(vbase, row, k_hi - row, p.ldv, p.d, stage + Tile::BYTES, wave);
  };
  if (tiles > 0) issue(0);
  for (int t = 0; t < tiles; ++t) {
    wait_vmcnt0();
    __syncthreads();
    if (t + 1 < tiles) issue(t + 1);
    const int k0 = k_lo + t * BN;
    if (w0 >= w.end || k0 >= any_hi || k0 + BN <= any_lo) continue;
    const char* ks = smem + (t & 1) * 2 * Tile::BYTES;
    const char* vs = ks + Tile::BYTES;
    f32x16 s[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) s[b] = f32x16{};
    products<KB * Tile::STEPS, 4>([&](auto i) { return at.row(ks + Tile::block(i.value / Tile::STEPS), i.value % Tile::STEPS); },
                                  [&](auto i, auto k) { mma(s[i.value / Tile::STEPS], k, qf[i.value % Tile::STEPS]); });
    if (shaped) {
#pragma unroll
      for (int b = 0; b < KB; ++b) s[b] = shape_scores<T, false>(p, s[b], slope2, k0 + 32 * b + 4 * h, mine, nullptr);
    }
    if (k0 < full_lo || k0 + BN > full_hi) {
      const int base = k0 + 4 * h - lo;
#pragma unroll
      for (int b = 0; b < KB; ++b)
        for_regs([&](int r) { if ((uint32_t)(base + 32 * b + 8 * (r >> 2) + (r & 3)) >= (uint32_t)span) s[b][r] = -INFINITY; });
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < KB; ++b)
      for_regs([&](int r) { top = fmaxf(top, s[b][r]); });
    top = half_max(top) * c2;
    if (__any(top > m)) {
      const float next = fmaxf(m, top), by = fast_exp2(m - (next == -INFINITY ? 0.f : next));
      m = next;
      l *= by;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        o[db] *= by;
    }
    const float minus = m == -INFINITY ? 0.f : -m;
#pragma unroll
    for (int b = 0; b < KB; ++b)
      for_regs([&](int r) {
        s[b][r] = fast_exp2(__builtin_fmaf(s[b][r], c2, minus));
        l += s[b][r];
      });
    typename TransFrag<T>::type pf[2 * KB];
#pragma unroll
    for (int u = 0; u < 2 * KB; ++u) pf[u] = step_operand<T>(s[u / 2], u & 1);
    products<2 * KB * DB, 4>([&](auto i) { return at.column(vs, i.value / DB, i.value % DB); },
                             [&](auto i, auto v) { mma(o[i.value % DB], v, pf[i.value / DB]); });
  }
  if (!there) return;
  l = half_sum(l);
  store_row<T, DB>((T*)p.o + (int64_t)mine * p.ldo + (int64_t)w.head * p.d, o, l == 0.f ? 0.f : 1.f / l, p.d, h);
  if (h == 0) p.lse[(int64_t)w.head * p.n + mine] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---- backward: gradient of the queries -----------------------------------------------------------------------
// As the forward pass; delta = dO . O of this work-group's rows is formed on the way and kept for the keys' gradient.
template <typename T, int DB, int NW> __global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void attn_dq_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, DB>;
  constexpr int BM = NW * 32, BN = Tile::BN, KB = BN / 32;
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AttnRows w = attn_rows<BM>(p, p.heads, lane, true);
  if (w.empty) return;
  const int kv = w.head / p.group;
  const int w0 = w.first + wave * 32;
  const int w1 = w0 + 31 < w.end ? w0 + 31 : w.end - 1;
  const int mine = w0 + c < w.end ? w0 + c : w.end - 1;
  const bool there = w0 + c < w.end;

  typename DirectFrag<T>::type qf[Tile::STEPS], df[Tile::STEPS];
  load_row<T, DB>(qf, (const T*)p.q + (int64_t)w.head * p.d, mine, p.ldq, p.d, h, !w.dead);
  load_row<T, DB>(df, (const T*)p.dout + (int64_t)w.head * p.d, mine, p.ldo, p.d, h, !w.dead);
  float delta = 0.f;
  {
    typename DirectFrag<T>::type of[Tile::STEPS];
    load_row<T, DB>(of, (const T*)p.o_in + (int64_t)w.head * p.d, mine, p.ldo, p.d, h, !w.dead);
#pragma unroll
    for (int s = 0; s < Tile::STEPS; ++s)
#pragma unroll
      for (int e = 0; e < Tile::PER_CHUNK; ++e) delta += (float)of[s][e] * (float)df[s][e];
    delta = half_sum(delta);
  }
  const int64_t row = (int64_t)w.head * p.n + mine;
  if (there && h == 0) p.delta[row] = delta;
  const float lse2 = w.dead ? 0.f : p.lse[row] * kLog2e;
  const float minus = lse2 == -INFINITY ? -INFINITY : -lse2;   // a row without keys has no probabilities

  const T* kbase = (const T*)p.k + (int64_t)kv * p.d;
  const T* vbase = (const T*)p.v + (int64_t)kv * p.d;
  const int last = w.first + BM < w.end ? w.first + BM - 1 : w.end - 1;
  const int k_lo = keys_lo(p, w, w.first), k_hi = w.dead ? k_lo : keys_hi(p, w, last);
  const int lo = keys_lo(p, w, mine), span = keys_hi(p, w, mine) - lo;
  const int full_lo = keys_lo(p, w, w1), full_hi = keys_hi(p, w, w0);
  const int any_lo = keys_lo(p, w, w0), any_hi = keys_hi(p, w, w1);
  const bool shaped = p.cap2 > 0.f || p.slopes;
  const float slope2 = p.slopes ? p.slopes[w.head] * kLog2e : 0.f, c2 = shaped ? 1.f : p.c2;

  const Tile32Reads<T, DB> at(lane);
  const Tile32Loader<T, DB, NW> kload(lane, wave, p.ldk, p.d), vload(lane, wave, p.ldv, p.d);
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = f32x16{};
  const int tiles = (k_hi - k_lo + BN - 1) / BN;
  auto issue = [&](int t) {
    const int r = k_lo + t * BN;
    const uint32_t stage = lds + (t & 1) * 2 * Tile::BYTES;
    kload.issue(kbase, r, k_hi - r, p.ldk, p.d, stage, wave);
    vload.issue(vbase, r, k_hi - r, p.ldv, p.d, stage + Tile::BYTES, wave);
  };
  if (tiles > 0) issue(0);
  for (int t = 0; t < tiles; ++t) {
    wait_vmcnt0();
    __syncthreads();
    if (t + 1 < tiles) issue(t + 1);
    const int k0 = k_lo + t * BN;
    if (w0 >= w.end || k0 >= any_hi || k0 + BN <= any_lo) continue;
    const char* ks = smem + (t & 1) * 2 * Tile::BYTES;
    const char* vs = ks + Tile::BYTES;
    const bool masked = k0 < full_lo || k0 + BN > full_hi;
    static_for<0, KB>([&](auto block) {
      constexpr int b = decltype(block)::value;
      f32x16 s{}, dp{}, by{};
      products<2 * Tile::STEPS, 4>([&](auto i) { return at.row((i.value < Tile::STEPS ? ks : vs) + Tile::block(b), i.value % Tile::STEPS); },
                                   [&](auto i, auto x) {
                                     if constexpr (i.value < Tile::STEPS) mma(s, x, qf[i.value]);
                                     else mma(dp, x, df[i.value - Tile::STEPS]);
                                   });
      if (shaped) s = shape_scores<T, true>(p, s, slope2, k0 + 32 * b + 4 * h, mine, &by);
      for_regs([&](int r) { s[r] = fast_exp2(__builtin_fmaf(s[r], c2, minus)) * (dp[r] - delta); });
      if (p.cap2 > 0.f) s *= by;
      if (masked) {
        const int base = k0 + 32 * b + 4 * h - lo;
        for_regs([&](int r) { if ((uint32_t)(base + 8 * (r >> 2) + (r & 3)) >= (uint32_t)span) s[r] = 0.f; });
      }
      const typename TransFrag<T>::type sf[2] = {step_operand<T>(s, 0), step_operand<T>(s, 1)};
      products<2 * DB, 4>([&](auto i) { return at.column(ks, 2 * b + i.value / DB, i.value % DB); },
                          [&](auto i, auto k) { mma(dq[i.value % DB], k, sf[i.value / DB]); });
    });
  }
  if (there) store_row<T, DB>((T*)p.dq + (int64_t)mine * p.ldq + (int64_t)w.head * p.d, dq, p.scale, p.d, h);
}

// ---- backward: gradients of the keys and values --------------------------------------------------------------
// A work-group has 128 keys of one key head, 32 for each of four waves, and goes over the queries of the heads that share it, so that the sum
// over them is taken in its accumulators.  bfloat16: eight waves, two for the same keys, which take the two halves of a tile of queries and add
// their sums up at the end; the keys' rows stay in LDS.  (Two waves a SIMD need 256 registers each, of which the sums take 128: with the
// keys' rows in registers too there is one, and nothing runs while it waits.)  float: four waves, the keys' rows in registers.
template <typename T, int DB> struct DkvLayout {
  using Tile = Tile32<T, DB>;
  static constexpr int HALVES = sizeof(T) == 2 ? 2 : 1, NW = 4 * HALVES, BM = 128, BQ = Tile::BN;
  static constexpr int KEYS = HALVES == 2 ? 2 * (BM / Tile::BN) * Tile::BYTES : 0;   // bytes of K and V
  static constexpr int STAGE = 2 * Tile::BYTES + 512;   // queries, their outputs' gradients, log-sum-exps and deltas
  static constexpr int SUMS = HALVES == 2 ? 4 * DB * 16 * 64 * 4 : 0;   // one half's sums of one tensor
  static constexpr int BYTES = KEYS + 2 * STAGE > SUMS ? KEYS + 2 * STAGE : SUMS;
};

template <typename T, int DB> __global__ __launch_bounds__((DkvLayout<T, DB>::NW * 64), (DkvLayout<T, DB>::HALVES)) void attn_dkv_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, DB>;
  using Layout = DkvLayout<T, DB>;
  constexpr int NW = Layout::NW, BM = Layout::BM, BQ = Layout::BQ, STAGE = Layout::STAGE;
  constexpr bool IN_LDS = Layout::HALVES == 2;
  constexpr int QB = BQ / 32 / Layout::HALVES;   // blocks of queries of a wave
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), key_wave = wave & 3, half = wave >> 2;
  const AttnRows w = attn_rows<BM>(p, p.kv_heads, lane, false);
  if (w.empty) return;
  const int w0 = w.first + key_wave * 32;
  const int w1 = w0 + 31 < w.end ? w0 + 31 : w.end - 1;
  const int mine = w0 + c < w.end ? w0 + c : w.end - 1;
  const bool there = w0 + c < w.end;

  const T* kbase = (const T*)p.k + (int64_t)w.head * p.d;
  const T* vbase = (const T*)p.v + (int64_t)w.head * p.d;
  const int last = w.first + BM < w.end ? w.first + BM - 1 : w.end - 1;
  const int q_lo = queries_lo(p, w, w.first), q_hi = w.dead ? q_lo : queries_hi(p, w, last);
  const int lo = queries_lo(p, w, mine), span = queries_hi(p, w, mine) - lo;
  const int full_lo = queries_lo(p, w, w1), full_hi = queries_hi(p, w, w0);
  const int any_lo = queries_lo(p, w, w0), any_hi = queries_hi(p, w, w1);
  const bool shaped = p.cap2 > 0.f || p.slopes;
  const float c2 = shaped ? 1.f : p.c2;

  const Tile32Reads<T, DB> at(lane);
  const Tile32Loader<T, DB, NW> qload(lane, wave, p.ldq, p.d), dload(lane, wave, p.ldo, p.d);
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  typename DirectFrag<T>::type kf[IN_LDS ? 1 : Tile::STEPS], vf[IN_LDS ? 1 : Tile::STEPS];
  const char *ks = smem + Tile::block(key_wave), *vs = ks + Layout::KEYS / 2;   // this wave's keys
  if constexpr (IN_LDS) {
    if (!w.dead) {
      const Tile32Loader<T, DB, NW> kload(lane, wave, p.ldk, p.d), vload(lane, wave, p.ldv, p.d);
#pragma unroll
      for (int i = 0; i < BM / Tile::BN; ++i) {
        const int row = w.first + i * Tile::BN;   // (a tile behind the document's end is not read)
        if (row >= w.end) continue;
        kload.issue(kbase, row, w.end - row, p.ldk, p.d, lds + i * Tile::BYTES, wave);
        vload.issue(vbase, row, w.end - row, p.ldv, p.d, lds + Layout::KEYS / 2 + i * Tile::BYTES, wave);
      }
    }
  } else {
    load_row<T, DB>(kf, kbase, mine, p.ldk, p.d, h, !w.dead);
    load_row<T, DB>(vf, vbase, mine, p.ldv, p.d, h, !w.dead);
  }
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = f32x16{};
  const int per_head = (q_hi - q_lo + BQ - 1) / BQ, tiles = per_head * p.group;
  auto issue = [&](int head, int tile, int t) {
    const int row = q_lo + tile * BQ;
    const uint32_t stage = lds + Layout::KEYS + (t & 1) * STAGE;
    qload.issue((const T*)p.q + (int64_t)head * p.d, row, q_hi - row, p.ldq, p.d, stage, wave);
    dload.issue((const T*)p.dout + (int64_t)head * p.d, row, q_hi - row, p.ldo, p.d, stage + Tile::BYTES, wave);
    if (wave < 2) {
      const int rows = q_hi - row < BQ ? q_hi - row : BQ;
      const u32x4 rsrc = make_rsrc((wave ? p.delta : p.lse) + (int64_t)head * p.n + row, rows * 4);
      buffer_to_lds_b32(rsrc, lane * 4, stage + 2 * Tile::BYTES + wave * 256);
    }
  };
  int head = w.head * p.group, tile = 0, next_head = head, next_tile = 0;
  auto advance = [&](int& a, int& b) {
    if (++b == per_head) {
      b = 0;
      ++a;
    }
  };
  if (tiles > 0) issue(head, 0, 0);
  for (int t = 0; t < tiles; ++t, advance(head, tile)) {
    wait_vmcnt0();
    __syncthreads();
    advance(next_head, next_tile);
    if (t + 1 < tiles) issue(next_head, next_tile, t + 1);
    const int q0 = q_lo + tile * BQ + half * QB * 32;   // this wave's queries
    if (w0 >= w.end || q0 >= any_hi || q0 + QB * 32 <= any_lo) continue;
    const char* qs = smem + Layout::KEYS + (t & 1) * STAGE + Tile::block(half * QB);
    const char* ds = qs + Tile::BYTES;
    const float* stats = (const float*)(smem + Layout::KEYS + (t & 1) * STAGE + 2 * Tile::BYTES) + half * QB * 32;
    const float slope2 = p.slopes ? p.slopes[head] * kLog2e : 0.f;
    const bool masked = q0 < full_lo || q0 + QB * 32 > full_hi;
    static_for<0, QB>([&](auto block) {
      constexpr int b = decltype(block)::value;
      f32x16 s{}, dp{}, by{};
      using Frag = typename DirectFrag<T>::type;
      if constexpr (IN_LDS) {
        struct Pair { Frag q, k; };
        products<2 * Tile::STEPS, 3>(
            [&](auto i) {
              constexpr bool second = i.value >= Tile::STEPS;
              return Pair{at.row((second ? ds : qs) + Tile::block(b), i.value % Tile::STEPS), at.row(second ? vs : ks, i.value % Tile::STEPS)};
            },
            [&](auto i, const Pair& x) { mma(i.value < Tile::STEPS ? s : dp, x.q, x.k); });
      } else {
        products<2 * Tile::STEPS, 4>([&](auto i) { return at.row((i.value < Tile::STEPS ? qs : ds) + Tile::block(b), i.value % Tile::STEPS); },
                                     [&](auto i, const Frag& x) {
                                       if constexpr (i.value < Tile::STEPS) mma(s, x, kf[i.value]);
                                       else mma(dp, x, vf[i.value - Tile::STEPS]);
                                     });
      }
      if (shaped) s = shape_scores<T, true>(p, s, slope2, q0 + 32 * b + 4 * h, mine, &by);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 lse = *(const f32x4*)(stats + 32 * b + 8 * g + 4 * h), delta = *(const f32x4*)(stats + 64 + 32 * b + 8 * g + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          const float minus = lse[e] == -INFINITY ? -INFINITY : lse[e] * -kLog2e;
          s[r] = fast_exp2(__builtin_fmaf(s[r], c2, minus));
          dp[r] = s[r] * (dp[r] - delta[e]);
        }
      }
      if (p.cap2 > 0.f) dp *= by;
      if (masked) {
        const int base = q0 + 32 * b + 4 * h - lo;
        for_regs([&](int r) { if ((uint32_t)(base + 8 * (r >> 2) + (r & 3)) >= (uint32_t)span) s[r] = dp[r] = 0.f; });
      }
      const typename TransFrag<T>::type pf[2] = {step_operand<T>(s, 0), step_operand<T>(s, 1)}, sf[2] = {step_operand<T>(dp, 0), step_operand<T>(dp, 1)};
      products<4 * DB, 4>([&](auto i) { return at.column(i.value & 1 ? qs : ds, 2 * b + i.value / 2 / DB, i.value / 2 % DB); },
                          [&](auto i, auto x) {
                            if constexpr (i.value & 1) mma(dk[i.value / 2 % DB], x, sf[i.value / 2 / DB]);
                            else mma(dv[i.value / 2 % DB], x, pf[i.value / 2 / DB]);
                          });
    });
  }
  if constexpr (IN_LDS) {   // the second half's sums to the first
    wait_vmcnt0();
    float* sums = (float*)smem + key_wave * DB * 16 * 64 + lane;
    auto meet = [&](f32x16* x) {
      __syncthreads();
      if (half) {
#pragma unroll
        for (int db = 0; db < DB; ++db) for_regs([&](int r) { sums[(db * 16 + r) * 64] = x[db][r]; });
      }
      __syncthreads();
      if (!half) {
#pragma unroll
        for (int db = 0; db < DB; ++db) for_regs([&](int r) { x[db][r] += sums[(db * 16 + r) * 64]; });
      }
    };
    meet(dk);
    meet(dv);
    if (half) return;
  }
  if (!there) return;
  store_row<T, DB>((T*)p.dk + (int64_t)mine * p.ldk + (int64_t)w.head * p.d, dk, p.scale, p.d, h);
  store_row<T, DB>((T*)p.dv + (int64_t)mine * p.ldv + (int64_t)w.head * p.d, dv, 1.f, p.d, h);
}

}  // namespace acc
