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
  float *lse, *minus, *delta;   // minus: -log-sum-exp in units of log 2 (backward)
  const int64_t *starts, *prefix;
  const float* slopes;
  int64_t ldq, ldk, ldv, ldo;   // elements
  int n, docs, seq;             // docs == 0: sequences of seq rows
  int heads, kv_heads, group, d;
  int tiles;                    // of one head, those that hold no row included
  int strands, strand_tiles;    // of one key head's tiles
  int causal, window;
  float c2, scale;              // scale log2 e, scale
  float cap2, inv_cap;          // cap log2 e (0: none), scale / cap
  // Where there are few work-groups each one's tiles are dealt to `parts` of them, which leave float sums here: [parts][n][heads d] (O, dQ) or
  // [parts][2][n][kv_heads d] (dK, dV); part_stats [parts][2][heads][n]: the forward pass' maxima and sums of exponentials.
  float *part, *part_stats;
  int parts;
};

// ---- which rows a work-group has -----------------------------------------------------------------------------
struct AttnRows {
  int head, first;     // its first row
  int begin, end;      // the document's rows
  int prefix_end;
  bool empty, dead;    // no row at all; rows of no document
};

// Work-group -> head and tile.  An XCD (work-groups are dealt round-robin to the eight) has a contiguous run of (key head, strand, tile, `share`
// query heads on it), so that its L2 holds the keys and values that its work-groups are at.  Where the key heads are no multiple of eight
// their tiles are dealt to several strands, or one XCD would have a head's long tiles and the next its short ones.  Last tiles first, which have
// the most keys where the mask is causal.
// (One document of 16384 rows on 4 key heads, forward: 1475 us, with one strand 2000; 6001 rows with a window of 1000 in all 425, 496.)
// A document's tiles start at its first row.  Tile number t belongs to document e (0: the rows before the first, docs + 1: those behind the
// last) where e is the last with b_e / BM + e <= t, b_e its first row: these numbers rise by at least the document's tiles from one to the next.
// A document of whole tiles leaves one number without rows behind it, and with many of them every second or fourth work-group would have none,
// which all fall to the same strands and shader engines: sixteen neighbours are rotated by the number of their run (128 documents of 128 rows,
// 16 heads of 128: forward 65 us, without 104; documents of odd lengths: the same).
template <int BM> __device__ __forceinline__ AttnRows attn_rows(const AttnParams& p, int share, int lane, bool last_first) {
  AttnRows w{};
  const int per = gridDim.x >> 3, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  const int each = p.strand_tiles * share, strand = id / each, in = id - strand * each;
  w.head = strand / p.strands * share + in % share;
  int t = in / share * p.strands + strand % p.strands;
  w.empty = t >= p.tiles;
  if (w.empty) return w;
  if (p.docs * 8 > p.tiles && (t | 15) < p.tiles) t = (t & ~15) | ((t + (t >> 4)) & 15);
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
// Whether row i as a query sees the key i alone.  Its dS, P (dP - delta) with P = 1, is a difference of two sums that are equal but for their
// roundings, and is taken as the zero that it is.  (Tiles that hold such a row are never seen whole.)
__device__ __forceinline__ bool alone(const AttnParams& p, const AttnRows& w, int i) {
  return p.window == 1 || (i == w.begin && (p.causal ? w.prefix_end <= w.begin + 1 : w.end - w.begin == 1));
}

__device__ __forceinline__ void store_quad(float* to, f32x4 x) { *(f32x4*)to = x; }
__device__ __forceinline__ void store_quad(bf16* to, f32x4 x) { *(bf16x4*)to = __builtin_convertvector(x, bf16x4); }

// The part'th of `parts` runs of whole tiles of rows lo .. hi - 1.
template <int BN> __device__ __forceinline__ void part_of(int& lo, int& hi, int part, int parts) {
  if (parts == 1) return;
  const int tiles = (hi - lo + BN - 1) / BN, from = tiles * part / parts, to = tiles * (part + 1) / parts;
  hi = to < tiles ? lo + to * BN : hi;
  lo += from * BN;
}

// Scores of one block (S, row 4 h of it at `at`, this lane's own row `own`) to their logits in units of log 2, in place, and the cap's
// derivative; where there is neither cap nor bias they stay products, and the factor p.c2 is applied with the subtraction of the maximum.
template <typename T, bool GRAD>
__device__ __forceinline__ f32x16 shape_scores(const AttnParams& p, f32x16 s, float slope2, int at, int own, f32x16* slope_of_cap) {
  if (p.cap2 > 0.f) {
    const float twice = here(p.inv_cap * (2.f * kLog2e));   // (in a vector register: sixteen copies of a scalar one are kept otherwise)
    f32x16 inv;
    if constexpr (GRAD || sizeof(T) == 2) for_regs([&](int r) { inv[r] = __builtin_amdgcn_rcpf(1.f + fast_exp2(s[r] * twice)); });   // (1 - tanh x) / 2
    if constexpr (sizeof(T) == 2) {
      const float cap2 = here(p.cap2), minus = here(-2.f * p.cap2);
      for_regs([&](int r) { s[r] = __builtin_fmaf(inv[r], minus, cap2); });
    } else {
      for_regs([&](int r) { s[r] = p.cap2 * tanhf(s[r] * p.inv_cap); });
    }
    if constexpr (GRAD) {
      const f32x16 four = 4.f * inv;
      for_regs([&](int r) { (*slope_of_cap)[r] = __builtin_fmaf(-four[r], inv[r], four[r]); });
    }
  } else {
    s *= here(p.c2);
  }
  if (slope2 != 0.f) {
    const float gap = (float)(at - own);
    for_regs([&](int r) { s[r] -= slope2 * fabsf(gap + (float)(8 * (r >> 2) + (r & 3))); });
  }
  return s;
}

// How far a score may lie above a row's running maximum, in units of log 2, before the maximum is raised: probabilities reach 2^8 then, which
// costs float nothing, and a wave seldom rescales its sums (training step's forward 608 us, with 0 here 669).
constexpr float kSlack = 8.f;
constexpr int kFewKeys = 64;

// ---- forward -------------------------------------------------------------------------------------------------
// A work-group of NW waves has NW x 32 queries of one head; their rows stay in registers as operands.  Tiles of 64 keys (float 32), two in LDS,
// leave room for two work-groups on a compute unit.  Bound by the waits for transfers and barrier (left out, 26 % less; V's transfers are the last
// to go), by power and by the vector instructions beside the matrix ones (six to one, of them one exponential and one maximum a score): 4 x 4096
// rows, 32 heads of 128 on 8, 597 to 654 us, 0.84 to 0.92 PFLOP/s, the matrix pipe busy half of the time; on zeros, at the full clock, 490.
template <typename T, int DB, int NW> __global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void attn_fwd_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, DB>;
  constexpr int BM = NW * 32, BN = Tile::BN, KB = BN / 32;
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  AttnRows w = attn_rows<BM>(p, p.group * p.parts, lane, true);
  if (w.empty) return;
  const int part = w.head % p.parts;
  w.head /= p.parts;
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
  int k_lo = keys_lo(p, w, w.first), k_hi = w.dead ? k_lo : keys_hi(p, w, last);
  part_of<BN>(k_lo, k_hi, part, p.parts);
  const int lo = keys_lo(p, w, mine), span = keys_hi(p, w, mine) - lo;
  const int full_lo = keys_lo(p, w, w1), full_hi = keys_hi(p, w, w0);       // tiles inside are seen whole by the wave
  const int any_lo = keys_lo(p, w, w0), any_hi = keys_hi(p, w, w1);         // tiles outside not at all
  const bool shaped = p.cap2 > 0.f || p.slopes;
  const float slope2 = p.slopes ? p.slopes[w.head] * kLog2e : 0.f, c2 = shaped ? 1.f : p.c2;

  const Tile32Reads<T, DB> at(lane);
  using KVLoader = Tile32Loader<T, DB, NW>;
  const KVLoader kload(lane, wave, p.ldk, p.d), vload(lane, wave, p.ldv, p.d);
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16{};
  float m = -INFINITY, l = 0.f;

  const int tiles = (k_hi - k_lo + BN - 1) / BN;
  constexpr int PIECES = 2 * KVLoader::LOADS;
  Tile32Run<T, DB, NW> krun(kbase, k_lo, k_hi - k_lo, p.ldk, p.d), vrun(vbase, k_lo, k_hi - k_lo, p.ldv, p.d);
  uint32_t stage = lds;
  auto next = [&](int t) {   // tile t's transfers
    stage = lds + (t & 1) * 2 * Tile::BYTES;
    krun.advance(t, tiles);
    vrun.advance(t, tiles);
  };
  auto piece = [&](int i) {
    if (i < KVLoader::LOADS) kload.one(krun.rsrc, i, stage, wave);
    else vload.one(vrun.rsrc, i - KVLoader::LOADS, stage + Tile::BYTES, wave);
  };
  auto pieces = [&]() {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) piece(i);
  };
  if (tiles > 0) pieces();
  for (int t = 0; t < tiles; ++t) {
    wait_vmcnt0();
    __syncthreads();
    next(t + 1);   // (behind the last one: no rows, zeros)
    const int k0 = k_lo + t * BN;
    if (w0 >= w.end || k0 >= any_hi || k0 + BN <= any_lo) {
      pieces();
      continue;
    }
    const char* ks = smem + (t & 1) * 2 * Tile::BYTES;
    const char* vs = ks + Tile::BYTES;
    const bool masked = k0 < full_lo || k0 + BN > full_hi;
    f32x16 s[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) s[b] = f32x16{};
    typename TransFrag<T>::type pf[2];
    float minus = 0.f, by = 1.f;
    bool changed = false;
    // Block b's scores to what their exponentials are taken of.  The maximum that they are relative to is raised where a score is kSlack
    // (powers of 2) above it, not for every new one: probabilities up to 2^kSlack are as exact, and O is hardly ever multiplied.
    auto begin = [&](auto block) {
      constexpr int b = block.value;
      if (shaped) s[b] = shape_scores<T, false>(p, s[b], slope2, k0 + 32 * b + 4 * h, mine, nullptr);
      if (masked) {
        const int base = k0 + 32 * b + 4 * h - lo;
        for_regs([&](int r) { if ((uint32_t)(base + 8 * (r >> 2) + (r & 3)) >= (uint32_t)span) s[b][r] = -INFINITY; });
      }
      float top = fmaxf(s[b][0], s[b][1]);
      static_for<2, 16>([&](auto r) { top = fmaxf(top, s[b][r.value]); });
      top = half_max(top) * c2;
      changed = __any(top > m + kSlack);
      if (changed) {
        const float next = fmaxf(m, top);
        by = fast_exp2(m - (next == -INFINITY ? 0.f : next));
        m = next;
        l *= by;
      }
      minus = m == -INFINITY ? 0.f : -m;
    };
    auto exponential = [&](int b, int r) {
      s[b][r] = here(fast_exp2(__builtin_fmaf(s[b][r], c2, minus)));
      l += s[b][r];
    };
    auto rescale = [&]() {
      if (!changed) return;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= by;
    };
    auto pack = [&](int b) {
      pf[0] = here(step_operand<T>(s[b], 0));
      pf[1] = here(step_operand<T>(s[b], 1));
    };
    // scores of block 0, of block 1 (block 0's exponentials), O of block 0 (block 1's exponentials), O of block 1
    constexpr int LS = Tile::STEPS, LO = 2 * DB;
    products<KB * (LS + LO), sizeof(T) == 2 ? 4 : 1>(
        [&](auto i) {
          if constexpr (i.value < KB * LS) return widened(at.row(ks + Tile::block(i.value / LS), i.value % LS));
          else return at.column(vs, (i.value - KB * LS) / DB, (i.value - KB * LS) % DB);
        },
        [&](auto i, auto x) {
          if constexpr (i.value < KB * LS) mma(s[i.value / LS], narrowed<T>(x), qf[i.value % LS]);
          else mma(o[(i.value - KB * LS) % DB], x, pf[(i.value - KB * LS) / DB % 2]);
        },
        [&](auto i) {
          // the next tile's transfers a few products apart: one after another they hold the wave up
          constexpr int apart = KB * (LS + LO) / PIECES;
          if constexpr (i.value % apart == 0 && i.value / apart < PIECES) piece(i.value / apart);
          if constexpr (KB == 2) {
            constexpr int phase = i.value < 2 * LS ? i.value / LS : 2 + (i.value - 2 * LS) / LO;
            constexpr int step = i.value < 2 * LS ? i.value % LS : (i.value - 2 * LS) % LO, steps = phase < 2 ? LS : LO;
            if constexpr (phase == 1 || phase == 2) {
              constexpr int b = phase - 1;
              if constexpr (step == 0) {
                begin(std::integral_constant<int, b>{});
                if constexpr (b == 0) rescale();
              }
              spread<step, steps>([&](int r) { exponential(b, r); });
              if constexpr (step == steps - 1) {
                pack(b);
                if constexpr (b == 1) rescale();   // block 0's part is in O
              }
            }
          } else if constexpr (i.value == LS - 1) {
            begin(std::integral_constant<int, 0>{});
            rescale();
            for_regs([&](int r) { exponential(0, r); });
            pack(0);
          }
        });
  }
  wait_vmcnt0();
  if (!there) return;
  l = half_sum(l);
  if (p.parts > 1) {
    store_row<float, DB>(p.part + ((int64_t)part * p.n + mine) * p.heads * p.d + (int64_t)w.head * p.d, o, 1.f, p.d, h);
    p.part_stats[((int64_t)(2 * part + h) * p.heads + w.head) * p.n + mine] = h ? l : m;
    return;
  }
  store_row<T, DB>((T*)p.o + (int64_t)mine * p.ldo + (int64_t)w.head * p.d, o, l == 0.f ? 0.f : 1.f / l, p.d, h);
  if (h == 0) p.lse[(int64_t)w.head * p.n + mine] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// O and the log-sum-exps from the parts, four channels a lane: bound by the parts' bytes (1031 rows, 8 heads of 64, five parts: 7 us; 2048 rows, 16
// heads of 128, two: 10.6).
template <typename T> __global__ __launch_bounds__(256) void attn_join_kernel(AttnParams p) {
  const int quads = p.d / 4, row_quads = p.heads * quads;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)p.n * row_quads) return;
  const int64_t row = i / row_quads;
  const int head = (int)(i % row_quads) / quads, c = (int)(i % row_quads) * 4;
  const float* stats = p.part_stats + (int64_t)head * p.n + row;
  const int64_t side = (int64_t)p.heads * p.n;
  float m = -INFINITY;
  for (int k = 0; k < p.parts; ++k) m = fmaxf(m, stats[2 * k * side]);
  float l = 0.f;
  f32x4 sum{};
  for (int k = 0; k < p.parts; ++k) {
    const float by = m == -INFINITY ? 1.f : fast_exp2(stats[2 * k * side] - m);
    l += by * stats[(2 * k + 1) * side];
    sum += by * *(const f32x4*)(p.part + (int64_t)k * p.n * row_quads * 4 + i * 4);
  }
  sum *= l == 0.f ? 0.f : 1.f / l;
  store_quad((T*)p.o + row * p.ldo + c, sum);
  if (c % p.d == 0) p.lse[(int64_t)head * p.n + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---- backward: gradient of the queries -----------------------------------------------------------------------
// As the forward pass; delta = dO . O of this work-group's rows is formed on the way and kept for the keys' gradient, from O as it is stored: with O
// in float dQ would be off by 2.4e-3 instead of 2.6e-3 (4096 keys), at twice the bytes kept of O.  The fewer keys a row has the more dP and delta
// cancel (five keys: 2.3e-3 would become 4.3e-3, two 6e-3), so of a row with at most kFewKeys keys, the first ones of a long document too, delta is
// the sum of P dP, which it is by definition, in a pass of its own over the one tile or, with a window, the few that there are (8192 rows in 200
// documents, 16 heads of 64: 37 us for 31; in 60, 32 heads of 128: 117 for 112; long documents: within 1 %.  For longer rows it would be two of three
// products again).  A kernel of
// its own, which forms scores and dP a second time: sums over work-groups would be atomics, in an order that changes.  Bound as the forward pass,
// with fewer vector instructions (four to one): 748 to 818 us where that takes 597 to 654, 1.01 to 1.10 PFLOP/s.
template <typename T, int DB, int NW> __global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void attn_dq_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, DB>;
  constexpr int BM = NW * 32, BN = Tile::BN, KB = BN / 32;
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  AttnRows w = attn_rows<BM>(p, p.group * p.parts, lane, true);
  if (w.empty) return;
  const int part = w.head % p.parts;
  w.head /= p.parts;
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
  const float lse = w.dead ? -INFINITY : p.lse[row];
  const float minus = lse == -INFINITY ? -INFINITY : lse * -kLog2e;   // a row without keys has no probabilities

  const T* kbase = (const T*)p.k + (int64_t)kv * p.d;
  const T* vbase = (const T*)p.v + (int64_t)kv * p.d;
  const int last = w.first + BM < w.end ? w.first + BM - 1 : w.end - 1;
  int k_lo = keys_lo(p, w, w.first), k_hi = w.dead ? k_lo : keys_hi(p, w, last);
  const int lo = keys_lo(p, w, mine), seen = keys_hi(p, w, mine) - lo, span = alone(p, w, mine) ? 0 : seen;   // span: of dS
  const int full_lo = keys_lo(p, w, w1), full_hi = keys_hi(p, w, w0);
  const int any_lo = keys_lo(p, w, w0), any_hi = keys_hi(p, w, w1);
  const bool shaped = p.cap2 > 0.f || p.slopes;
  const float slope2 = p.slopes ? p.slopes[w.head] * kLog2e : 0.f, c2 = shaped ? 1.f : p.c2;

  const Tile32Reads<T, DB> at(lane);
  using KVLoader = Tile32Loader<T, DB, NW>;
  const KVLoader kload(lane, wave, p.ldk, p.d), vload(lane, wave, p.ldv, p.d);
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  if constexpr (sizeof(T) == 2) {
    // Rows of few keys are all of them (a window as short, a whole document) or the first ones of a document; their keys end at few_hi.
    auto few = [&](int i) { return keys_hi(p, w, i) - keys_lo(p, w, i) <= kFewKeys; };
    const int few_hi = (p.window && p.window <= kFewKeys) || k_hi - w.begin <= kFewKeys ? k_hi : w.begin + kFewKeys;
    if (!w.dead && few(w.first)) {
      float sum = 0.f;
      for (int k0 = k_lo; k0 < few_hi; k0 += BN) {
        __syncthreads();
        kload.issue(kbase, k0, few_hi - k0, p.ldk, p.d, lds, wave);
        vload.issue(vbase, k0, few_hi - k0, p.ldv, p.d, lds + Tile::BYTES, wave);
        wait_vmcnt0();
        __syncthreads();
        if (w0 >= w.end || !few(w0)) continue;
        static_for<0, KB>([&](auto block) {
          constexpr int b = block.value;
          f32x16 s{}, dp{};
#pragma unroll
          for (int i = 0; i < Tile::STEPS; ++i) {
            mma(s, at.row(smem + Tile::block(b), i), qf[i]);
            mma(dp, at.row(smem + Tile::BYTES + Tile::block(b), i), df[i]);
          }
          if (shaped) s = shape_scores<T, false>(p, s, slope2, k0 + 32 * b + 4 * h, mine, nullptr);
          const int base = k0 + 32 * b + 4 * h - lo;
          for_regs([&](int r) {
            const float of = fast_exp2(__builtin_fmaf(s[r], c2, minus)) * dp[r];
            sum += (uint32_t)(base + 8 * (r >> 2) + (r & 3)) < (uint32_t)seen ? of : 0.f;
          });
        });
      }
      sum = half_sum(sum);
      if (seen <= kFewKeys) delta = sum;
      __syncthreads();
    }
  }
  if (there && h == 0) {
    p.delta[row] = delta;
    p.minus[row] = minus;
  }
  part_of<BN>(k_lo, k_hi, part, p.parts);
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = f32x16{};
  const int tiles = (k_hi - k_lo + BN - 1) / BN;
  constexpr int PIECES = 2 * KVLoader::LOADS;
  Tile32Run<T, DB, NW> krun(kbase, k_lo, k_hi - k_lo, p.ldk, p.d), vrun(vbase, k_lo, k_hi - k_lo, p.ldv, p.d);
  uint32_t stage = lds;
  auto next = [&](int t) {   // tile t's transfers
    stage = lds + (t & 1) * 2 * Tile::BYTES;
    krun.advance(t, tiles);
    vrun.advance(t, tiles);
  };
  auto piece = [&](int i) {
    if (i < KVLoader::LOADS) kload.one(krun.rsrc, i, stage, wave);
    else vload.one(vrun.rsrc, i - KVLoader::LOADS, stage + Tile::BYTES, wave);
  };
  auto pieces = [&]() {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) piece(i);
  };
  if (tiles > 0) pieces();
  for (int t = 0; t < tiles; ++t) {
    wait_vmcnt0();
    __syncthreads();
    next(t + 1);   // (behind the last one: no rows, zeros)
    const int k0 = k_lo + t * BN;
    if (w0 >= w.end || k0 >= any_hi || k0 + BN <= any_lo) {
      pieces();
      continue;
    }
    const char* ks = smem + (t & 1) * 2 * Tile::BYTES;
    const char* vs = ks + Tile::BYTES;
    const bool masked = k0 < full_lo || k0 + BN > full_hi;
    f32x16 s[KB], dp[KB], by;   // by: the cap's slope, where there is one
#pragma unroll
    for (int b = 0; b < KB; ++b) s[b] = dp[b] = f32x16{};
    typename TransFrag<T>::type sf[2];
    auto shape = [&](auto block) {
      constexpr int b = block.value;
      if (shaped) s[b] = shape_scores<T, true>(p, s[b], slope2, k0 + 32 * b + 4 * h, mine, &by);
    };
    auto probability = [&](int b, int r) { s[b][r] = here(fast_exp2(__builtin_fmaf(s[b][r], c2, minus))); };
    auto gradient = [&](int b, int r) { s[b][r] = here(s[b][r] * (dp[b][r] - delta)); };
    auto pack = [&](auto block) {
      constexpr int b = block.value;
      if (p.cap2 > 0.f) s[b] = here(s[b] * by);   // (a branch: sixteen selections otherwise)
      if (masked) {
        const int base = k0 + 32 * b + 4 * h - lo;
        for_regs([&](int r) { if ((uint32_t)(base + 8 * (r >> 2) + (r & 3)) >= (uint32_t)span) s[b][r] = 0.f; });
      }
      sf[0] = here(step_operand<T>(s[b], 0));
      sf[1] = here(step_operand<T>(s[b], 1));
    };
    // scores and dP of block 0 (its probabilities), scores of block 1 (block 0's dS), dP of block 1 (its probabilities), dQ of block 0 (block 1's
    // dS), dQ of block 1
    constexpr int LS = Tile::STEPS, LO = 2 * DB;
    products<KB * (2 * LS + LO), sizeof(T) == 2 ? 3 : 1>(
        [&](auto i) {
          if constexpr (i.value < KB * 2 * LS) return widened(at.row((i.value / LS & 1 ? vs : ks) + Tile::block(i.value / (2 * LS)), i.value % LS));
          else return at.column(ks, (i.value - KB * 2 * LS) / DB, (i.value - KB * 2 * LS) % DB);
        },
        [&](auto i, auto x) {
          if constexpr (i.value < KB * 2 * LS) {
            if constexpr (i.value / LS & 1) mma(dp[i.value / (2 * LS)], narrowed<T>(x), df[i.value % LS]);
            else mma(s[i.value / (2 * LS)], narrowed<T>(x), qf[i.value % LS]);
          } else {
            mma(dq[(i.value - KB * 2 * LS) % DB], x, sf[(i.value - KB * 2 * LS) / DB % 2]);
          }
        },
        [&](auto i) {
          using std::integral_constant;
          constexpr int apart = KB * (2 * LS + LO) / PIECES;
          if constexpr (i.value % apart == 0 && i.value / apart < PIECES) piece(i.value / apart);
          constexpr int last_score = KB * 2 * LS, phase = i.value < last_score ? i.value / LS : KB * 2 + (i.value - last_score) / LO;
          constexpr int step = i.value < last_score ? i.value % LS : (i.value - last_score) % LO, steps = phase < KB * 2 ? LS : LO;
          if constexpr (phase < KB * 2 && (phase & 1)) {
            if constexpr (step == 0) shape(integral_constant<int, phase / 2>{});
            spread<step, steps>([&](int r) { probability(phase / 2, r); });
          }
          if constexpr (KB == 2 && (phase == 2 || phase == 4)) {
            constexpr int b = phase / 2 - 1;
            spread<step, steps>([&](int r) { gradient(b, r); });
            if constexpr (step == steps - 1) pack(integral_constant<int, b>{});
          }
          if constexpr (KB == 1 && phase == 1 && step == steps - 1) {
            for_regs([&](int r) { gradient(0, r); });
            pack(integral_constant<int, 0>{});
          }
        });
  }
  wait_vmcnt0();
  if (!there) return;
  if (p.parts > 1) store_row<float, DB>(p.part + ((int64_t)part * p.n + mine) * p.heads * p.d + (int64_t)w.head * p.d, dq, p.scale, p.d, h);
  else store_row<T, DB>((T*)p.dq + (int64_t)mine * p.ldq + (int64_t)w.head * p.d, dq, p.scale, p.d, h);
}

// ---- backward: gradients of the keys and values --------------------------------------------------------------
// A work-group has KW x 32 keys of one key head and goes over the queries of the heads that share it, so that the sum
// over them is taken in its accumulators.  bfloat16: twice KW waves, two for the same keys, which take the two halves of a tile of queries and add
// their sums up at the end; the keys' rows stay in LDS.  (Two waves a SIMD need 256 registers each, of which the sums take 128: with the
// keys' rows in registers too there is one, and nothing runs while it waits: 4 x 4096 rows, 32 heads of 128 on 8, both passes 2.82 ms, so 3.54.)
// float: the keys' rows in registers.  Where there are few or short rows two waves' keys are a work-group (KW).  The same rows: 1098 to 1193 us,
// 0.92 to 1.00 PFLOP/s, three vector instructions to a matrix one.
template <typename T, int DB, int KW> struct DkvLayout {
  using Tile = Tile32<T, DB>;
  static constexpr int HALVES = sizeof(T) == 2 ? 2 : 1, NW = KW * HALVES, BM = 32 * KW, BQ = Tile::BN;
  static constexpr int KEYS = HALVES == 2 ? 2 * (BM / Tile::BN) * Tile::BYTES : 0;   // bytes of K and V
  static constexpr int STAGE = 2 * Tile::BYTES + 512;   // queries, their outputs' gradients, log-sum-exps and deltas
  static constexpr int SUMS = HALVES == 2 ? KW * DB * 16 * 64 * 4 : 0;   // one half's sums of one tensor
  static constexpr int BYTES = KEYS + 2 * STAGE > SUMS ? KEYS + 2 * STAGE : SUMS;
};

template <typename T, int DB, int KW>
__global__ __launch_bounds__((DkvLayout<T, DB, KW>::NW * 64), (DkvLayout<T, DB, KW>::HALVES)) void attn_dkv_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, DB>;
  using Layout = DkvLayout<T, DB, KW>;
  constexpr int NW = Layout::NW, BM = Layout::BM, BQ = Layout::BQ, STAGE = Layout::STAGE;
  constexpr bool IN_LDS = Layout::HALVES == 2;
  constexpr int QB = BQ / 32 / Layout::HALVES;   // blocks of queries of a wave
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), key_wave = wave % KW, half = wave / KW;
  const AttnRows w = attn_rows<BM>(p, p.parts, lane, false);
  if (w.empty) return;
  const int kv = w.head / p.parts, part = w.head - kv * p.parts;
  const int w0 = w.first + key_wave * 32;
  const int w1 = w0 + 31 < w.end ? w0 + 31 : w.end - 1;
  const int mine = w0 + c < w.end ? w0 + c : w.end - 1;
  const bool there = w0 + c < w.end;

  const T* kbase = (const T*)p.k + (int64_t)kv * p.d;
  const T* vbase = (const T*)p.v + (int64_t)kv * p.d;
  const int last = w.first + BM < w.end ? w.first + BM - 1 : w.end - 1;
  const int q_lo = queries_lo(p, w, w.first), q_hi = w.dead ? q_lo : queries_hi(p, w, last);
  const int lo = queries_lo(p, w, mine), span = queries_hi(p, w, mine) - lo, skip = alone(p, w, mine);   // (the first of them has no dS)
  const int full_lo = queries_lo(p, w, w1), full_hi = queries_hi(p, w, w0);
  const int any_lo = queries_lo(p, w, w0), any_hi = queries_hi(p, w, w1);
  const bool shaped = p.cap2 > 0.f || p.slopes;
  const float c2 = shaped ? 1.f : p.c2;

  const Tile32Reads<T, DB> at(lane);
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
  // this part's tiles: of query head `head` from `tile` on, then those of the heads behind it
  const int per_head = (q_hi - q_lo + BQ - 1) / BQ, all = per_head * p.group;
  const int from = (int)((int64_t)all * part / p.parts), tiles = (int)((int64_t)all * (part + 1) / p.parts) - from;
  int head = kv * p.group + (per_head ? from / per_head : 0), tile = per_head ? from % per_head : 0, next_tile = 0;
  using QLoader = Tile32Loader<T, DB, NW>;
  const QLoader qload(lane, wave, p.ldq, p.d), dload(lane, wave, p.ldo, p.d);
  constexpr int PIECES = 2 * QLoader::LOADS + 1;
  Tile32Run<T, DB, NW> qrun((const T*)p.q + (int64_t)head * p.d, q_lo, q_hi - q_lo, p.ldq, p.d), drun((const T*)p.dout + (int64_t)head * p.d, q_lo, q_hi - q_lo, p.ldo, p.d);
  qrun.skip(tile, per_head);
  drun.skip(tile, per_head);
  u32x4 srows = make_rsrc((wave ? p.delta : p.minus) + (int64_t)head * p.n + q_lo, (int64_t)(q_hi - q_lo) * 4);
  uint32_t stage = lds + Layout::KEYS, stats_at = (tile * BQ + lane) * 4;
  // the transfers of the tile of queries behind the one that they are at; the last head's last tile is followed by tiles without rows
  auto next = [&](int tile, int t) {
    stage = lds + Layout::KEYS + (t & 1) * STAGE;
    if (tile == 0 && t < tiles) {
      qrun.back(per_head, (int64_t)p.d * sizeof(T));
      drun.back(per_head, (int64_t)p.d * sizeof(T));
      const uint64_t at = ((uint64_t)srows[1] << 32 | srows[0]) + (uint64_t)p.n * 4;
      srows[0] = (uint32_t)at;
      srows[1] = (uint32_t)(at >> 32);
      stats_at = lane * 4;
    } else {
      qrun.advance(t < tiles ? tile : per_head, per_head);
      drun.advance(t < tiles ? tile : per_head, per_head);
      stats_at += BQ * 4;
    }
  };
  auto piece = [&](int i) {
    if (i < QLoader::LOADS) qload.one(qrun.rsrc, i, stage, wave);
    else if (i < 2 * QLoader::LOADS) dload.one(drun.rsrc, i - QLoader::LOADS, stage + Tile::BYTES, wave);
    else if (wave < 2) buffer_to_lds_b32(srows, stats_at, stage + 2 * Tile::BYTES + wave * 256);
  };
  auto pieces = [&]() {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) piece(i);
  };
  if (tiles > 0) pieces();
  for (int t = 0; t < tiles; ++t) {
    wait_vmcnt0();
    __syncthreads();
    if (t > 0) {
      head += next_tile == 0;
      tile = next_tile;
    }
    next_tile = tile + 1 == per_head ? 0 : tile + 1;
    next(next_tile, t + 1);
    const int q0 = q_lo + tile * BQ + half * QB * 32;   // this wave's queries
    if (w0 >= w.end || q0 >= any_hi || q0 + QB * 32 <= any_lo) {
      pieces();
      continue;
    }
    const char* qs = smem + Layout::KEYS + (t & 1) * STAGE + Tile::block(half * QB);
    const char* ds = qs + Tile::BYTES;
    const float* stats = (const float*)(smem + Layout::KEYS + (t & 1) * STAGE + 2 * Tile::BYTES) + half * QB * 32;
    const float slope2 = p.slopes ? p.slopes[head] * kLog2e : 0.f;
    const bool masked = q0 < full_lo || q0 + QB * 32 > full_hi;
    static_for<0, QB>([&](auto block) {
      constexpr int b = block.value;
      f32x16 s{}, dp{}, by;   // by: the cap's slope, where there is one
      f32x4 minus[4], delta[4];
      using Frag = typename TransFrag<T>::type;
      Frag pf[2], sf[2];
      struct Pair { Frag x, y; };
      struct Single { Frag x; };
      using Operands = std::conditional_t<IN_LDS, Pair, Single>;
      // scores, dP (the probabilities), dV (dS), dK
      constexpr int LS = Tile::STEPS, LO = 2 * DB;
      products<2 * LS + 2 * LO, sizeof(T) == 2 ? 2 : 1>(
          [&](auto i) {
            Operands o;
            if constexpr (i.value < 2 * LS) {
              o.x = widened(at.row((i.value < LS ? qs : ds) + Tile::block(b), i.value % LS));
              if constexpr (IN_LDS) o.y = widened(at.row(i.value < LS ? ks : vs, i.value % LS));
            } else {
              o.x = at.column(i.value < 2 * LS + LO ? ds : qs, 2 * b + (i.value - 2 * LS) % LO / DB, (i.value - 2 * LS) % DB);
            }
            return o;
          },
          [&](auto i, const Operands& o) {
            if constexpr (i.value < 2 * LS) {
              f32x16& to = i.value < LS ? s : dp;
              if constexpr (IN_LDS) mma(to, narrowed<T>(o.x), narrowed<T>(o.y));
              else mma(to, narrowed<T>(o.x), i.value < LS ? kf[i.value % LS] : vf[i.value % LS]);
            } else if constexpr (i.value < 2 * LS + LO) {
              mma(dv[(i.value - 2 * LS) % DB], o.x, pf[(i.value - 2 * LS) / DB]);
            } else {
              mma(dk[(i.value - 2 * LS) % DB], o.x, sf[(i.value - 2 * LS - LO) / DB]);
            }
          },
          [&](auto i) {
            constexpr int apart = (2 * LS + 2 * LO) / PIECES;
            if constexpr (b == 0 && i.value % apart == 0 && i.value / apart < PIECES) piece(i.value / apart);
            constexpr int phase = i.value < 2 * LS ? i.value / LS : 2 + (i.value - 2 * LS) / LO;
            constexpr int step = i.value < 2 * LS ? i.value % LS : (i.value - 2 * LS) % LO, steps = phase < 2 ? LS : LO;
            if constexpr (phase == (IN_LDS ? 0 : 1) && step == 0) {
#pragma unroll
              for (int g = 0; g < 4; ++g) minus[g] = *(const f32x4*)(stats + 32 * b + 8 * g + 4 * h);
            }
            if constexpr (phase == 1) {
              if constexpr (step == 0) {
                if (shaped) s = shape_scores<T, true>(p, s, slope2, q0 + 32 * b + 4 * h, mine, &by);
              }
              spread<step, steps>([&](int r) { s[r] = here(fast_exp2(__builtin_fmaf(s[r], c2, minus[r >> 2][r & 3]))); });
              if constexpr (step == steps - 1) {
                if (masked) {
                  const int base = q0 + 32 * b + 4 * h - lo;
                  for_regs([&](int r) { if ((uint32_t)(base + 8 * (r >> 2) + (r & 3)) >= (uint32_t)span) s[r] = 0.f; });
                }
                pf[0] = here(step_operand<T>(s, 0));
                pf[1] = here(step_operand<T>(s, 1));
                if (p.cap2 > 0.f) s = here(s * by);   // (a branch: sixteen selections otherwise)
#pragma unroll
                for (int g = 0; g < 4; ++g) delta[g] = *(const f32x4*)(stats + 64 + 32 * b + 8 * g + 4 * h);
              }
            }
            if constexpr (phase == 2) {
              spread<step, steps>([&](int r) { dp[r] = here(s[r] * (dp[r] - delta[r >> 2][r & 3])); });
              if constexpr (step == steps - 1) {
                if (masked) {   // (a probability of zero does not make what is not finite zero)
                  const int base = q0 + 32 * b + 4 * h - lo - skip;
                  for_regs([&](int r) { if ((uint32_t)(base + 8 * (r >> 2) + (r & 3)) >= (uint32_t)(span - skip)) dp[r] = 0.f; });
                }
                sf[0] = here(step_operand<T>(dp, 0));
                sf[1] = here(step_operand<T>(dp, 1));
              }
            }
          });
    });
  }
  wait_vmcnt0();
  if constexpr (IN_LDS) {   // the second half's sums to the first
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
  if (p.parts > 1) {
    float* to = p.part + ((int64_t)part * 2 * p.n + mine) * p.kv_heads * p.d + (int64_t)kv * p.d;
    store_row<float, DB>(to, dk, p.scale, p.d, h);
    store_row<float, DB>(to + (int64_t)p.n * p.kv_heads * p.d, dv, 1.f, p.d, h);
    return;
  }
  store_row<T, DB>((T*)p.dk + (int64_t)mine * p.ldk + (int64_t)kv * p.d, dk, p.scale, p.d, h);
  store_row<T, DB>((T*)p.dv + (int64_t)mine * p.ldv + (int64_t)kv * p.d, dv, 1.f, p.d, h);
}

// One or two matrices [n, width] as sums of their parts [parts][matrices][n][width], four channels a lane: bound by the parts' bytes (dK and dV of
// 6001 rows, 4 key heads of 80, three parts: 46 MB in 9 us).
template <typename T>
__global__ __launch_bounds__(256) void attn_parts_kernel(const float* part, int parts, int64_t n, int width, T* first, int64_t ld_first, T* second, int64_t ld_second) {
  const int quads = width / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (second ? 2 : 1) * n * quads;
  if (i >= all) return;
  f32x4 sum = *(const f32x4*)(part + i * 4);
  for (int k = 1; k < parts; ++k) sum += *(const f32x4*)(part + (k * all + i) * 4);
  const int64_t row = i / quads;
  const int c = (int)(i - row * quads) * 4;
  store_quad(row < n ? first + row * ld_first + c : second + (row - n) * ld_second + c, sum);
}

}  // namespace acc
