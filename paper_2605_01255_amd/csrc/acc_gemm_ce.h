// What the products with the vocabulary's matrix do with their output tiles (acc_ce.h has the rest of the cross entropy): the
// logits stay in the accumulators and become sums of exponentials (forward) or the logits' gradient (backward).
// A wave's tile is TM x TN blocks of 16 x 16: lane l16 + 16 g4 holds row l16 of each block and its columns 4 g4 .. + 3.
#pragma once
#include "acc_gemm.h"

namespace acc {

enum class Epilogue { kStore, kExpSums, kGradient, kParts };

constexpr float kLog2e = 1.44269504088896341f;
template <Epilogue EPI> __device__ __forceinline__ void take_live_rows(FastGemmParams& p, int bm) {
  if (!p.live) return;   // all of them
  int rows = *p.live;
  if (EPI == Epilogue::kGradient && rows < p.least_rows) rows = p.least_rows;
  p.M = rows;
  p.tiles_m = (rows + bm - 1) / bm;
}
__device__ __forceinline__ void take_live_tokens(FastGemmParams& p) {
  if (!p.live) return;
  const int rows = *p.live;
  p.K = rows < p.least_rows ? p.least_rows : rows;
}

__device__ __forceinline__ int64_t ce_clamped(const FastGemmParams& p, int64_t row) { return row < p.ce.rows ? row : p.ce.rows - 1; }
__device__ __forceinline__ int ce_target(const FastGemmParams& p, int64_t row) {   // -1: none
  const int64_t t = p.ce.targets[ce_clamped(p, row)];
  return t < 0 || t > (1 << 30) ? -1 : (int)t;
}
// Targets of this lane's row of each block row from m0 on.
template <int TM> __device__ __forceinline__ void ce_targets(const FastGemmParams& p, int (&target)[TM], int64_t m0, int l16) {
  static_for<0, TM>([&](auto row) { target[decltype(row)::value] = ce_target(p, m0 + decltype(row)::value * 16 + l16); });
}

// The value is one that the compiler has in an accumulator register here, and copies it from here on: without it the copies of all 256
// are made in front of ce_sums' branches, and others are pushed out into scratch memory.
__device__ __forceinline__ void in_accumulators(f32x4& v) { asm volatile("" : "+a"(v)); }

// The wave's sums: per row the maximum over the strip of TN * 16 columns and the sum of exponentials above it, and the logit of a
// target in it.  Exponentials as powers of two: the product with log2 e and the difference are one operation.
template <int TM, int TN>
__device__ __forceinline__ void ce_sums(const FastGemmParams& p, f32x4 (&acc)[TM][TN], const int (&target)[TM], int64_t m0, int64_t n0, int l16, int g4) {
  constexpr int STRIP = TN * 16;
  if (n0 >= p.N) return;
  const int64_t strip = (p.ce.v0 + n0) / STRIP;   // pieces are whole numbers of strips
  const int left = (int)(p.N - n0 < STRIP ? p.N - n0 : STRIP) - 4 * g4;   // columns of this lane's that exist have j * 16 + e below this
  auto block_row = [&](auto row, auto edge) {
    constexpr int i = decltype(row)::value;
    constexpr bool EDGE = decltype(edge)::value;
    __builtin_amdgcn_sched_barrier(0);
    const int64_t gm = m0 + i * 16 + l16;
    const bool exists = gm < p.M;
    f32x4 x[TN];
    float m = -INFINITY;
    static_for<0, TN>([&](auto col) {
      constexpr int j = decltype(col)::value;
      in_accumulators(acc[i][j]);
      x[j] = acc[i][j];
      if constexpr (EDGE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = j * 16 + e < left ? x[j][e] : -INFINITY;
      }
      m = fmaxf(m, fmaxf(fmaxf(x[j][0], x[j][1]), fmaxf(x[j][2], x[j][3])));
    });
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    if (isinf(m)) m = 0.f;   // exponentials of what is infinite are 0 or infinite, never NaN
    const float m2 = m * kLog2e;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    // few waves hold a target's column
    const int64_t rel = exists ? target[i] - (p.ce.v0 + n0) : -1;
    if (__any(rel >= 0 && rel < STRIP)) {
      const int at = rel >= 0 && rel < STRIP ? (int)rel - 4 * g4 : -1;
      static_for<0, TN>([&](auto col) {
        constexpr int j = decltype(col)::value;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at == j * 16 + e) p.ce.target_logit[gm] = x[j][e];
      });
    }
    static_for<0, TN>([&](auto col) {
      constexpr int j = decltype(col)::value;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[j][e], kLog2e, -m2));
    });
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (exists && g4 == 0) p.ce.part[strip * p.ce.rows + gm] = f32x2{m, sum};
  };
  if (n0 + STRIP > p.N) static_for<0, TM>([&](auto row) { block_row(row, std::true_type{}); });
  else static_for<0, TM>([&](auto row) { block_row(row, std::false_type{}); });
  __builtin_amdgcn_sched_barrier(0);
}

// Of one row: log-sum-exp times log2 e, the incoming gradient g, the target's column counted from this lane's first one, and the
// target's own gradient g (exp(z - lse) - 1), where 1 is taken from the probability without cancellation.
// A row whose log-sum-exp is not finite gets NaN, as g.  That lets the exponent be cut off far above any probability's, which keeps
// the columns behind the vocabulary's end, where the logits are 0, finite: the product with W takes rows of zeros for them.
struct CeRow {
  float lse2, g, own;
  int at;
};
__device__ __forceinline__ CeRow ce_row(const FastGemmParams& p, int64_t row, int64_t n0, int g4) {
  row = ce_clamped(p, row);
  const float lse = p.ce.lse[row], g = isfinite(lse) ? p.ce.g[row] : NAN;
  const int target = ce_target(p, row);
  return CeRow{lse * kLog2e, g, g * expm1f(p.ce.target_logit[row] - lse), target < 0 ? -1 : target - (int)(p.ce.v0 + n0) - 4 * g4};
}
// The compiler has to have a requested value here.
__device__ __forceinline__ void landed(CeRow& r) { asm volatile("" : "+v"(r.lse2), "+v"(r.g), "+v"(r.own), "+v"(r.at)); }
__device__ __forceinline__ void landed(int& v) { asm volatile("" : "+v"(v)); }
// x: the logits of this lane's columns 16 j .. 16 j + 3.
__device__ __forceinline__ f32x4 ce_gradient(const CeRow& r, f32x4 x, int j) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float p = __builtin_amdgcn_exp2f(fminf(__builtin_fmaf(x[e], kLog2e, -r.lse2), 60.f));
    x[e] = r.at == j * 16 + e ? r.own : r.g * p;
  }
  return x;
}

}  // namespace acc
