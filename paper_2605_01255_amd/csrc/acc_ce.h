// The vocabulary's product and its softmax cross entropy without the logits:  z = X . W^T in pieces of the vocabulary,
//   lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_i,target;   dz_iv = g_i (exp(z_iv - lse_i) - [v = target_i]),
//   dX = dz . W,  dW = dz^T . X.
//
// Tokens without a loss (negative targets) take no part: the others are gathered into a dense matrix first, so that products cost what
// the tokens with a loss cost, and infinities or NaN in a padded token's row reach no sum (0 times NaN is NaN).  Nor do, in the
// backward pass, tokens whose target lies beyond the vocabulary: their loss is NaN and they have no gradient.
#pragma once
#include "acc_common.h"
#include "acc_gemm_ce.h"

namespace acc {

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// What a call knows of its tokens.  `order` lists those that take part (with a loss; in a backward call with a gradient) in their order,
// then the others; null: all tokens as they come.
struct CeTokens {
  const int64_t* targets;   // [n]
  int n;
  int64_t last;             // targets beyond take no part: none in a forward call, those beyond the vocabulary in a backward one
  int* order;               // [n]
  int* count;               // tokens that take part
  __device__ __forceinline__ bool takes_part(int64_t target) const { return target >= 0 && target <= last; }
  __device__ __forceinline__ int token(int64_t r) const { return order ? order[r] : (int)r; }
  __device__ __forceinline__ bool lives(int64_t r) const { return order ? r < *count : r < n && takes_part(targets[r]); }
};

// One work-group of 1024 threads, eight tokens of a thread at a time; the others fill the list from its end.
// largest (with dloss, backward): the largest magnitude among the incoming gradients of the tokens that take part, 1 if there is none.  dz is
// formed in units of it: the tokens' gradients are one value as a rule, which as part of dz would be rounded to bfloat16 the same way
// in every row (an error of up to 2^-8 in the gradients that does not average out), and in its own units is 1.
__global__ __launch_bounds__(1024) void ce_select_kernel(CeTokens t, const float* __restrict__ dloss, float* __restrict__ largest) {
  constexpr int PER = 8;
  __shared__ int wave_kept[2][16];
  __shared__ float wave_largest[16];
  float top = 0.f;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int kept = 0, turn = 0;   // kept: so far
  for (int first = 0; first < t.n; first += 1024 * PER, turn ^= 1) {
    const int i0 = first + tid * PER, last = t.n - 1;
    int64_t target[PER];
    float g[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) target[k] = t.targets[i0 + k < last ? i0 + k : last];
    if (dloss) {
#pragma unroll
      for (int k = 0; k < PER; ++k) g[k] = dloss[i0 + k < last ? i0 + k : last];
    }
    bool keep[PER];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      keep[k] = t.takes_part(target[k]);
      mine += keep[k] && i0 + k < t.n ? 1 : 0;
    }
    int before = mine;   // inclusive scan over the wave
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(before, d);
      before += lane >= d ? o : 0;
    }
    if (lane == 63) wave_kept[turn][wave] = before;
    __syncthreads();
    int total = 0, waves_before = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      waves_before += w < wave ? wave_kept[turn][w] : 0;
      total += wave_kept[turn][w];
    }
    int at = kept + waves_before + before - mine;   // tokens that take part before this thread's
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (i0 + k >= t.n) break;
      if (dloss && keep[k] && isfinite(g[k])) top = fmaxf(top, fabsf(g[k]));
      if (keep[k]) t.order[at++] = i0 + k;
      else t.order[t.n - 1 - (i0 + k - at)] = i0 + k;
    }
    kept += total;
  }
  if (tid == 0) *t.count = kept;
  if (!dloss) return;
  top = wave_max(top);
  if (lane == 0) wave_largest[wave] = top;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 16; ++w) top = fmaxf(top, wave_largest[w]);
    *largest = top > 0.f ? top : 1.f;
  }
}

// What the products and the loss read of a token, in the order of the list; rows behind the last one are zero, up to 256 of them
// for the products' least rows.  targets: -1 where there is none in the vocabulary.  per_row, in a backward call: lse, the target's
// logit and the incoming gradient (over *unit), `rows` of each.
// SELECT: the selection as well, for up to kCeSelectHere tokens: every work-group finds its row's token by itself, from all targets, which
// saves a launch that takes 4.5 us with the pause behind it.
constexpr int kCeSelectHere = 1024;
template <typename T, bool SELECT>
__global__ __launch_bounds__(256) void ce_gather_kernel(CeTokens t, const T* __restrict__ X, int64_t ldx, int d, int64_t rows, T* __restrict__ Xc, int64_t V,
                                                        const float* __restrict__ stats, const float* __restrict__ dloss, float* __restrict__ unit,
                                                        int64_t stats_stride, int64_t* __restrict__ targets, float* __restrict__ per_row) {
  constexpr int VEC = 16 / sizeof(T);
  typedef T vecT __attribute__((ext_vector_type(VEC)));
  const int64_t r = blockIdx.x;
  int count, i = 0;
  float g_unit = 1.f;
  if constexpr (SELECT) {
    constexpr int PER = kCeSelectHere / 256;
    __shared__ int wave_kept[4], token;
    __shared__ float wave_largest[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i0 = tid * PER;
    bool keep[PER];
    int mine = 0;
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int at = i0 + k < t.n ? i0 + k : t.n - 1;
      keep[k] = t.takes_part(t.targets[at]) && i0 + k < t.n;
      mine += keep[k] ? 1 : 0;
      if (unit) {
        const float g = dloss[at];
        if (keep[k] && isfinite(g)) top = fmaxf(top, fabsf(g));
      }
    }
    int before = mine;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_up(before, s);
      before += lane >= s ? o : 0;
    }
    top = wave_max(top);
    if (lane == 63) {
      wave_kept[wave] = before;
      wave_largest[wave] = top;
    }
    __syncthreads();
    count = wave_kept[0] + wave_kept[1] + wave_kept[2] + wave_kept[3];
    if (unit) {
      top = fmaxf(fmaxf(wave_largest[0], wave_largest[1]), fmaxf(wave_largest[2], wave_largest[3]));
      g_unit = top > 0.f ? top : 1.f;
    }
    int at = before - mine;   // tokens that take part before this thread's
#pragma unroll
    for (int w = 0; w < 3; ++w) at += w < wave ? wave_kept[w] : 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {   // the others behind those that take part
      if (i0 + k < t.n && (keep[k] ? at : count + i0 + k - at) == r) token = i0 + k;
      at += keep[k] ? 1 : 0;
    }
    __syncthreads();
    if (r < t.n) {
      i = token;
      if (tid == 0) t.order[r] = i;
    }
    if (r == 0 && tid == 0) {
      *t.count = count;
      if (unit) *unit = g_unit;
    }
  } else {
    count = *t.count;
    if (r < count) i = t.order[r];
    if (unit) g_unit = *unit;
  }
  const bool lives = r < count;
  if (threadIdx.x == 0) {
    const int64_t target = lives ? t.targets[i] : -1;
    targets[r] = target < V ? target : -1;
    if (stats) {
      per_row[r] = lives ? stats[i] : 0.f;
      per_row[rows + r] = lives ? stats[stats_stride + i] : 0.f;
      per_row[2 * rows + r] = lives ? dloss[i] / g_unit : 0.f;
    }
  }
  if (sizeof(T) == 2 && !lives && r >= 256) return;   // the float32 products read every row
  for (int c = (int)threadIdx.x * VEC; c < d; c += 256 * VEC) {
    vecT v = {};
    if (lives) v = *(const vecT*)(X + (int64_t)i * ldx + c);
    *(vecT*)(Xc + r * d + c) = v;
  }
}

// A sum of exponentials as (m, s) = s exp(m), m finite; s = 0: nothing.
struct ExpSum {
  float m, s;
};
__device__ __forceinline__ ExpSum operator+(ExpSum a, ExpSum b) {
  if (a.s == 0.f) return b;
  if (b.s == 0.f) return a;
  const float m = fmaxf(a.m, b.m);
  return ExpSum{m, a.s * expf(a.m - m) + b.s * expf(b.m - m)};
}

// (m, s) over eight values at a time, each requested before the first is used.
constexpr int kCeAtOnce = 8;
__device__ __forceinline__ ExpSum with_values(ExpSum sum, const float (&v)[kCeAtOnce]) {   // -infinity: no value
  float m = sum.s == 0.f ? -INFINITY : sum.m;   // an empty sum's maximum does not count; NaN is not 0
#pragma unroll
  for (int u = 0; u < kCeAtOnce; ++u) m = fmaxf(m, v[u]);
  if (isinf(m)) m = 0.f;                        // exponentials of what is infinite are 0 or infinite, never NaN
  float s = sum.s == 0.f ? 0.f : sum.s * __builtin_amdgcn_exp2f((sum.m - m) * kLog2e);
#pragma unroll
  for (int u = 0; u < kCeAtOnce; ++u) s += __builtin_amdgcn_exp2f((v[u] - m) * kLog2e);
  return ExpSum{m, s};
}

// Losses and statistics, one work-group per token, from the logits of one piece [rows, vp] (rows 16-byte aligned); running sums between
// the pieces.
__global__ __launch_bounds__(256) void ce_piece_stats_kernel(CeTokens t, const float* __restrict__ Z, int64_t ldz, int64_t v0, int vp, bool first,
                                                             bool last, int64_t V, float* __restrict__ run_m, float* __restrict__ run_z,
                                                             float* __restrict__ run_s, float* __restrict__ loss, float* __restrict__ stats,
                                                             int64_t stats_stride) {
  __shared__ ExpSum sums[256];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const int i = t.order[r];
  if (r >= *t.count) {
    if (last && tid == 0) loss[i] = stats[i] = stats[stats_stride + i] = 0.f;
    return;
  }
  const float* z = Z + r * ldz;
  ExpSum sum{0.f, 0.f};
  for (int c = 8 * tid; c < vp; c += 2048) {   // ldz is a multiple of eight
    const f32x4 lo = *(const f32x4*)(z + c), hi = *(const f32x4*)(z + c + 4);
    float v[8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v[u] = c + u < vp ? lo[u] : -INFINITY;
      v[4 + u] = c + 4 + u < vp ? hi[u] : -INFINITY;
    }
    sum = with_values(sum, v);
  }
  sums[tid] = sum;
  __syncthreads();
  for (int half = 128; half; half /= 2) {
    if (tid < half) sums[tid] = sums[tid] + sums[tid + half];
    __syncthreads();
  }
  if (tid) return;
  sum = sums[0];
  if (!first) sum = sum + ExpSum{run_m[r], run_s[r]};
  const int64_t target = t.targets[i];
  if (target >= v0 && target < v0 + vp) run_z[r] = z[target - v0];
  if (last) {
    const float lse = sum.m + logf(sum.s), zt = target < V ? run_z[r] : NAN;
    loss[i] = lse - zt;
    stats[i] = lse;
    stats[stats_stride + i] = zt;
  } else {
    run_m[r] = sum.m;
    run_s[r] = sum.s;
  }
}

// dz of one piece from its logits, in place, one work-group per row; rows without a token and columns from vp to ldz are zero.  A row
// whose log-sum-exp is not finite gets NaN: its exponentials would be 0 wherever the logits are finite.
__global__ __launch_bounds__(256) void ce_piece_grad_kernel(CeTokens t, float* __restrict__ Z, int64_t ldz, int64_t v0, int vp, int64_t rows,
                                                            const int64_t* __restrict__ targets, const float* __restrict__ per_row) {
  const int64_t r = blockIdx.x, target = targets[r];   // -1 where there is no token or no gradient
  const float lse = per_row[r], zt = per_row[rows + r], g = isfinite(lse) ? per_row[2 * rows + r] : NAN;
  const float own = g * expm1f(zt - lse);
  for (int64_t c = 4 * threadIdx.x; c < ldz; c += 1024) {
    f32x4 x = *(const f32x4*)(Z + r * ldz + c);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float dz = v0 + c + u == target ? own : g * expf(x[u] - lse);
      x[u] = target >= 0 && c + u < vp ? dz : 0.f;
    }
    *(f32x4*)(Z + r * ldz + c) = x;
  }
}

// Losses and statistics from the strips' sums.  A work-group takes `across` rows (a power of two); the threads of a row share its
// strips, eight requested at a time.
__global__ __launch_bounds__(256) void ce_finish_kernel(CeTokens t, const f32x2* __restrict__ part, int strips, int64_t rows, int across, int64_t V,
                                                        const float* __restrict__ target_logit, float* __restrict__ loss,
                                                        float* __restrict__ stats, int64_t stats_stride) {
  __shared__ ExpSum sums[256];
  const int tid = threadIdx.x, mine = tid & (across - 1), first = tid / across, step = 256 / across;
  const int r = (int)blockIdx.x * across + mine;
  const bool exists = r < t.n, lives = exists && t.lives(r);
  ExpSum sum{0.f, 0.f};
  if (lives) {
    constexpr int AT_ONCE = 8;
    for (int k = first; k < strips; k += AT_ONCE * step) {
      f32x2 v[AT_ONCE];
      static_for<0, AT_ONCE>([&](auto u) {
        constexpr int U = decltype(u)::value;
        v[U] = f32x2{0.f, 0.f};
        if (k + U * step < strips) v[U] = part[(int64_t)(k + U * step) * rows + r];
      });
      float m = sum.s == 0.f ? -INFINITY : sum.m;   // an empty sum's maximum does not count; NaN is not 0
      static_for<0, AT_ONCE>([&](auto u) { m = v[decltype(u)::value][1] == 0.f ? m : fmaxf(m, v[decltype(u)::value][0]); });
      if (isinf(m)) continue;                       // all of them are empty
      float s = sum.s == 0.f ? 0.f : sum.s * __builtin_amdgcn_exp2f((sum.m - m) * kLog2e);
      static_for<0, AT_ONCE>([&](auto u) {
        const f32x2 x = v[decltype(u)::value];
        s += x[1] == 0.f ? 0.f : x[1] * __builtin_amdgcn_exp2f((x[0] - m) * kLog2e);
      });
      sum = ExpSum{m, s};
    }
  }
  sums[tid] = sum;
  __syncthreads();
  for (int half = step / 2; half; half /= 2) {
    if (first < half) sums[tid] = sums[tid] + sums[tid + half * across];
    __syncthreads();
  }
  if (first || !exists) return;
  const int i = t.token(r);
  float lse = 0.f, zt = 0.f;
  if (lives) {
    lse = sums[tid].m + logf(sums[tid].s);
    zt = t.targets[i] < V ? target_logit[r] : NAN;
  }
  loss[i] = lse - zt;
  stats[i] = lse;
  stats[stats_stride + i] = zt;
}

// A dense matrix [rows, d] as the sum of the parts of a product, `stride` apart, and of what there was before (null: nothing).
struct CeParts {
  const float* parts;
  int splits;
  int64_t stride;
  const float* before;
  __device__ __forceinline__ f32x4 at(int64_t e) const {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (before) v = *(const f32x4*)(before + e);
#pragma unroll 4
    for (int k = 0; k < splits; ++k) v += *(const f32x4*)(parts + k * stride + e);
    return v;
  }
};

// The sum between two pieces, for the rows with a token.  One work-group per row.
__global__ __launch_bounds__(256) void ce_add_kernel(CeTokens t, CeParts sum, int d, float* dXf) {
  const int64_t r = blockIdx.x;
  if (!t.lives(r)) return;
  for (int c = (int)threadIdx.x * 4; c < d; c += 1024) *(f32x4*)(dXf + r * d + c) = sum.at(r * d + c);
}

// dX [n, ldx] from the dense rows times *unit; tokens without a loss get zeros.  One work-group per row of the list.
template <typename T>
__global__ __launch_bounds__(256) void ce_scatter_kernel(CeTokens t, CeParts sum, const float* __restrict__ unit, int d, T* __restrict__ dX, int64_t ldx) {
  const int64_t r = blockIdx.x;
  const bool lives = t.lives(r);
  const int i = t.token(r);
  const float scale = unit ? *unit : 1.f;
  for (int c = (int)threadIdx.x * 4; c < d; c += 1024) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (lives) v = sum.at(r * d + c) * scale;
    T* dst = dX + (int64_t)i * ldx + c;
    if constexpr (sizeof(T) == 2) {
      bf16x4 o;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = (bf16)v[k];
      *(bf16x4*)dst = o;
    } else {
      *(f32x4*)dst = v;
    }
  }
}

}  // namespace acc
