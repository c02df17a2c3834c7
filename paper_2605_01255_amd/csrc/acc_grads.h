// The norm over all gradients of a model, and their scaling.
//
// Dense tensors: one pass, squares summed in double (a float square overflows above 1.8e19 and vanishes below 1e-23; at the rate of HBM the
// wider sum costs nothing).  Factored gradients, dW = L G^T with L [rows, r] and G [rows', r]: |dW|^2 = sum (L^T L) o (G^T G), so two sums over
// rows of r x r instead of the product; both are symmetric, and tiles below the diagonal are counted twice and not formed.  The tables of tensors
// travel in the kernels' arguments: nothing to keep, and a captured graph has its own.  Sums in a fixed order.
#pragma once
#include "acc_tile32.h"

namespace acc {

constexpr int kGradTensors = 64;             // of a launch
constexpr int64_t kGradChunk = 1 << 16;      // elements of a work-group
constexpr int kGradFactors = 32;             // of a launch
constexpr int kGramTile = 128, kGramRows = 2048;   // columns of a tile, rows that one work-group sums

struct GradList {
  const void* src[kGradTensors];
  void* dst[kGradTensors];
  int64_t count[kGradTensors];
  uint32_t first[kGradTensors + 1];   // work-group
  uint8_t src_b16[kGradTensors], dst_b16[kGradTensors];
  int tensors;
};

// This work-group's tensor.
__device__ __forceinline__ int grad_tensor(const GradList& g, uint32_t group) {
  const int lane = threadIdx.x & 63;
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < g.tensors && g.first[lane] <= group)) - 1);
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int s = 32; s; s >>= 1) x += __shfl_xor(x, s);
  return x;
}
// Sum over a work-group of 256 in lane 0.
__device__ __forceinline__ double group_sum(double x) {
  __shared__ double waves[4];
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  return waves[0] + waves[1] + waves[2] + waves[3];
}

template <typename T> __device__ __forceinline__ double grad_squares(const T* x, int count) {
  constexpr int E = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(E)));
  double sum[2] = {0.0, 0.0};
  const int whole = ((uintptr_t)x & 15) == 0 ? count / E : 0;   // (a tensor that starts inside 16 bytes goes element by element)
  int c = threadIdx.x;
  for (; c + 3 * 256 < whole; c += 1024) {
    vec v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = ((const vec*)x)[c + k * 256];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const double d = (double)to_f32(v[k][e]);
        sum[e & 1] = __builtin_fma(d, d, sum[e & 1]);
      }
  }
  for (; c < whole; c += 256) {
    const vec v = ((const vec*)x)[c];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double d = (double)to_f32(v[e]);
      sum[e & 1] = __builtin_fma(d, d, sum[e & 1]);
    }
  }
  for (int i = whole * E + threadIdx.x; i < count; i += 256) {
    const double d = (double)to_f32(x[i]);
    sum[0] = __builtin_fma(d, d, sum[0]);
  }
  return sum[0] + sum[1];
}

// Bound by HBM: 1.3e9 bfloat16 gradients in 452 us, 5.8 TB/s.
static __global__ __launch_bounds__(256) void grad_squares_kernel(GradList g, double* partial) {
  const int t = grad_tensor(g, blockIdx.x);
  const int64_t e0 = (int64_t)(blockIdx.x - g.first[t]) * kGradChunk;
  const int count = (int)(g.count[t] - e0 < kGradChunk ? g.count[t] - e0 : kGradChunk);
  const double sum = group_sum(g.src_b16[t] ? grad_squares((const bf16*)g.src[t] + e0, count) : grad_squares((const float*)g.src[t] + e0, count));
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename T, typename TD> __device__ __forceinline__ void grad_scale(const T* x, TD* y, int count, float by) {
  typedef T vec __attribute__((ext_vector_type(8)));
  typedef TD vecd __attribute__((ext_vector_type(8)));
  const int whole = (((uintptr_t)x | (uintptr_t)y) & 15) == 0 ? count / 8 : 0;
  int c = threadIdx.x;
  auto scaled = [&](vec v) {
    vecd out;
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = from_f32<TD>(to_f32(v[e]) * by);
    return out;
  };
  for (; c + 3 * 256 < whole; c += 1024) {
    vec v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) __builtin_memcpy(&v[k], __builtin_assume_aligned(x + (int64_t)(c + k * 256) * 8, 16), sizeof(vec));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const vecd out = scaled(v[k]);
      __builtin_memcpy(__builtin_assume_aligned(y + (int64_t)(c + k * 256) * 8, 16), &out, sizeof(vecd));
    }
  }
  for (; c < whole; c += 256) {
    vec v;
    __builtin_memcpy(&v, __builtin_assume_aligned(x + (int64_t)c * 8, 16), sizeof(vec));
    const vecd out = scaled(v);
    __builtin_memcpy(__builtin_assume_aligned(y + (int64_t)c * 8, 16), &out, sizeof(vecd));
  }
  for (int i = whole * 8 + threadIdx.x; i < count; i += 256) y[i] = from_f32<TD>(to_f32(x[i]) * by);
}

// The last work-groups' elements first: those the norm's pass has left in the memory-side cache.  1.3e9 bfloat16 gradients in place 972 us, 5.4 TB/s
// read and written.
static __global__ __launch_bounds__(256) void grad_scale_kernel(GradList g, const float* factor) {
  const uint32_t group = gridDim.x - 1 - blockIdx.x;
  const int t = grad_tensor(g, group);
  const float by = *factor;
  if (by == 1.f && g.src[t] == g.dst[t]) return;   // nothing changes
  const int64_t e0 = (int64_t)(group - g.first[t]) * kGradChunk;
  const int count = (int)(g.count[t] - e0 < kGradChunk ? g.count[t] - e0 : kGradChunk);
  if (g.src_b16[t]) {
    if (g.dst_b16[t]) grad_scale((const bf16*)g.src[t] + e0, (bf16*)g.dst[t] + e0, count, by);
    else grad_scale((const bf16*)g.src[t] + e0, (float*)g.dst[t] + e0, count, by);
  } else {
    if (g.dst_b16[t]) grad_scale((const float*)g.src[t] + e0, (bf16*)g.dst[t] + e0, count, by);
    else grad_scale((const float*)g.src[t] + e0, (float*)g.dst[t] + e0, count, by);
  }
}

// ---- factored gradients --------------------------------------------------------------------------------------
// One factor X of a pair: [rows, r], or [r, rows] where `wide`.
struct GramSide {
  const void* x;
  int64_t rows, ld;
  uint32_t first;      // work-group
  uint32_t splits;
  int64_t parts;       // floats from the workspace on: [splits][tiles][128][128]
  int r, wide;
};
struct GramList {
  GramSide side[2 * kGradFactors];
  int sides;
  float* parts;
};

// A tile of X^T X over kGramRows of the contracted index: 128 x 128, each of four waves 64 x 64.  28 pairs of rank 256 (4096 to 14336 rows a side):
// 54 us, 0.6 PFLOP/s of the three tiles in four that are formed; their bytes take 35, the products 20.
template <typename T> __global__ __launch_bounds__(256, 1) void gram_kernel(GramList g) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  using Tile = Tile32<T, 4>;
  constexpr int BN = Tile::BN;
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave >> 1, wj = wave & 1;
  const int s = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < g.sides && g.side[lane < g.sides ? lane : 0].first <= blockIdx.x)) - 1);
  const GramSide& x = g.side[s];
  const int n_tiles = (x.r + kGramTile - 1) / kGramTile, tiles = n_tiles * (n_tiles + 1) / 2;
  const int unit = (int)(blockIdx.x - x.first), split = unit / tiles;
  int ti = 0, tj = unit - split * tiles;   // tj <= ti
  while (tj > ti) tj -= ++ti;
  const int64_t k0 = (int64_t)split * kGramRows;
  const int k_count = (int)(x.rows - k0 < kGramRows ? x.rows - k0 : kGramRows);
  const bool diagonal = ti == tj;
  const Tile32Reads<T, 4> at(lane, 2 * wi), bt(lane, 2 * wj);
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x16{};

  if (!x.wide) {   // both operands are columns of tiles of BN rows x 128
    const Tile32Loader<T, 4, 4> a(lane, wave, x.ld, x.r - ti * kGramTile), b(lane, wave, x.ld, x.r - tj * kGramTile);
    const T* base = (const T*)x.x + k0 * x.ld;
    const int steps = (k_count + BN - 1) / BN;
    auto width = [&](int t) { return x.r - t * kGramTile < kGramTile ? x.r - t * kGramTile : kGramTile; };
    auto issue = [&](int t) {
      const uint32_t stage = lds + (t & 1) * 2 * Tile::BYTES;
      a.issue(base + ti * kGramTile, t * BN, k_count - t * BN, x.ld, width(ti), stage, wave);
      if (!diagonal) b.issue(base + tj * kGramTile, t * BN, k_count - t * BN, x.ld, width(tj), stage + Tile::BYTES, wave);
    };
    issue(0);
    for (int t = 0; t < steps; ++t) {
      wait_vmcnt0();
      __syncthreads();
      if (t + 1 < steps) issue(t + 1);
      const char* as = smem + (t & 1) * 2 * Tile::BYTES;
      const char* bs = diagonal ? as : as + Tile::BYTES;
#pragma unroll
      for (int u = 0; u < BN / 16; ++u) {
        typename TransFrag<T>::type af[2], bf[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          af[i] = at.column(as, u, i);
          bf[i] = bt.column(bs, u, i);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) mma(acc[i][j], af[i], bf[j]);
      }
    }
  } else {         // both are rows of tiles of 128 x 128 elements along the contracted index
    constexpr int HALVES = 128 / BN;   // tiles of BN rows
    const int steps = (k_count + 127) / 128;
    const T* base = (const T*)x.x + k0;
    for (int t = 0; t < steps; ++t) {
      const int left = k_count - t * 128;
      const Tile32Loader<T, 4, 4> load(lane, wave, x.ld, left);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2 * HALVES; ++i) {
        const int row = (i < HALVES ? ti : tj) * kGramTile + (i % HALVES) * BN, there = x.r - row;
        // (rows behind r: the last one's, whose sums are not used)
        load.issue(base + t * 128, there > 0 ? row : x.r - 1, there > 0 ? there : 1, x.ld, left < 128 ? left : 128, lds + i * Tile::BYTES, wave);
      }
      wait_vmcnt0();
      __syncthreads();
#pragma unroll
      for (int st = 0; st < Tile::STEPS; ++st) {
        typename DirectFrag<T>::type af[2], bf[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // 32 rows each, one tile after another
          af[i] = at.row(smem + Tile::block(2 * wi + i), st);
          bf[i] = at.row(smem + HALVES * Tile::BYTES + Tile::block(2 * wj + i), st);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) mma(acc[i][j], af[i], bf[j]);
      }
    }
  }
  // columns are the lanes': [row of the tile][column]
  float* out = g.parts + x.parts + (int64_t)unit * kGramTile * kGramTile;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      for_regs([&](int r) { out[(64 * wi + 32 * i + 8 * (r >> 2) + 4 * h + (r & 3)) * kGramTile + 64 * wj + 32 * j + c] = acc[i][j][r]; });
}

// sum (L^T L) o (G^T G) of pair p (its sides 2 p and 2 p + 1), 16 rows of a tile a work-group; tiles off the diagonal count twice.  8 us for 28 pairs.
struct GramSumList {
  GramList g;
  uint32_t first[kGradFactors];
  int pairs;
};
static __global__ __launch_bounds__(256) void gram_sum_kernel(GramSumList l, double* partial) {
  const int lane = threadIdx.x & 63;
  const int p = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < l.pairs && l.first[lane < l.pairs ? lane : 0] <= blockIdx.x)) - 1);
  const GramSide &a = l.g.side[2 * p], &b = l.g.side[2 * p + 1];
  const int n_tiles = (a.r + kGramTile - 1) / kGramTile, tiles = n_tiles * (n_tiles + 1) / 2;
  const int unit = (int)(blockIdx.x - l.first[p]), tile = unit / 8, rows = unit - tile * 8;
  int ti = 0, tj = tile;
  while (tj > ti) tj -= ++ti;
  double sum = 0.0;
  for (int e = threadIdx.x; e < 4 * kGramTile; e += 256) {   // four columns a lane
    const int i = rows * 16 + e / (kGramTile / 4), j = e % (kGramTile / 4) * 4;
    if (ti * kGramTile + i >= a.r || tj * kGramTile + j >= a.r) continue;
    double one[2][4];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const GramSide& s = side ? b : a;
      const float* from = l.g.parts + s.parts + (int64_t)tile * kGramTile * kGramTile + i * kGramTile + j;
#pragma unroll
      for (int c = 0; c < 4; ++c) one[side][c] = 0.0;
#pragma unroll 4
      for (uint32_t k = 0; k < s.splits; ++k) {
        const f32x4 x = *(const f32x4*)(from + (int64_t)k * tiles * kGramTile * kGramTile);
#pragma unroll
        for (int c = 0; c < 4; ++c) one[side][c] += (double)x[c];
      }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) sum += one[0][c] * one[1][c];
  }
  sum = group_sum(ti == tj ? sum : 2.0 * sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// out[0] = the norm, out[1] = min(1, max_norm / (norm + 1e-6)); NaN where the norm is.
static __global__ __launch_bounds__(256) void grad_norm_kernel(const double* partial, int64_t count, float max_norm, float* out) {
  double sum = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < count; i += 256) sum += partial[i];
  sum = group_sum(sum);
  if (threadIdx.x) return;
  const double norm = sqrt(sum < 0.0 ? 0.0 : sum);   // (a pair whose product vanishes may leave less than nothing)
  const double by = (double)max_norm / (norm + 1e-6);
  out[0] = (float)norm;
  out[1] = by > 1.0 ? 1.f : (float)by;
}

}  // namespace acc
