// Blocks of 32 x 32 on the matrix pipe and the LDS tiles that feed them, bfloat16 or float (attention, sums over the rows of a matrix).
#pragma once
#include "acc_gemm.h"

namespace acc {

// f of 0 .. 15 as constants: registers of a block, which an ordinary loop may be unrolled too late to keep out of scratch memory.
template <typename F> __device__ __forceinline__ void for_regs(F&& f) { static_for<0, 16>(f); }

// A row of a tile takes PITCH bytes of LDS, a power of two; 16-byte chunk c of row r lies at chunk c ^ row_swizzle(r).  Direct reads of one
// chunk of 16 rows, and transposing reads of 4 rows x 32 columns, then fall on all 64 banks.
template <int PITCH> __device__ __forceinline__ int row_swizzle(int row) {
  if constexpr (PITCH == 128) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  else return ((row & 3) << 2) | ((row >> 2) & 3);
}

template <typename T, int DB> struct Tile32 {
  static constexpr int ROW = DB * 32 * (int)sizeof(T);
  static constexpr int PITCH = ROW <= 128 ? 128 : ROW <= 256 ? 256 : 512;
  static constexpr int CHUNKS = PITCH / 16, ROWS_PER_LOAD = 1024 / PITCH, PER_CHUNK = 16 / (int)sizeof(T);
  static constexpr int STEPS = DB * 32 / (2 * PER_CHUNK);   // direct operands along the channels
  static constexpr int BN = sizeof(T) == 2 ? 64 : 32;       // rows of a tile
  static constexpr int BYTES = BN * PITCH;
};

template <typename T> struct DirectFrag { using type = bf16x8; };
template <> struct DirectFrag<float> { using type = f32x4; };
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T> struct TransFrag { using type = bf16x8; };
template <> struct TransFrag<float> { using type = f32x8; };

__device__ __forceinline__ void mma(f32x16& c, bf16x8 a, bf16x8 b) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mma(f32x16& c, f32x4 a, f32x4 b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& c, f32x8 a, f32x8 b) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
}

// This lane's places in a tile.
template <typename T, int DB> struct Tile32Reads {
  using Tile = Tile32<T, DB>;
  static constexpr int TRANS = sizeof(T) == 2 ? 2 : 4;
  int direct[Tile::STEPS];
  int trans[DB][TRANS];
  // columns are counted from 32-channel block `from` on
  __device__ __forceinline__ explicit Tile32Reads(int lane, int from = 0) {
    const int c = lane & 31, h = lane >> 5;
#pragma unroll
    for (int s = 0; s < Tile::STEPS; ++s) direct[s] = c * Tile::PITCH + (((2 * s + h) ^ row_swizzle<Tile::PITCH>(c)) << 4);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int t = 0; t < TRANS; ++t) {
        if constexpr (sizeof(T) == 2) {   // rows 4 h + 8 t .. + 3 of a step of 16
          const int row = 4 * h + 8 * t + ((lane & 15) >> 2), col = (from + db) * 32 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          trans[db][t] = row * Tile::PITCH + (((col >> 3) ^ row_swizzle<Tile::PITCH>(row)) << 4) + (col & 7) * 2;
        } else {   // rows 4 h + t and 8 more
          const int row = 4 * h + t, col = (from + db) * 32 + c;
          trans[db][t] = row * Tile::PITCH + (((col >> 2) ^ row_swizzle<Tile::PITCH>(row)) << 4) + (col & 3) * 4;
        }
      }
  }
  // rows 32 block + l % 32, channels of step s
  __device__ __forceinline__ typename DirectFrag<T>::type row(const char* tile, int block, int s) const {
    return *(const typename DirectFrag<T>::type*)(tile + direct[s] + block * 32 * Tile::PITCH);
  }
  // channels 32 db + l % 32, rows 16 u + (0 .. 15) in the accumulators' order
  __device__ __forceinline__ typename TransFrag<T>::type column(const char* tile, int u, int db) const {
    if constexpr (sizeof(T) == 2) {
      const s16x4 lo = lds_read_tr16_b64(tile, trans[db][0] + u * 16 * Tile::PITCH);
      const s16x4 hi = lds_read_tr16_b64(tile, trans[db][1] + u * 16 * Tile::PITCH);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f32x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) {   // 8 rows further on the swizzle's low bits are the other way round
        const int base = e < 4 ? trans[db][e] : trans[db][e - 4] ^ (2 << 4);
        v[e] = *(const float*)(tile + base + (u * 16 + (e < 4 ? 0 : 8)) * Tile::PITCH);
      }
      return v;
    }
  }
};

// The eight accumulators of step u as an operand.  bfloat16: each rounded once, as the product takes them.
template <typename T> __device__ __forceinline__ typename TransFrag<T>::type step_operand(f32x16 x, int u) {
  const f32x8 y = u ? __builtin_shufflevector(x, x, 8, 9, 10, 11, 12, 13, 14, 15) : __builtin_shufflevector(x, x, 0, 1, 2, 3, 4, 5, 6, 7);
  if constexpr (sizeof(T) == 2) return __builtin_convertvector(y, bf16x8);
  else return y;
}

// This lane's row from memory as direct operands; rows that are none, and channels behind d, as zeros.
template <typename T, int DB> __device__ __forceinline__ void load_row(typename DirectFrag<T>::type* f, const T* base, int64_t row, int64_t ld, int d, int h, bool there) {
  using Tile = Tile32<T, DB>;
#pragma unroll
  for (int s = 0; s < Tile::STEPS; ++s) {
    const int c = (2 * s + h) * Tile::PER_CHUNK;
    typename DirectFrag<T>::type zero{};
    f[s] = there && c < d ? *(const typename DirectFrag<T>::type*)(base + row * ld + c) : zero;
  }
}

// Transposed accumulators (this lane's row, channels 32 db + 8 (r / 4) + 4 h + r % 4) times `by` to memory.
template <typename T, int DB> __device__ __forceinline__ void store_row(T* row, const f32x16* x, float by, int d, int h) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = db * 32 + 8 * g + 4 * h;
      if (c >= d) continue;
      if constexpr (sizeof(T) == 2) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16)(x[db][4 * g + e] * by);
        *(bf16x4*)(row + c) = v;
      } else {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[db][4 * g + e] * by;
        *(f32x4*)(row + c) = v;
      }
    }
}

// Rows of a matrix to LDS tiles.  `there` rows from `row` on of which the tile takes BN; the rest, and channels behind d, become zeros.
template <typename T, int DB, int NW> struct Tile32Loader {
  using Tile = Tile32<T, DB>;
  static constexpr int LOADS = Tile::BYTES / 1024 / NW;
  static_assert(LOADS * 1024 * NW == Tile::BYTES, "whole loads");
  uint32_t src[LOADS];
  __device__ __forceinline__ Tile32Loader(int lane, int wave, int64_t ld, int d) {
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      const int row = (t * NW + wave) * Tile::ROWS_PER_LOAD + lane / Tile::CHUNKS;
      const int chunk = (lane % Tile::CHUNKS) ^ row_swizzle<Tile::PITCH>(row);
      src[t] = chunk * Tile::PER_CHUNK < d ? (uint32_t)(row * (int)ld * (int)sizeof(T) + (chunk << 4)) : 0xFFFFFFF0u;
    }
  }
  __device__ __forceinline__ void issue(const T* base, int64_t row, int there, int64_t ld, int d, uint32_t lds, int wave) const {
    const int rows = there < Tile::BN ? there : Tile::BN;
    const u32x4 rsrc = make_rsrc(base + row * ld, ((int64_t)(rows - 1) * ld + d) * (int64_t)sizeof(T));
#pragma unroll
    for (int t = 0; t < LOADS; ++t) buffer_to_lds_b128(rsrc, src[t], 0, lds + (t * NW + wave) * 1024);
  }
};

// 64 lanes x 4 bytes, global -> LDS (see buffer_to_lds_b128).
__device__ __forceinline__ void buffer_to_lds_b32(u32x4 rsrc, uint32_t voffset, uint32_t lds_wave_base) {
  asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" : : "v"(voffset), "s"(rsrc), "{m0}"(lds_wave_base) : "memory");
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// x of lane % 32 and x of lane % 32 + 32.
__device__ __forceinline__ f32x2 halves(float x) {
  const uint32_t a = __builtin_bit_cast(uint32_t, x);
  const auto p = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  const uint32_t lo = p[0], hi = p[1];   // (a bit cast of an element itself takes the first)
  return f32x2{__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}
__device__ __forceinline__ float half_max(float x) { const f32x2 p = halves(x); return fmaxf(p[0], p[1]); }
__device__ __forceinline__ float half_sum(float x) { const f32x2 p = halves(x); return p[0] + p[1]; }

}  // namespace acc
