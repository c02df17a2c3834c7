// Blocks of 32 x 32 on the matrix pipe and the LDS tiles that feed them, bfloat16 or float (attention, sums over the rows of a matrix).
#pragma once
#include "acc_gemm.h"

namespace acc {

// f of 0 .. 15 as constants: registers of a block, which an ordinary loop may be unrolled too late to keep out of scratch memory.
template <typename F> __device__ __forceinline__ void for_regs(F&& f) { static_for<0, 16>(f); }

// A tile lies in LDS as super-rows of 256 bytes (a row; two rows, r and r + 32, where a row has 128; half a row where it has 512), four of
// them to a transfer of 1024 bytes and 16 bytes of room behind it: 16-byte chunk c of super-row r is at
// 1040 (r / 4) + 256 (c / 4) + 64 (r % 4) + 16 (c % 4).  Direct reads of one chunk of 16 rows, and transposing reads of 4 rows x 32 columns,
// fall on all 64 banks, a transfer takes 64 bytes of a row at a time, and every operand is at a fixed distance from one address a lane (a
// swizzle by exclusive or needs sixteen addresses, or an instruction a read).
constexpr int kTileGroup = 1040;

template <typename T, int DB> struct Tile32 {
  static constexpr int ROW = DB * 32 * (int)sizeof(T);
  static constexpr int PITCH = ROW <= 128 ? 128 : ROW <= 256 ? 256 : 512;
  static constexpr int PER_CHUNK = 16 / (int)sizeof(T);
  static constexpr int STEPS = DB * 32 / (2 * PER_CHUNK);   // direct operands along the channels
  static constexpr int BN = sizeof(T) == 2 ? 64 : 32;       // rows of a tile
  static constexpr int GROUPS = BN * PITCH / 1024, BYTES = GROUPS * kTileGroup;
  // blocks of 32 rows of one or several tiles one after another
  __device__ __forceinline__ static constexpr int block(int b) {
    return PITCH == 128 ? (b >> 1) * BYTES + (b & 1) * 512 : PITCH == 256 ? b * 8 * kTileGroup : b * BYTES;
  }
};

template <typename T> struct DirectFrag { using type = bf16x8; };
template <> struct DirectFrag<float> { using type = f32x4; };
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T> struct TransFrag { using type = bf16x8; };
template <> struct TransFrag<float> { using type = f32x8; };
// A direct operand where transposed ones go too.
__device__ __forceinline__ bf16x8 widened(bf16x8 x) { return x; }
__device__ __forceinline__ f32x8 widened(f32x4 x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }
template <typename T> __device__ __forceinline__ typename DirectFrag<T>::type narrowed(typename TransFrag<T>::type x) {
  if constexpr (sizeof(T) == 2) return x;
  else return __builtin_shufflevector(x, x, 0, 1, 2, 3);
}

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
  static constexpr int PITCH = Tile::PITCH, G = kTileGroup;
  int direct, trans;
  // columns are counted from 32-channel block `from` on
  __device__ __forceinline__ explicit Tile32Reads(int lane, int from = 0) {
    const int c = lane & 31, h = lane >> 5;
    direct = (c >> 2) * G + (c & 3) * 64 + h * 16;
    if constexpr (sizeof(T) == 2) trans = h * G + ((lane >> 2) & 3) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8 + from * 256;
    else trans = h * G + (c >> 4) * 256 + (c & 15) * 4 + columns(from);
  }
  __device__ __forceinline__ static constexpr int columns(int db) {
    if constexpr (sizeof(T) == 2) return db * 256;
    else return (db >> 1) * 8 * G + (db & 1) * 512;
  }
  // rows 32 block + l % 32 (tile: where block 0 begins), channels of step s
  __device__ __forceinline__ typename DirectFrag<T>::type row(const char* tile, int s) const {
    return *(const typename DirectFrag<T>::type*)(tile + direct + (2 * s >> 4) * 8 * G + ((2 * s & 15) >> 2) * 256 + (2 * s & 3) * 16);
  }
  // channels 32 db + l % 32, rows 16 u + (0 .. 15) in the accumulators' order
  __device__ __forceinline__ typename TransFrag<T>::type column(const char* tile, int u, int db) const {
    const char* at = tile + trans + columns(db) + (PITCH == 128 ? (u & 1) * 4 * G + (u >> 1) * 512 : u * 4 * G);
    if constexpr (sizeof(T) == 2) {
      const s16x4 lo = lds_read_tr16_b64(at, 0);
      const s16x4 hi = lds_read_tr16_b64(at, 2 * G);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f32x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = *(const float*)(at + (e >> 2) * 2 * G + (e & 3) * 64);
      return v;
    }
  }
};

// N products in their order: product(i, what read(i) gave AHEAD products before), and behind each of them work(i), what the vector pipe does
// while the matrix pipe is busy.  The fences keep the order: left alone the compiler puts each read right in front of its product, and the
// vector work in one piece behind them all.  (A product holds the vector pipe for 8 of its 32 clocks where instructions of the same wave
// follow it, for 17 where another wave's do: 8 multiply-adds for a product take 24.4 ns in one wave, 26.9 from two, of 15.8 and 18.8 alone.)
template <int N, int AHEAD, typename Read, typename Product, typename Work>
__device__ __forceinline__ void products(Read&& read, Product&& product, Work&& work) {
  decltype(read(std::integral_constant<int, 0>{})) ring[AHEAD];
  static_for<0, (AHEAD < N ? AHEAD : N)>([&](auto i) { ring[i.value] = read(i); });
  __builtin_amdgcn_sched_barrier(0);
  static_for<0, N>([&](auto i) {
    product(i, ring[i.value % AHEAD]);
    if constexpr (i.value + AHEAD < N) ring[i.value % AHEAD] = read(std::integral_constant<int, i.value + AHEAD>{});
    work(i);
    __builtin_amdgcn_sched_barrier(0);
  });
}

// x, computed here: what is only used behind a branch is moved there otherwise, past the fences.
template <typename V> __device__ __forceinline__ V here(V x) {
  asm volatile("" : "+v"(x));
  return x;
}

// f(r) for the registers of a block that fall to step j of `steps`, the first of which is left out.
template <int J, int STEPS, typename F> __device__ __forceinline__ void spread(F&& f) {
  if constexpr (J > 0) static_for<16 * (J - 1) / (STEPS - 1), 16 * J / (STEPS - 1)>([&](auto r) { f((int)r.value); });
}

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
  static constexpr int LOADS = Tile::GROUPS / NW;
  static_assert(LOADS * NW == Tile::GROUPS, "whole transfers");
  uint32_t src[LOADS];
  __device__ __forceinline__ Tile32Loader(int lane, int wave, int64_t ld, int d) {
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      const int super = 4 * (t * NW + wave) + ((lane >> 2) & 3), cc = (lane >> 4) * 4 + (lane & 3);
      const int row = Tile::PITCH == 128 ? super + 32 * (cc >> 3) : Tile::PITCH == 256 ? super : super & 31;
      const int chunk = Tile::PITCH == 128 ? cc & 7 : Tile::PITCH == 256 ? cc : cc + 16 * (super >> 5);
      src[t] = chunk * Tile::PER_CHUNK < d ? (uint32_t)(row * (int)ld * (int)sizeof(T) + (chunk << 4)) : 0xFFFFFFF0u;
    }
  }
  __device__ __forceinline__ static u32x4 rows(const T* base, int64_t row, int there, int64_t ld, int d) {
    return make_rsrc(base + row * ld, bytes(there, ld, d));
  }
  __device__ __forceinline__ static int64_t bytes(int there, int64_t ld, int d) {
    return there > 0 ? ((int64_t)((there < Tile::BN ? there : Tile::BN) - 1) * ld + d) * (int64_t)sizeof(T) : 0;
  }
  // transfer t of LOADS
  __device__ __forceinline__ void one(const u32x4& rsrc, int t, uint32_t lds, int wave) const { buffer_to_lds_b128(rsrc, src[t], 0, lds + (t * NW + wave) * kTileGroup); }
  __device__ __forceinline__ void issue(const T* base, int64_t row, int there, int64_t ld, int d, uint32_t lds, int wave) const {
    const u32x4 rsrc = rows(base, row, there, ld, d);
#pragma unroll
    for (int t = 0; t < LOADS; ++t) one(rsrc, t, lds, wave);
  }
};

// One tile after another of a run of rows: the resource moves on by additions (made anew from row and count it is three times the scalar
// instructions of a tile's transfers).  Behind the last tile there are no rows.
template <typename T, int DB, int NW> struct Tile32Run {
  using Loader = Tile32Loader<T, DB, NW>;
  u32x4 rsrc;
  uint32_t step, whole, rest;   // bytes of BN rows from the first to the first, of a whole tile, of the last one
  __device__ __forceinline__ Tile32Run(const T* base, int64_t row, int count, int64_t ld, int d) {
    constexpr int BN = Loader::Tile::BN;
    step = __builtin_amdgcn_readfirstlane((uint32_t)(BN * ld * (int64_t)sizeof(T)));
    whole = __builtin_amdgcn_readfirstlane((uint32_t)Loader::bytes(BN, ld, d));
    rest = __builtin_amdgcn_readfirstlane((uint32_t)Loader::bytes(count - (count - 1) / BN * BN, ld, d));
    rsrc = make_rsrc(base + row * ld, count > BN ? whole : rest);
  }
  __device__ __forceinline__ void skip(int t, int tiles) {
    const uint64_t at = ((uint64_t)rsrc[1] << 32 | rsrc[0]) + (uint64_t)t * step;
    rsrc[0] = (uint32_t)at;
    rsrc[1] = (uint32_t)(at >> 32);
    rsrc[2] = t + 1 < tiles ? whole : rest;
  }
  // to tile t of `tiles`, the one behind that it is at
  __device__ __forceinline__ void advance(int t, int tiles) {
    const uint64_t at = ((uint64_t)rsrc[1] << 32 | rsrc[0]) + step;
    rsrc[0] = (uint32_t)at;
    rsrc[1] = (uint32_t)(at >> 32);
    rsrc[2] = t + 1 < tiles ? whole : t + 1 == tiles ? rest : 0;
  }
  // the same rows of a matrix `bytes` further on
  __device__ __forceinline__ void back(int tiles, int64_t bytes) {
    const uint64_t at = ((uint64_t)rsrc[1] << 32 | rsrc[0]) + bytes - (uint64_t)(tiles - 1) * step;
    rsrc[0] = (uint32_t)at;
    rsrc[1] = (uint32_t)(at >> 32);
    rsrc[2] = tiles > 1 ? whole : rest;
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
