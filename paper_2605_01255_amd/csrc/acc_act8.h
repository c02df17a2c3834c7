// 8-bit checkpoints of activations: X [n, c] -> one byte per element and one power-of-two scale 2^e for every 32 consecutive tokens
// of a channel, and back.
//
//   e = the least whole number >= -100 with max |x| <= T 2^e over the block's finite elements, T = 448 (e4m3) or 127 (int8);
//   q = x / 2^e rounded to nearest even; what is not finite gets the format's code for it (0x7F, -128) and reads back as NaN.
//   Magnitudes above 1.875 2^127 are kept as that, so that no finite value reads back as infinite.
//
// Why blocks along the tokens: the large magnitudes of a trained model's activations sit in few channels, which a block along the
// channels would share with their neighbours and flush those.  Why powers of two: a byte times its scale is then a bfloat16 number
// exactly (e4m3 has four significant bits, int8 seven), so a product of the checkpoint on the matrix instructions rounds nothing
// that the quantisation did not; and the exponent is one byte.  e >= -100 keeps every value that is read back a normal number.
//
// All kernels here are bound by HBM.  One wave takes 32 tokens x 64 channels: lane = 8 channels (16 bytes of bfloat16) of 4 tokens,
// all its loads requested at once, so a block's maximum needs three exchanges between lanes and no LDS, and rows are read in whole
// cache lines.  Eight tokens a lane take twice the registers: the gated forward pass of 16384 x 8192 226 us against 203 on one box
// (189 to 203 since, its backward pass 186 to 192: 5.3 to 5.8 TB/s, where a copy runs at 5.0); pack and unpack of 16384 x 4096 the same
// with both (35 to 40 and 31 us).
#pragma once
#include "acc_common.h"

namespace acc {

constexpr int kActBlock = ACC_ACT8_BLOCK;
constexpr int kActTokens = 4;               // tokens of a lane
constexpr int kActLanes = 64 / (kActBlock / kActTokens);   // side by side, 8 channels each; the lanes above them hold the block's other tokens
constexpr int kActChannels = 8 * kActLanes; // of a wave
constexpr uint32_t kActTop = 0x7F700000u;   // 1.875 2^127, as float bits
constexpr uint32_t kInf = 0x7F800000u;

// Eight consecutive elements as they lie in memory (16-byte aligned).
template <typename T> struct ActRow;
template <> struct ActRow<bf16> {
  u32x4 raw;
  __device__ __forceinline__ void load(const bf16* p) { raw = *(const u32x4*)p; }
  __device__ __forceinline__ void clear() { raw = u32x4{0, 0, 0, 0}; }
  // The compiler takes the value for a new one: it does not keep what it has unpacked of it in registers of its own.
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(raw)); }
  template <int T> __device__ __forceinline__ float get() const { return __uint_as_float(T % 2 ? raw[T / 2] & 0xFFFF0000u : raw[T / 2] << 16); }
  // bits: a float whose lower half is zero
  template <int T> __device__ __forceinline__ void set(uint32_t bits) { raw[T / 2] = T % 2 ? (raw[T / 2] & 0xFFFFu) | bits : (raw[T / 2] & 0xFFFF0000u) | bits >> 16; }
};
template <> struct ActRow<float> {
  u32x4 raw[2];
  __device__ __forceinline__ void load(const float* p) {
    raw[0] = *(const u32x4*)p;
    raw[1] = *(const u32x4*)(p + 4);
  }
  __device__ __forceinline__ void clear() { raw[0] = raw[1] = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(raw[0]), "+v"(raw[1])); }
  template <int T> __device__ __forceinline__ float get() const { return __uint_as_float(raw[T / 4][T % 4]); }
  template <int T> __device__ __forceinline__ void set(uint32_t bits) { raw[T / 4][T % 4] = bits; }
};
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  bf16x8 x;
#pragma unroll
  for (int t = 0; t < 8; ++t) x[t] = (bf16)v[t];
  *(bf16x8*)p = x;
}

// The largest magnitude of each of a block's eight channels, as float bits, over this lane's tokens and those of the three lanes that
// hold the block's others.  bfloat16 magnitudes are compared as they lie, two at a time.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ void act_largest(const ActRow<bf16> (&x)[kActTokens], uint32_t (&largest)[8]) {
  static_for<0, 4>([&](auto pair) {
    constexpr int P = decltype(pair)::value;
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < kActTokens; ++k) m = max_halves(m, x[k].raw[P] & 0x7FFF7FFFu);
#pragma unroll
    for (int d = kActLanes; d < 64; d *= 2) m = max_halves(m, (uint32_t)__shfl_xor((int)m, d));
    largest[2 * P] = m << 16;
    largest[2 * P + 1] = m & 0xFFFF0000u;
  });
}
__device__ __forceinline__ void act_largest(const ActRow<float> (&x)[kActTokens], uint32_t (&largest)[8]) {
  static_for<0, 8>([&](auto channel) {
    constexpr int C = decltype(channel)::value;
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < kActTokens; ++k) {
      const uint32_t a = x[k].raw[C / 4][C % 4] & 0x7FFFFFFFu;
      m = a > m ? a : m;
    }
#pragma unroll
    for (int d = kActLanes; d < 64; d *= 2) {
      const uint32_t o = (uint32_t)__shfl_xor((int)m, d);
      m = o > m ? o : m;
    }
    largest[C] = m;
  });
}

// e + 127 of a block whose largest finite magnitude has these float bits.
template <int FORMAT> __device__ __forceinline__ uint32_t act_exponent(uint32_t largest) {
  if (largest > kActTop) largest = kActTop;
  // 448 = 1.75 2^8, 127 = 1.984375 2^6
  constexpr uint32_t FRAC = FORMAT == ACC_ACT8_E4M3 ? 0x600000u : 0x7E0000u;
  constexpr int SHIFT = FORMAT == ACC_ACT8_E4M3 ? 8 : 6;
  const int e = (int)(largest >> 23) - SHIFT + ((largest & 0x7FFFFFu) > FRAC ? 1 : 0);
  return (uint32_t)(e < 27 ? 27 : e);
}
__device__ __forceinline__ float act_scale(uint32_t e) { return __uint_as_float(e << 23); }                 // 2^e
__device__ __forceinline__ float act_inverse_scale(uint32_t e) { return __uint_as_float((254u - e) << 23); }  // 2^-e

// Four elements over their scales, |y| <= T, as four bytes.
template <int FORMAT> __device__ __forceinline__ uint32_t act_bytes(float y0, float y1, float y2, float y3) {
  if constexpr (FORMAT == ACC_ACT8_E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y0, y1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y2, y3, w, true);
  } else {
    // 1.5 2^23 + y: the sum's last place is 1, so it is rounded to a whole number whose low byte is y in two's complement
    const uint32_t b0 = __float_as_uint(y0 + 12582912.f), b1 = __float_as_uint(y1 + 12582912.f);
    const uint32_t b2 = __float_as_uint(y2 + 12582912.f), b3 = __float_as_uint(y3 + 12582912.f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b3, b2, 0x0C0C0400u), __builtin_amdgcn_perm(b1, b0, 0x0C0C0400u), 0x05040100u);
  }
}
template <int FORMAT> constexpr uint32_t kActNotFinite = FORMAT == ACC_ACT8_E4M3 ? 0x7Fu : 0x80u;

// Whether a lane's bytes may hold a code for what is not finite: the sign bits of bytes that are the int8 code (the lowest of them
// exactly, others beside it perhaps).  e4m3's conversion gives NaN by itself.
template <int FORMAT> __device__ __forceinline__ uint32_t act_odd(u32x2 q) {
  if constexpr (FORMAT == ACC_ACT8_E4M3) return 0;
  const uint32_t a = q[0] ^ 0x80808080u, b = q[1] ^ 0x80808080u;
  return (((a - 0x01010101u) & ~a) | ((b - 0x01010101u) & ~b)) & 0x80808080u;
}
// Element t of four bytes as float, without its scale; CHECK: the int8 code for what is not finite may be among them.
template <int FORMAT, int T, bool CHECK> __device__ __forceinline__ float act_element(uint32_t w) {
  if constexpr (FORMAT == ACC_ACT8_E4M3) {
    return __builtin_amdgcn_cvt_f32_fp8((int)w, T);
  } else {
    const int q = (int)(int8_t)(w >> (8 * T));
    return CHECK && q == -128 ? __uint_as_float(0x7FC00000u) : (float)q;
  }
}
// Eight bytes' scales; eight bytes times them.
__device__ __forceinline__ void act_scales(u32x2 e, float (&scale)[8]) {
  static_for<0, 8>([&](auto t) { scale[decltype(t)::value] = act_scale((e[decltype(t)::value / 4] >> (8 * (decltype(t)::value % 4))) & 0xFFu); });
}
template <int FORMAT, bool CHECK> __device__ __forceinline__ void act_values(u32x2 q, const float (&scale)[8], float (&v)[8]) {
  static_for<0, 8>([&](auto t) {
    constexpr int T = decltype(t)::value;
    v[T] = act_element<FORMAT, T % 4, CHECK>(q[T / 4]) * scale[T];
  });
}

// A wave's tile: 8 channels from `c`, tokens row .. row + 3 of block `block`.
struct ActLane {
  int64_t block, row, c;
  int rows;       // tokens of this lane that exist (0: none, or its channels do not)
  int group;      // which part of the block
};
__device__ __forceinline__ ActLane act_lane(int64_t n, int64_t c) {
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
  const int64_t across = (c + kActChannels - 1) / kActChannels;
  ActLane l;
  l.block = wave / across;
  l.group = lane / kActLanes;
  l.c = (wave - l.block * across) * kActChannels + (lane % kActLanes) * 8;
  l.row = l.block * kActBlock + l.group * kActTokens;
  const int64_t left = n - l.row;
  l.rows = l.c >= c || left <= 0 ? 0 : (int)(left < kActTokens ? left : kActTokens);
  return l;
}
inline __host__ int64_t act_work_groups(int64_t n, int64_t c) {  // of 256 lanes
  return ceil_div(ceil_div(n, kActBlock) * ceil_div(c, kActChannels), 4);
}

// This lane's four tokens of eight channels (0 where a token does not exist) into the checkpoint [n, c].
template <int FORMAT, typename T>
__device__ __forceinline__ void act_keep(const ActLane& l, int64_t c, ActRow<T> (&x)[kActTokens], uint8_t* __restrict__ Q, uint8_t* __restrict__ E) {
  uint32_t largest[8], any = 0;
  act_largest(x, largest);
#pragma unroll
  for (int t = 0; t < 8; ++t) any = largest[t] > any ? largest[t] : any;
  uint64_t odd = 0;   // bit 8 k + t: element [k][t] is not finite
  if (__any(any > kActTop)) {
    static_for<0, kActTokens * 8>([&](auto at) {
      constexpr int K = decltype(at)::value / 8, C = decltype(at)::value % 8;
      const uint32_t bits = __float_as_uint(x[K].template get<C>()), a = bits & 0x7FFFFFFFu;
      if (a >= kInf) odd |= (uint64_t)1 << (8 * K + C);
      x[K].template set<C>(a >= kInf ? 0u : a > kActTop ? (bits & 0x80000000u) | kActTop : bits);
    });
    act_largest(x, largest);
  }
#pragma unroll
  for (int k = 0; k < kActTokens; ++k) x[k].renew();
  if (l.rows == 0) return;
  uint32_t e[8];
  float inv[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    e[t] = act_exponent<FORMAT>(largest[t]);
    inv[t] = act_inverse_scale(e[t]);
  }
  if (l.group == 0) {
    const u32x2 packed = {e[0] | e[1] << 8 | e[2] << 16 | e[3] << 24, e[4] | e[5] << 8 | e[6] << 16 | e[7] << 24};
    *(u32x2*)(E + l.block * c + l.c) = packed;
  }
  static_for<0, kActTokens>([&](auto token) {
    constexpr int K = decltype(token)::value;
    __builtin_amdgcn_sched_barrier(0);
    if (K >= l.rows) return;
    u32x2 q;
    static_for<0, 2>([&](auto half) {
      constexpr int H = decltype(half)::value, C = 4 * H;
      uint32_t w = act_bytes<FORMAT>(x[K].template get<C>() * inv[C], x[K].template get<C + 1>() * inv[C + 1], x[K].template get<C + 2>() * inv[C + 2],
                                     x[K].template get<C + 3>() * inv[C + 3]);
      if (odd) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (odd >> (8 * K + C + t) & 1) w = (w & ~(0xFFu << (8 * t))) | kActNotFinite<FORMAT> << (8 * t);
      }
      q[H] = w;
    });
    *(u32x2*)(Q + (l.row + K) * c + l.c) = q;
  });
}

template <typename T> __device__ __forceinline__ void act_load(const ActLane& l, const T* __restrict__ X, int64_t ld, ActRow<T> (&x)[kActTokens]) {
#pragma unroll
  for (int k = 0; k < kActTokens; ++k) {
    if (k < l.rows) x[k].load(X + (l.row + k) * ld + l.c);
    else x[k].clear();
  }
}

template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void act8_pack_kernel(const T* __restrict__ X, int64_t n, int64_t c, int64_t ld, uint8_t* __restrict__ Q, uint8_t* __restrict__ E) {
  const ActLane l = act_lane(n, c);
  ActRow<T> x[kActTokens];
  act_load(l, X, ld, x);
  act_keep<FORMAT>(l, c, x, Q, E);
}

template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void act8_unpack_kernel(const uint8_t* __restrict__ Q, const uint8_t* __restrict__ E, int64_t n, int64_t c, int64_t ld, T* __restrict__ X) {
  const ActLane l = act_lane(n, c);
  if (l.rows == 0) return;
  const u32x2 e = *(const u32x2*)(E + l.block * c + l.c);
  u32x2 q[kActTokens];
#pragma unroll
  for (int k = 0; k < kActTokens; ++k)
    if (k < l.rows) q[k] = *(const u32x2*)(Q + (l.row + k) * c + l.c);
  float scale[8];
  act_scales(e, scale);
#pragma unroll
  for (int k = 0; k < kActTokens; ++k) {
    if (k >= l.rows) break;
    float v[8];
    act_values<FORMAT, true>(q[k], scale, v);
    store8(X + (l.row + k) * ld + l.c, v);
  }
}

// The parts of a product added up: C[row, ldc] (+)= sum of `splits` matrices of `count` elements, rows of `row`.  Four elements a thread,
// eight parts requested at a time.
template <typename TC, bool SUM>
__global__ __launch_bounds__(256) void add_parts_kernel(const float* __restrict__ parts, int splits, int64_t count, int64_t row, int64_t ldc, TC* __restrict__ C) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= count) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = 0; k < splits; ++k) sum += *(const f32x4*)(parts + k * count + e);
  TC* dst = C + e / row * ldc + e % row;
#pragma unroll
  for (int t = 0; t < 4; ++t) dst[t] = from_f32<TC>(SUM ? sum[t] + to_f32(dst[t]) : sum[t]);
}

// 1 / (1 + exp(-x)); 0 and 1 at the ends, as exp overflows to infinity or vanishes.  bfloat16 results take the hardware's
// exponential and reciprocal (a few 2^-23 of the value, under the rounding of 2^-8), float32 ones the library's.
template <typename T> __device__ __forceinline__ float sigmoid(float x) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.f + __expf(-x));
  else return 1.f / (1.f + expf(-x));
}

// H = silu(G) o U, and G and U into their checkpoints.  A row of H at a time: unrolled together the rows' intermediate values take the
// registers of two waves more per SIMD.
template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void gated_fwd_kernel(const T* __restrict__ G, const T* __restrict__ U, int64_t n, int64_t f, int64_t ldg, int64_t ldh,
                                                        T* __restrict__ H, uint8_t* __restrict__ Qg, uint8_t* __restrict__ Eg, uint8_t* __restrict__ Qu,
                                                        uint8_t* __restrict__ Eu) {
  const ActLane l = act_lane(n, f);
  ActRow<T> g[kActTokens], u[kActTokens];
  act_load(l, G, ldg, g);
  act_load(l, U, ldg, u);
  static_for<0, kActTokens>([&](auto token) {
    constexpr int K = decltype(token)::value;
    __builtin_amdgcn_sched_barrier(0);
    if (K >= l.rows) return;
    float h[8];
    static_for<0, 8>([&](auto t) {
      constexpr int C = decltype(t)::value;
      const float x = g[K].template get<C>();
      h[C] = x * sigmoid<T>(x) * u[K].template get<C>();
    });
    store8(H + (l.row + K) * ldh + l.c, h);
  });
#pragma unroll
  for (int k = 0; k < kActTokens; ++k) {
    g[k].renew();
    u[k].renew();
  }
  __builtin_amdgcn_sched_barrier(0);
  act_keep<FORMAT>(l, f, g, Qg, Eg);
  __builtin_amdgcn_sched_barrier(0);
  act_keep<FORMAT>(l, f, u, Qu, Eu);
}

// With s = sigmoid(G^):  dU = dH o G^ s,  dG = dH o U^ s (1 + G^ (1 - s)),  and on request H = G^ s o U^ again.  A row at a time, as in
// the forward pass.
template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void gated_bwd_kernel(const T* __restrict__ dH, const uint8_t* __restrict__ Qg, const uint8_t* __restrict__ Eg,
                                                        const uint8_t* __restrict__ Qu, const uint8_t* __restrict__ Eu, int64_t n, int64_t f, int64_t ldg,
                                                        int64_t ldh, T* __restrict__ dG, T* __restrict__ dU, T* __restrict__ H) {
  const ActLane l = act_lane(n, f);
  if (l.rows == 0) return;
  const u32x2 eg = *(const u32x2*)(Eg + l.block * f + l.c), eu = *(const u32x2*)(Eu + l.block * f + l.c);
  u32x2 qg[kActTokens], qu[kActTokens];
  ActRow<T> dh[kActTokens];
  uint32_t odd = 0;
#pragma unroll
  for (int k = 0; k < kActTokens; ++k)
    if (k < l.rows) {
      const int64_t row = l.row + k;
      qg[k] = *(const u32x2*)(Qg + row * f + l.c);
      qu[k] = *(const u32x2*)(Qu + row * f + l.c);
      dh[k].load(dH + row * ldh + l.c);
    }
  float sg[8], su[8];
  act_scales(eg, sg);
  act_scales(eu, su);
#pragma unroll
  for (int k = 0; k < kActTokens; ++k)
    if (k < l.rows) odd |= act_odd<FORMAT>(qg[k]) | act_odd<FORMAT>(qu[k]);
  auto rows = [&](auto check) {
    static_for<0, kActTokens>([&](auto token) {
      constexpr int K = decltype(token)::value;
      constexpr bool CHECK = decltype(check)::value;
      __builtin_amdgcn_sched_barrier(0);
      if (K >= l.rows) return;
      const int64_t row = l.row + K;
      float g[8], u[8], dg[8], du[8];
      act_values<FORMAT, CHECK>(qg[K], sg, g);
      act_values<FORMAT, CHECK>(qu[K], su, u);
      static_for<0, 8>([&](auto t) {
        constexpr int C = decltype(t)::value;
        const float s = sigmoid<T>(g[C]), a = g[C] * s, d = dh[K].template get<C>();
        du[C] = d * a;
        dg[C] = d * u[C] * (s + a * (1.f - s));
        u[C] *= a;
      });
      store8(dG + row * ldg + l.c, dg);
      store8(dU + row * ldg + l.c, du);
      if (H) store8(H + row * ldh + l.c, u);
    });
  };
  if (__any(odd)) rows(std::true_type{});
  else rows(std::false_type{});
}

}  // namespace acc
