// The vocabulary's table at the other end of a model: Y_i = scale W[ids_i], and dW[w] = scale sum of dY_i over the tokens i of word w, in
// their order, so that the result is the same bits every time.
//
// Tokens are grouped by word first.  Words are dealt to kBuckets work-groups by their low bits (frequent words have small numbers in most
// tables); each counts the tokens of its words and of all smaller buckets in one pass over the numbers, so it knows its place in the grouped
// order without a word from the others, and orders its tokens by a stable counting sort.  The sums then take the grouped order in blocks of
// kEmbedBlock tokens whatever the words' frequencies are: a word inside a block is finished there, one that crosses blocks leaves a part
// for each, added up behind it in their order.  Bound by the bytes of dY and dW.
#pragma once
#include "acc_common.h"

namespace acc {

constexpr int kBuckets = 256, kBucketBits = 8, kEmbedBlock = 32;
constexpr int kWaveList = 256, kListAhead = 16;   // tokens of a wave's list; rows of numbers that it requests together
constexpr int kEmbedCounters = 16384;   // of a bucket's counting sort: its words times the waves that count apart

struct EmbedParams {
  const void *w, *dy;
  const int64_t* ids;
  void *y, *dw;
  int64_t n, v, ldw, ldy;
  int d;
  float scale;
  int add;            // dW +=
  int bins, waves;    // words of a bucket; waves of its sort
  int* order;         // tokens, grouped by word
  int2* rows;         // [kBuckets][bins] first place and number of a word's tokens
  int2* list;         // a bucket's tokens and words before they are sorted
  int* total;         // tokens of any word
  float* parts;       // [blocks][2][d]: a block's part of the word that began before it, and of the one that goes on behind it
  int grad_groups;    // work-groups of the sums; those behind them write zeros
};

// Rows of `per` tokens a work-group, 16 bytes a lane, four requested together.  16384 tokens of 4096 channels: 50 us, 5.4 TB/s, where words repeat.
template <typename T> __global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedParams p, int per) {
  constexpr int E = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(E)));
  const uint32_t row_chunks = p.d / E;
  const int64_t first = (int64_t)blockIdx.x * per;
  const uint32_t chunks = (uint32_t)(p.n - first < per ? p.n - first : per) * row_chunks;
  for (uint32_t base = 0; base < chunks; base += 1024) {
    vec x[4];
    int64_t id[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = base + k * 256 + threadIdx.x;
      id[k] = c < chunks ? p.ids[first + c / row_chunks] : -1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = base + k * 256 + threadIdx.x;
      x[k] = vec{};
      if (id[k] >= 0 && id[k] < p.v) x[k] = *(const vec*)((const T*)p.w + id[k] * p.ldw + c % row_chunks * E);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t c = base + k * 256 + threadIdx.x;
      if (c >= chunks) continue;
      vec y;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = from_f32<T>(id[k] >= p.v ? __builtin_nanf("") : to_f32(x[k][e]) * p.scale);
      if (id[k] < 0) y = vec{};
      *(vec*)((T*)p.y + (first + c / row_chunks) * p.ldy + c % row_chunks * E) = y;
    }
  }
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// One work-group of 1024 for each bucket: its tokens in p.order, its words' places in p.rows.  LDS: p.bins * p.waves counters, then a list of
// kWaveList tokens for each wave.  A wave goes over a sixteenth of the numbers and appends its tokens to its list, so the lists one after another
// are in the tokens' order; where one is too short (a word that most tokens have, very many tokens) the work-group goes over the numbers again,
// all waves together, and lists its tokens in memory.  12 us for 16384 and 32768 tokens, waits one after another; with a second
// pass for all of them 16 and 21.
static __global__ __launch_bounds__(1024) void embed_group_kernel(EmbedParams p) {
  extern __shared__ int counter[];
  __shared__ int sums[2][16], listed[16], scan[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, bucket = blockIdx.x;
  const int n = (int)p.n, counters = p.bins * p.waves;
  int2* lists = (int2*)(counter + (counters + 1) / 2 * 2);
  for (int i = tid; i < counters; i += 1024) counter[i] = 0;
  // tokens of the buckets before this one, and of this one
  int before = 0, own = 0;
  {
    const int run = (n + 16 * 64 - 1) / (16 * 64) * 64, end = n - wave * run < run ? n : (wave + 1) * run;
    for (int i0 = wave * run; i0 < end; i0 += 64 * kListAhead) {
      int64_t id[kListAhead];
#pragma unroll
      for (int k = 0; k < kListAhead; ++k) id[k] = i0 + k * 64 + lane < end ? p.ids[i0 + k * 64 + lane] : -1;
#pragma unroll
      for (int k = 0; k < kListAhead; ++k) {
        const bool word = (uint64_t)id[k] < (uint64_t)p.v;
        const int b = (int)(id[k] & (kBuckets - 1));
        before += word && b < bucket;
        const uint64_t mine = __ballot(word && b == bucket);
        const int at = own + lanes_below(mine);
        if (word && b == bucket && at < kWaveList) lists[wave * kWaveList + at] = make_int2(i0 + k * 64 + lane, (int)(id[k] >> kBucketBits));
        own += __popcll(mine);
      }
    }
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) before += __shfl_xor(before, s);
  if (lane == 0) {
    sums[0][wave] = before;
    listed[wave] = own;
  }
  __syncthreads();
  bool again = false;
  before = own = 0;
  for (int w = 0; w < 16; ++w) {
    before += sums[0][w];
    own += listed[w];
    again |= listed[w] > kWaveList;
  }
  if (bucket == kBuckets - 1 && tid == 0) *p.total = before + own;

  // this bucket's tokens in their order, four neighbours a lane
  int2* list = p.list;
  if (again) {
    __syncthreads();
    int at = before;
    int64_t ahead[4];
    auto request = [&](int i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) ahead[e] = i + e < n ? p.ids[i + e] : -1;
    };
    request(4 * tid);
    for (int i0 = 0, turn = 0; i0 < n; i0 += 4096, turn ^= 1) {
      const int i = i0 + 4 * tid;
      int64_t id[4];
      uint32_t mine = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) id[e] = ahead[e];
      request(i + 4096);   // (behind the last number: none)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((uint64_t)id[e] < (uint64_t)p.v && (int)(id[e] & (kBuckets - 1)) == bucket) mine |= 1u << e;
      }
      const int count = __popc(mine);
      int below = 0, all = 0;
#pragma unroll
      for (int bit = 0; bit < 3; ++bit) {
        const uint64_t m = __ballot((count >> bit) & 1);
        below += lanes_below(m) << bit;
        all += __popcll(m) << bit;
      }
      if (lane == 0) sums[turn][wave] = all;
      __syncthreads();
      int to = at + below;
      for (int w = 0; w < 16; ++w) {
        const int s = sums[turn][w];
        to += w < wave ? s : 0;
        at += s;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (mine >> e & 1) list[to++] = make_int2(i + e, (int)(id[e] >> kBucketBits));
    }
    __syncthreads();
  }
  // Counting sort: wave w has a run of the list, counter[word][w] its tokens of a word, then their first place.
  const bool sorts = wave < p.waves;
  auto pieces = [&](auto&& f) {   // f(tokens and words, their number) for the pieces of this wave's run
    if (!sorts) return;
    if (again) {
      const int run = (own + p.waves * 64 - 1) / (p.waves * 64) * 64;
      const int from = wave * run < own ? wave * run : own, until = (wave + 1) * run < own ? (wave + 1) * run : own;
      f(list + before + from, until - from);
    } else {
      for (int w = wave * (16 / p.waves); w < (wave + 1) * (16 / p.waves); ++w) f(lists + w * kWaveList, listed[w]);
    }
  };
  pieces([&](const int2* x, int count) {
    for (int k = lane; k < count; k += 64) atomicAdd(&counter[x[k].y * p.waves + wave], 1);
  });
  __syncthreads();
  // exclusive sums over the counters, a run of them for each lane
  const int each = (counters + 1023) / 1024, c0 = tid * each < counters ? tid * each : counters, c1 = c0 + each < counters ? c0 + each : counters;
  int sum = 0;
  for (int c = c0; c < c1; ++c) sum += counter[c];
  int upto = sum;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int x = __shfl_up(upto, s);
    upto += lane >= s ? x : 0;
  }
  if (lane == 63) scan[wave] = upto;
  __syncthreads();
  int place = before + upto - sum;
  for (int w = 0; w < wave; ++w) place += scan[w];
  for (int c = c0; c < c1; ++c) {
    const int x = counter[c];
    counter[c] = place;
    place += x;
  }
  __syncthreads();
  for (int b = tid; b < p.bins; b += 1024) {
    const int start = counter[b * p.waves], end = b + 1 < p.bins ? counter[(b + 1) * p.waves] : before + own;
    p.rows[bucket * p.bins + b] = make_int2(start, end - start);
  }
  __syncthreads();
  pieces([&](const int2* from, int count) {
    for (int k = 0; k < count; k += 64) {
      const bool there = k + lane < count;
      const int2 x = there ? from[k + lane] : make_int2(0, 0);
      uint64_t same = __ballot(there);   // lanes with this lane's word
      for (int bit = 1; bit < p.bins; bit <<= 1) {
        const uint64_t m = __ballot((x.y & bit) != 0);
        same &= x.y & bit ? m : ~m;
      }
      const int rank = lanes_below(same), first = there ? __ffsll((unsigned long long)same) - 1 : lane;
      int to = 0;
      if (there && first == lane) to = atomicAdd(&counter[x.y * p.waves + wave], __popcll(same));
      to = __shfl(to, first);
      if (there) p.order[to + rank] = x.x;
    }
  });
}

template <int E> __device__ __forceinline__ void embed_store(float* to, const float* x, float by, bool add) {
#pragma unroll
  for (int g = 0; g < E; g += 4) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[g + e] * by;
    if (add) v += *(const f32x4*)(to + g);
    *(f32x4*)(to + g) = v;
  }
}
template <int E> __device__ __forceinline__ void embed_store(bf16* to, const float* x, float by, bool add) {
  typedef bf16 vec __attribute__((ext_vector_type(E)));
  vec old{}, v;
  if (add) old = *(const vec*)to;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = (bf16)(x[e] * by + (float)old[e]);
  *(vec*)to = v;
}

__device__ __forceinline__ int2 embed_row(const EmbedParams& p, int64_t id) { return p.rows[(int)(id & (kBuckets - 1)) * p.bins + (int)(id >> kBucketBits)]; }

// Bound by HBM: 16384 tokens of 4096 channels and 128000 words, 1.18 GB read and written in 205 us; 23000 of 1024 channels into float, 176 MB in 34.
// The sums of a block of kEmbedBlock places of the grouped order over `across` lanes' columns; where nothing is added to, the work-groups behind
// p.grad_groups write the zeros of words without a token.
template <typename T, typename TD> __global__ __launch_bounds__(256) void embed_bwd_kernel(EmbedParams p, int across) {
  constexpr int E = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(E)));
  if ((int)blockIdx.x >= p.grad_groups) {
    const int64_t e0 = (int64_t)(blockIdx.x - p.grad_groups) * 32;
    const int chunks = p.d * (int)sizeof(TD) / 16, lane = threadIdx.x & 63;
    // (the counts of all 32 at once: one after another their loads took 10 us)
    const int64_t mine = e0 + (lane & 31);
    const int b = (int)(mine / p.bins);
    const int64_t id = ((mine - (int64_t)b * p.bins) << kBucketBits) + b;
    const bool empty = lane < 32 && mine < (int64_t)kBuckets * p.bins && id < p.v && p.rows[mine].y == 0;
    for (uint64_t left = __ballot(empty); left; left &= left - 1) {
      const int64_t word = __shfl(id, __ffsll((unsigned long long)left) - 1);
      for (int c = threadIdx.x; c < chunks; c += 256) *(u32x4*)((char*)p.dw + word * p.d * (int64_t)sizeof(TD) + (int64_t)c * 16) = u32x4{0, 0, 0, 0};
    }
    return;
  }
  const int total = *p.total;
  const int row_chunks = p.d / E, slices = (row_chunks + across - 1) / across;
  const int64_t unit = (int64_t)blockIdx.x * (256 / across) + threadIdx.x / across;
  const int block = (int)(unit / slices), chunk = (int)(unit - (int64_t)block * slices) * across + threadIdx.x % across;
  const int64_t start = (int64_t)block * kEmbedBlock;
  if (start >= total || chunk >= row_chunks) return;
  const int p0 = (int)start, p1 = total - p0 < kEmbedBlock ? total : p0 + kEmbedBlock;
  const int col = chunk * E;
  float sum[E];
  int64_t word = -1;
  int2 place = make_int2(0, 0);
  auto finish = [&]() {
    if (place.x >= p0 && place.x + place.y <= p1) embed_store<E>((TD*)p.dw + word * p.d + col, sum, p.scale, p.add != 0);
    else embed_store<E>(p.parts + ((int64_t)block * 2 + (place.x < p0 ? 0 : 1)) * p.d + col, sum, 1.f, false);
  };
  for (int q = p0; q < p1; q += 8) {
    int64_t id[8];
    int2 places[8];
    vec x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int token = p.order[q + k < p1 ? q + k : p1 - 1];
      id[k] = p.ids[token];
      x[k] = *(const vec*)((const T*)p.dy + (int64_t)token * p.ldy + col);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) places[k] = embed_row(p, id[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (q + k >= p1) break;
      if (id[k] != word) {
        if (word >= 0) finish();
        word = id[k];
        place = places[k];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = to_f32(x[k][e]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += to_f32(x[k][e]);
      }
    }
  }
  finish();
}

// The words that cross blocks: four waves add a quarter of the parts each, 256 columns a work-group.  (A launch has the units from `first` on:
// going over more of them in one work-group takes 14 us for 10.6 on 16384 tokens of 4096 channels.)
template <typename TD> __global__ __launch_bounds__(256) void embed_parts_kernel(EmbedParams p, uint32_t first) {
  __shared__ f32x4 quarter[3][64];
  const uint32_t slices = (p.d + 255) / 256, unit = first + blockIdx.x;
  const int block = unit / slices, slice = unit - block * slices;
  const int total = *p.total;
  const int64_t start = (int64_t)block * kEmbedBlock;
  if (start >= total) return;
  const int p0 = (int)start, p1 = total - p0 < kEmbedBlock ? total : p0 + kEmbedBlock;
  const int64_t word = p.ids[p.order[p1 - 1]];
  const int2 place = embed_row(p, word);
  if (place.x < p0 || place.x + place.y <= p1) return;   // (the same in all lanes)
  const int last = (place.x + place.y - 1) / kEmbedBlock, count = last - block + 1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = slice * 256 + lane * 4;
  const int each = (count + 3) / 4, from = wave * each < count ? wave * each : count, until = from + each < count ? from + each : count;
  f32x4 sum{};
  if (col < p.d) {
#pragma unroll 8
    for (int k = from; k < until; ++k) sum += *(const f32x4*)(p.parts + ((int64_t)(block + k) * 2 + (k == 0 ? 1 : 0)) * p.d + col);
  }
  if (wave) quarter[wave - 1][lane] = sum;
  __syncthreads();
  if (wave || col >= p.d) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) sum += quarter[w][lane];
  embed_store<4>((TD*)p.dw + word * p.d + col, (const float*)&sum, p.scale, p.add != 0);
}

}  // namespace acc
