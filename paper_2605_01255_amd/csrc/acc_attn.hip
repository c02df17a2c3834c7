// Host side of attention over packed documents.  Nothing is allocated and nothing synchronised: every entry point only enqueues on the
// caller's stream.
#include "acc_attn.h"

#include <math.h>

#include "acc_host.h"

namespace acc {
namespace {

// Work-groups of a kernel whose work-groups have `rows` rows of one of p.kv_heads * share heads.
struct AttnGrid {
  int tiles, strands, strand_tiles;
  int64_t groups;
};
AttnGrid attn_grid(const acc_attn_desc* d, int64_t seq, int64_t rows, int64_t share) {
  const int64_t tiles = d->docs ? d->n / rows + d->docs + 2 : ceil_div(d->n, seq) * ceil_div(seq, rows);
  int strands = 1;
  while (d->kv_heads * strands % 8) strands *= 2;
  const int64_t strand_tiles = ceil_div(tiles, strands), groups = d->kv_heads * strands * strand_tiles * share;
  return AttnGrid{(int)(tiles < INT32_MAX ? tiles : INT32_MAX), strands, (int)(strand_tiles < INT32_MAX ? strand_tiles : INT32_MAX), groups};
}

struct AttnPlan {
  AttnParams p;
  int waves, key_waves;                // of a work-group: over the queries; over the keys (their halves apart)
  AttnGrid queries, keys;
  int query_parts, key_parts;
  size_t stats, forward, minus, delta, part, backward;   // workspace
};

// Work-groups that fill the card: two of the queries' on a compute unit (float: four, of half the waves); of the keys' one, and more of them so
// that the last round is short.  (6001 rows with a window of 1000, dK and dV: 153 + 9 us, with half as many 193, with twice as many 165 + 15;
// one document of 8192 rows, 4 heads, O: 101 + 10, 167, 92 + 17.)
constexpr int64_t kFewGroups = 512, kFewKeyGroups = 640;

int plan_attn(const acc_attn_desc* d, AttnPlan* plan) {
  if (!d || (d->flags & ~(uint32_t)ACC_ATTN_CAUSAL)) return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(d->io_dtype)) return ACC_ERR_DTYPE;
  const bool causal = (d->flags & ACC_ATTN_CAUSAL) != 0;
  if (!(d->scale >= 0.f) || !(d->cap >= 0.f) || isinf(d->scale) || isinf(d->cap)) return ACC_ERR_INVALID_ARG;
  if (d->window < 0 || (d->window && !causal)) return ACC_ERR_INVALID_ARG;
  if (d->n <= 0 || d->n > 1 << 30 || d->heads <= 0 || d->heads > 1 << 15 || d->kv_heads <= 0 || d->heads % d->kv_heads) return ACC_ERR_SHAPE;
  if (d->d <= 0 || d->d > 128 || d->d % 8) return ACC_ERR_SHAPE;
  if (d->docs < 0 || d->docs > 1 << 28 || d->seq < 0 || (d->docs && d->seq)) return ACC_ERR_SHAPE;
  AttnParams& p = plan->p;
  p = AttnParams{};
  p.ldq = d->ldq ? d->ldq : d->heads * d->d;
  p.ldk = d->ldk ? d->ldk : d->kv_heads * d->d;
  p.ldv = d->ldv ? d->ldv : d->kv_heads * d->d;
  p.ldo = d->ldo ? d->ldo : d->heads * d->d;
  for (int64_t ld : {p.ldq, p.ldk, p.ldv, p.ldo})
    if (ld % 8 || ld > 1 << 18) return ACC_ERR_SHAPE;
  if (p.ldq < d->heads * d->d || p.ldo < d->heads * d->d || p.ldk < d->kv_heads * d->d || p.ldv < d->kv_heads * d->d) return ACC_ERR_SHAPE;
  const int64_t seq = d->seq && d->seq < d->n ? d->seq : d->n;
  p.n = (int)d->n;
  p.docs = (int)d->docs;
  p.seq = (int)seq;
  p.heads = (int)d->heads;
  p.kv_heads = (int)d->kv_heads;
  p.group = p.heads / p.kv_heads;
  p.d = (int)d->d;
  p.causal = causal;
  p.window = d->window > d->n ? 0 : (int)d->window;   // no row is that far away
  p.scale = d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->d);
  p.c2 = p.scale * kLog2e;
  p.cap2 = d->cap * kLog2e;
  p.inv_cap = d->cap > 0.f ? p.scale / d->cap : 0.f;
  if (!isfinite(p.c2) || !isfinite(2.f * p.cap2) || !isfinite(p.inv_cap * (2.f * kLog2e))) return ACC_ERR_INVALID_ARG;   // (a score of zero would be NaN)
  const bool b16 = d->io_dtype == ACC_BF16;
  const int64_t tile = b16 ? 64 : 32, length = d->docs ? ceil_div(d->n, d->docs) : seq;   // rows of a tile; of a document, on average
  const int64_t seen = d->window && d->window < length ? d->window : length;
  // Work-groups of 64 rows, not of 128, which share a tile's transfers among more waves:
  //   float, whose products take sixteen times as long as their rows' transfers;
  //   documents of up to 64 rows (8192 rows in 200 of them, 16 heads of 64 channels: forward and dQ 25 + 30 us, of 128 rows 30 + 50, both without delta's own pass);
  //   fewer than 128 of them with 128 rows (1024 rows, 8 heads of 128: 17 + 19 us and 7 to join parts, of 128 rows 16 + 21 and 11; 4096 rows, 32
  //   heads: 241 + 280 us, of 128 rows 170 + 206);
  //   for the keys' gradients heads of up to 64 channels, two work-groups of which fit a compute unit, so that one multiplies while the other
  //   waits (16 heads of 64, documents of 2048 rows: 199 us, of 128 rows 241; 32 heads of 128, 4096 rows: 355 us, of 128 rows 296).
  // (By the documents' average length: a long one among many short ones has the short ones' shape and no parts.  One of 4096 rows and 128 of 32
  // rows, 16 heads of 128 on 4: 590 us forward and backward, the two kinds in calls of their own 415 + 105.)
  const int64_t whole = d->heads * ceil_div(d->n, 128);
  plan->waves = b16 && length > 64 && whole >= 128 ? 4 : 2;
  plan->key_waves = b16 && length > 64 && whole >= 128 && d->d > 64 ? 4 : 2;
  // Parts: so many that the compute units are filled, of `least` tiles each at least.  A part is written and read as floats, which for the keys
  // takes the time of seven of its tiles.  (Three float documents of 344 rows, 8 heads: 160 us in all, without parts 305; 2048 rows, 16 heads on
  // 4 of 128 channels: dK and dV 56 + 8 us in 8 parts, 66 + 11 in 10, 190 in one; 40 documents of 51 rows: 14 us, in two parts 23 + 5.)
  auto parts_of = [&](int64_t groups, int64_t tiles, int64_t few, int64_t least) {
    int64_t parts = few / groups;
    if (parts > tiles / least) parts = tiles / least;
    if (parts > 16) parts = 16;
    return (int)(parts < 1 ? 1 : parts);
  };
  plan->query_parts = parts_of(d->heads * ceil_div(d->n, 32 * plan->waves), ceil_div(seen, tile), b16 ? kFewGroups : 2 * kFewGroups, b16 ? 4 : 2);
  plan->key_parts = parts_of(d->kv_heads * ceil_div(d->n, 32 * plan->key_waves), ceil_div(seen, tile) * p.group, kFewKeyGroups, b16 ? 16 : 2);
  plan->queries = attn_grid(d, seq, 32 * plan->waves, p.group * plan->query_parts);
  plan->keys = attn_grid(d, seq, 32 * plan->key_waves, plan->key_parts);
  const int64_t key_threads = plan->key_waves * (b16 ? 128 : 64);
  if (plan->queries.groups * plan->waves * 64 > UINT32_MAX || plan->keys.groups * key_threads > UINT32_MAX) return ACC_ERR_SHAPE;   // of a launch
  const int64_t query_floats = plan->query_parts > 1 ? (int64_t)plan->query_parts * d->n * d->heads * d->d : 0;
  const int64_t key_floats = plan->key_parts > 1 ? (int64_t)plan->key_parts * 2 * d->n * d->kv_heads * d->d : 0;
  plan->stats = (size_t)round_up(query_floats * 4, 256);
  plan->forward = plan->stats + (plan->query_parts > 1 ? (size_t)plan->query_parts * 2 * d->heads * d->n * 4 : 0);
  plan->minus = 0;
  plan->delta = (size_t)round_up(d->heads * d->n * 4, 256);
  plan->part = 2 * plan->delta;   // of the queries' gradient, then of the keys'
  plan->backward = plan->part + (size_t)(query_floats > key_floats ? query_floats : key_floats) * 4;
  if (plan->backward < plan->forward) plan->backward = plan->forward;
  return ACC_OK;
}

int check_masks(const acc_attn_desc* d, const int64_t* starts, const int64_t* prefix, const float* slopes) {
  if ((d->docs != 0) != (starts != nullptr)) return ACC_ERR_INVALID_ARG;
  if (prefix && (!(d->flags & ACC_ATTN_CAUSAL) || d->window)) return ACC_ERR_INVALID_ARG;
  return aligned16(starts) && aligned16(prefix) && aligned16(slopes) ? ACC_OK : ACC_ERR_ALIGN;
}

// f(a value of the element type, blocks of 32 channels as a constant)
template <typename F> void with_attn(const acc_attn_desc* d, F&& f) {
  using std::integral_constant;
  auto typed = [&](auto value) {
    if (d->d <= 64) f(value, integral_constant<int, 2>{});
    else if (d->d <= 96) f(value, integral_constant<int, 3>{});
    else f(value, integral_constant<int, 4>{});
  };
  if (d->io_dtype == ACC_BF16) typed(bf16{});
  else typed(float{});
}

// f(waves as a constant); float has two.
template <typename T, typename F> void with_waves(int waves, F&& f) {
  if constexpr (sizeof(T) == 2) {
    if (waves == 4) return f(std::integral_constant<int, 4>{});
  }
  f(std::integral_constant<int, 2>{});
}

void on_grid(AttnParams& p, const AttnGrid& g, int parts) {
  p.parts = parts;
  p.tiles = g.tiles;
  p.strands = g.strands;
  p.strand_tiles = g.strand_tiles;
}

}  // namespace
}  // namespace acc

using namespace acc;

extern "C" {

size_t acc_attn_workspace_bytes(const acc_attn_desc* desc, int is_backward) {
  AttnPlan plan;
  if (plan_attn(desc, &plan) != ACC_OK) return 0;
  return is_backward ? plan.backward : plan.forward;
}

int acc_attn_fwd(const acc_attn_desc* desc, const void* Q, const void* K, const void* V, const int64_t* starts, const int64_t* prefix,
                 const float* slopes, void* O, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  AttnPlan plan;
  int rc = plan_attn(desc, &plan);
  if (rc != ACC_OK) return rc;
  if (!Q || !K || !V || !O || !lse) return ACC_ERR_INVALID_ARG;
  if ((rc = check_masks(desc, starts, prefix, slopes)) != ACC_OK) return rc;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(lse) || !aligned16(workspace)) return ACC_ERR_ALIGN;
  if (plan.forward && (!workspace || ws_bytes < plan.forward)) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  AttnParams p = plan.p;
  p.q = Q; p.k = K; p.v = V; p.o = O; p.lse = lse;
  p.part = (float*)workspace;
  p.part_stats = (float*)((char*)workspace + plan.stats);
  p.starts = starts; p.prefix = prefix; p.slopes = slopes;
  auto quads = [&](int heads) { return dim3((unsigned)ceil_div((int64_t)p.n * heads * p.d / 4, 256)); };
  with_attn(desc, [&](auto value, auto db) {
    using T = decltype(value);
    constexpr int DB = decltype(db)::value;
    on_grid(p, plan.queries, plan.query_parts);
    with_waves<T>(plan.waves, [&](auto nw) {
      constexpr int NW = decltype(nw)::value;
      L.launch_lds(attn_fwd_kernel<T, DB, NW>, dim3((unsigned)plan.queries.groups), dim3(NW * 64), (size_t)4 * Tile32<T, DB>::BYTES, p);
    });
    if (p.parts > 1) L(attn_join_kernel<T>, quads(p.heads), dim3(256), p);
  });
  return L.status();
}

int acc_attn_bwd(const acc_attn_desc* desc, const void* Q, const void* K, const void* V, const int64_t* starts, const int64_t* prefix,
                 const float* slopes, const void* O, const float* lse, const void* dO, void* dQ, void* dK, void* dV, void* workspace,
                 size_t ws_bytes, void* stream) {
  AttnPlan plan;
  int rc = plan_attn(desc, &plan);
  if (rc != ACC_OK) return rc;
  if (!Q || !K || !V || !O || !lse || !dO || !dQ || !dK || !dV) return ACC_ERR_INVALID_ARG;
  if ((rc = check_masks(desc, starts, prefix, slopes)) != ACC_OK) return rc;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(lse) || !aligned16(dO) || !aligned16(dQ) || !aligned16(dK) ||
      !aligned16(dV) || !aligned16(workspace))
    return ACC_ERR_ALIGN;
  if (!workspace || ws_bytes < plan.backward) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  AttnParams p = plan.p;
  p.q = Q; p.k = K; p.v = V; p.o_in = O; p.lse = const_cast<float*>(lse); p.dout = dO;
  p.dq = dQ; p.dk = dK; p.dv = dV;
  p.minus = (float*)((char*)workspace + plan.minus);
  p.delta = (float*)((char*)workspace + plan.delta);
  p.part = (float*)((char*)workspace + plan.part);
  p.starts = starts; p.prefix = prefix; p.slopes = slopes;
  auto quads = [&](int heads) { return dim3((unsigned)ceil_div((int64_t)p.n * heads * p.d / 4, 256)); };
  with_attn(desc, [&](auto value, auto db) {
    using T = decltype(value);
    constexpr int DB = decltype(db)::value;
    on_grid(p, plan.queries, plan.query_parts);
    with_waves<T>(plan.waves, [&](auto nw) {
      constexpr int NW = decltype(nw)::value;
      L.launch_lds(attn_dq_kernel<T, DB, NW>, dim3((unsigned)plan.queries.groups), dim3(NW * 64), (size_t)4 * Tile32<T, DB>::BYTES, p);
    });
    if (p.parts > 1) L(attn_parts_kernel<T>, quads(p.heads), dim3(256), p.part, p.parts, (int64_t)p.n, p.heads * p.d, (T*)dQ, p.ldq, (T*)nullptr, (int64_t)0);
    on_grid(p, plan.keys, plan.key_parts);
    with_waves<T>(plan.key_waves, [&](auto nw) {
      constexpr int KW = decltype(nw)::value;
      using Layout = DkvLayout<T, DB, KW>;
      L.launch_lds(attn_dkv_kernel<T, DB, KW>, dim3((unsigned)plan.keys.groups), dim3(Layout::NW * 64), (size_t)Layout::BYTES, p);
    });
    if (p.parts > 1) L(attn_parts_kernel<T>, quads(2 * p.kv_heads), dim3(256), p.part, p.parts, (int64_t)p.n, p.kv_heads * p.d, (T*)dK, p.ldk, (T*)dV, p.ldv);
  });
  return L.status();
}

}  // extern "C"
