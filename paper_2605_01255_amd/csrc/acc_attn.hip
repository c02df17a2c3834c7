// Host side of attention over packed documents.  Nothing is allocated and nothing synchronised: every entry point only enqueues on the
// caller's stream.
#include "acc_attn.h"

#include <math.h>

#include "acc_host.h"

namespace acc {
namespace {

constexpr int kWaves = 4;   // of a work-group

struct AttnPlan {
  AttnParams p;
  int64_t groups, kv_groups;   // work-groups over the queries, over the keys
  size_t delta, backward;      // workspace
};

int64_t attn_tiles(const acc_attn_desc* d, int64_t seq, int64_t rows) {
  if (d->docs) return d->n / rows + d->docs + 2;
  return ceil_div(d->n, seq) * ceil_div(seq, rows);
}

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
  const int64_t tiles = attn_tiles(d, seq, 32 * kWaves);
  plan->groups = round_up(d->heads * tiles, 8);
  plan->kv_groups = round_up(d->kv_heads * tiles, 8);
  if (plan->groups >= 1 << 24) return ACC_ERR_SHAPE;
  p.n = (int)d->n;
  p.docs = (int)d->docs;
  p.seq = (int)seq;
  p.heads = (int)d->heads;
  p.kv_heads = (int)d->kv_heads;
  p.group = p.heads / p.kv_heads;
  p.d = (int)d->d;
  p.tiles = (int)tiles;
  p.causal = causal;
  p.window = d->window > d->n ? 0 : (int)d->window;   // no row is that far away
  p.scale = d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->d);
  p.c2 = p.scale * kLog2e;
  p.cap2 = d->cap * kLog2e;
  p.inv_cap = d->cap > 0.f ? p.scale / d->cap : 0.f;
  plan->delta = 0;
  plan->backward = (size_t)round_up(d->heads * d->n * 4, 256);
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

}  // namespace
}  // namespace acc

using namespace acc;

extern "C" {

size_t acc_attn_workspace_bytes(const acc_attn_desc* desc, int is_backward) {
  AttnPlan plan;
  if (plan_attn(desc, &plan) != ACC_OK || !is_backward) return 0;
  return plan.backward;
}

int acc_attn_fwd(const acc_attn_desc* desc, const void* Q, const void* K, const void* V, const int64_t* starts, const int64_t* prefix,
                 const float* slopes, void* O, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  AttnPlan plan;
  int rc = plan_attn(desc, &plan);
  if (rc != ACC_OK) return rc;
  if (!Q || !K || !V || !O || !lse) return ACC_ERR_INVALID_ARG;
  if ((rc = check_masks(desc, starts, prefix, slopes)) != ACC_OK) return rc;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(lse) || !aligned16(workspace)) return ACC_ERR_ALIGN;
  (void)ws_bytes;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  AttnParams p = plan.p;
  p.q = Q; p.k = K; p.v = V; p.o = O; p.lse = lse;
  p.starts = starts; p.prefix = prefix; p.slopes = slopes;
  with_attn(desc, [&](auto value, auto db) {
    using T = decltype(value);
    constexpr int DB = decltype(db)::value;
    L.launch_lds(attn_fwd_kernel<T, DB, kWaves>, dim3((unsigned)plan.groups), dim3(kWaves * 64), (size_t)4 * Tile32<T, DB>::BYTES, p);
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
  p.delta = (float*)((char*)workspace + plan.delta);
  p.starts = starts; p.prefix = prefix; p.slopes = slopes;
  with_attn(desc, [&](auto value, auto db) {
    using T = decltype(value);
    constexpr int DB = decltype(db)::value;
    const size_t lds = 4 * Tile32<T, DB>::BYTES;
    L.launch_lds(attn_dq_kernel<T, DB, kWaves>, dim3((unsigned)plan.groups), dim3(kWaves * 64), lds, p);
    L.launch_lds(attn_dkv_kernel<T, DB>, dim3((unsigned)plan.kv_groups), dim3(DkvLayout<T, DB>::NW * 64), (size_t)DkvLayout<T, DB>::BYTES, p);
  });
  return L.status();
}

}  // extern "C"
