// Host side of what a training step has around its layers: the vocabulary's table, the gradients' norm and scaling.  Nothing is allocated and
// nothing synchronised: every entry point only enqueues on the caller's stream.
#include <math.h>

#include "acc_embed.h"
#include "acc_grads.h"
#include "acc_host.h"

namespace acc {
namespace {

// ---- the vocabulary's table ----------------------------------------------------------------------------
struct EmbedPlan {
  EmbedParams p;
  int per, across;              // rows of a forward work-group; lanes along a row in the backward one
  int64_t blocks, slices;       // of the grouped order, of a row
  int64_t zero_groups, part_groups;
  size_t order, rows, list, total, parts, bytes;
};

int plan_embed(const acc_embed_desc* d, EmbedPlan* plan) {
  if (!d || (d->flags & ~(uint32_t)ACC_FLAG_DW_ACCUMULATE) || d->reserved || !isfinite(d->scale)) return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(d->io_dtype) || !valid_dtype(d->dw_dtype)) return ACC_ERR_DTYPE;
  if (d->n <= 0 || d->n > 1 << 30 || d->d <= 0 || d->d % 8 || d->d > 1 << 16 || d->v <= 0 || d->v > 1 << 21) return ACC_ERR_SHAPE;
  EmbedParams& p = plan->p;
  p = EmbedParams{};
  p.n = d->n;
  p.v = d->v;
  p.d = (int)d->d;
  p.ldw = d->ldw ? d->ldw : d->d;
  p.ldy = d->ldy ? d->ldy : d->d;
  for (int64_t ld : {p.ldw, p.ldy})
    if (ld < d->d || ld % 8 || ld > 1 << 18) return ACC_ERR_SHAPE;
  p.scale = d->scale;
  p.add = (d->flags & ACC_FLAG_DW_ACCUMULATE) != 0;
  const int64_t row_chunks = d->d * (int64_t)dtype_size(d->io_dtype) / 16;
  plan->per = row_chunks >= 1024 ? 1 : (int)(1024 / row_chunks);
  int across = 1;
  while (across < 256 && across < row_chunks) across *= 2;
  plan->across = across;
  plan->blocks = ceil_div(d->n, kEmbedBlock);
  plan->slices = ceil_div(row_chunks, across);
  p.grad_groups = (int)ceil_div(plan->blocks * plan->slices, 256 / across);
  p.bins = (int)ceil_div(d->v, kBuckets);
  int waves = 16;
  while (waves * p.bins > kEmbedCounters) waves /= 2;
  p.waves = waves;
  plan->zero_groups = p.add ? 0 : ceil_div((int64_t)kBuckets * p.bins, 32);
  plan->part_groups = plan->blocks * ceil_div(d->d, 256);
  if (ceil_div(d->n, plan->per) >= 1 << 24 || plan->blocks * plan->slices >= 1 << 30 || p.grad_groups + plan->zero_groups >= 1 << 24) return ACC_ERR_SHAPE;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t from = at;
    at += (size_t)round_up(bytes, 256);
    return from;
  };
  plan->order = take(d->n * 4);
  plan->rows = take((int64_t)kBuckets * p.bins * 8);
  plan->list = take(d->n * 8);
  plan->total = take(4);
  plan->parts = take(plan->blocks * 2 * d->d * 4);
  plan->bytes = at;
  return ACC_OK;
}

// ---- the gradients' norm -------------------------------------------------------------------------------
int64_t grad_groups(int64_t count) { return ceil_div(count, kGradChunk); }

int check_tensors(const acc_grad_tensor* t, int64_t count, bool scaled, int64_t* groups) {
  *groups = 0;
  if (count < 0 || count > 1 << 24 || (count && !t)) return ACC_ERR_INVALID_ARG;
  for (int64_t i = 0; i < count; ++i) {
    if (!valid_dtype(t[i].dtype) || (scaled && !valid_dtype(t[i].dst_dtype))) return ACC_ERR_DTYPE;
    if (t[i].count < 0 || t[i].count > (int64_t)1 << 39) return ACC_ERR_SHAPE;
    if (!t[i].count) continue;   // wherever it points
    if (!t[i].src || (scaled && !t[i].dst)) return ACC_ERR_INVALID_ARG;
    if ((uintptr_t)t[i].src % dtype_size(t[i].dtype) || (scaled && (uintptr_t)t[i].dst % dtype_size(t[i].dst_dtype))) return ACC_ERR_ALIGN;
    if (scaled && t[i].src == t[i].dst && t[i].dtype != t[i].dst_dtype) return ACC_ERR_INVALID_ARG;
    *groups += grad_groups(t[i].count);
  }
  return ACC_OK;
}

// f(a table, its work-groups) over all tensors that have elements, in tables of kGradTensors.
template <typename F> void grad_tables(const acc_grad_tensor* t, int64_t count, F&& f) {
  GradList g{};
  int64_t groups = 0;
  auto flush = [&]() {
    if (!g.tensors) return;
    g.first[g.tensors] = (uint32_t)groups;
    f(g, groups);
    g = GradList{};
    groups = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    const int64_t more = grad_groups(t[i].count);
    if (!more) continue;
    if (g.tensors == kGradTensors || groups + more >= 1 << 24) flush();
    const int k = g.tensors++;
    g.src[k] = t[i].src;
    g.dst[k] = t[i].dst;
    g.count[k] = t[i].count;
    g.first[k] = (uint32_t)groups;
    g.src_b16[k] = t[i].dtype == ACC_BF16;
    g.dst_b16[k] = t[i].dst_dtype == ACC_BF16;
    groups += more;
  }
  flush();
}

int check_factors(const acc_grad_factors* f, int64_t count) {
  if (count < 0 || count > 1 << 24 || (count && !f)) return ACC_ERR_INVALID_ARG;
  for (int64_t i = 0; i < count; ++i) {
    const acc_grad_factors& x = f[i];
    if (x.flags & ~(uint32_t)ACC_FLAG_W_OUT_IN) return ACC_ERR_INVALID_ARG;
    if (!valid_dtype(x.dtype)) return ACC_ERR_DTYPE;
    if (x.d_in <= 0 || x.d_out <= 0 || x.r <= 0 || x.d_in % 8 || x.d_out % 8 || x.r % 8 || x.d_in > 1 << 21 || x.d_out > 1 << 21 || x.r > 1 << 13)
      return ACC_ERR_SHAPE;
    const int64_t g_row = x.flags & ACC_FLAG_W_OUT_IN ? x.r : x.d_out;
    if ((x.ldl && (x.ldl < x.r || x.ldl % 8 || x.ldl > 1 << 22)) || (x.ldg && (x.ldg < g_row || x.ldg % 8 || x.ldg > 1 << 22))) return ACC_ERR_SHAPE;
    if (!x.left || !x.gr) return ACC_ERR_INVALID_ARG;
    if (!aligned16(x.left) || !aligned16(x.gr)) return ACC_ERR_ALIGN;
  }
  return ACC_OK;
}

struct GramBatch {
  GramSumList l;
  int64_t groups, sums;   // work-groups of both kernels
  int64_t floats;         // of the parts
};

// f(a batch, its dtype) over all pairs, those of one dtype after those of the other.
template <typename F> void gram_batches(const acc_grad_factors* f, int64_t count, F&& each) {
  for (int32_t dtype : {(int32_t)ACC_BF16, (int32_t)ACC_F32}) {
    GramBatch b{};
    auto flush = [&]() {
      if (b.l.pairs) each(b, dtype);
      b = GramBatch{};
    };
    for (int64_t i = 0; i < count; ++i) {
      const acc_grad_factors& x = f[i];
      if (x.dtype != dtype) continue;
      const int64_t n_tiles = ceil_div(x.r, kGramTile), tiles = n_tiles * (n_tiles + 1) / 2;
      const int64_t groups = tiles * (ceil_div(x.d_in, kGramRows) + ceil_div(x.d_out, kGramRows));
      if (b.l.pairs == kGradFactors || b.groups + groups >= 1 << 24) flush();
      const bool oi = (x.flags & ACC_FLAG_W_OUT_IN) != 0;
      for (int s = 0; s < 2; ++s) {
        GramSide& side = b.l.g.side[2 * b.l.pairs + s];
        side.x = s ? x.gr : x.left;
        side.rows = s ? x.d_out : x.d_in;
        side.r = (int)x.r;
        side.wide = s && !oi;
        side.ld = s ? (x.ldg ? x.ldg : oi ? x.r : x.d_out) : x.ldl ? x.ldl : x.r;
        side.first = (uint32_t)b.groups;
        side.splits = (uint32_t)ceil_div(side.rows, kGramRows);
        side.parts = b.floats;
        b.groups += tiles * side.splits;
        b.floats += tiles * side.splits * kGramTile * kGramTile;
      }
      b.l.first[b.l.pairs++] = (uint32_t)b.sums;
      b.l.g.sides = 2 * b.l.pairs;
      b.sums += tiles * 8;
    }
    flush();
  }
}

struct NormPlan {
  int64_t partials;        // doubles
  size_t parts, bytes;
};
int plan_norm(const acc_grad_tensor* t, int64_t count, const acc_grad_factors* f, int64_t pairs, NormPlan* plan) {
  int64_t groups;
  int rc = check_tensors(t, count, false, &groups);
  if (rc == ACC_OK) rc = check_factors(f, pairs);
  if (rc != ACC_OK) return rc;
  int64_t floats = 0;
  gram_batches(f, pairs, [&](const GramBatch& b, int32_t) {
    groups += b.sums;
    if (b.floats > floats) floats = b.floats;
  });
  plan->partials = groups;
  plan->parts = (size_t)round_up(groups * 8 + 8, 256);
  plan->bytes = plan->parts + (size_t)floats * 4;
  return ACC_OK;
}

}  // namespace
}  // namespace acc

using namespace acc;

extern "C" {

size_t acc_embed_workspace_bytes(const acc_embed_desc* desc) {
  EmbedPlan plan;
  return plan_embed(desc, &plan) == ACC_OK ? plan.bytes : 0;
}

int acc_embed_fwd(const acc_embed_desc* desc, const void* W, const int64_t* ids, void* Y, void* stream) {
  EmbedPlan plan;
  int rc = plan_embed(desc, &plan);
  if (rc != ACC_OK) return rc;
  if (!W || !ids || !Y) return ACC_ERR_INVALID_ARG;
  if (!aligned16(W) || !aligned16(ids) || !aligned16(Y)) return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  EmbedParams p = plan.p;
  p.w = W; p.ids = ids; p.y = Y;
  const dim3 grid((unsigned)ceil_div(p.n, plan.per));
  if (desc->io_dtype == ACC_BF16) L(embed_fwd_kernel<bf16>, grid, dim3(256), p, plan.per);
  else L(embed_fwd_kernel<float>, grid, dim3(256), p, plan.per);
  return L.status();
}

int acc_embed_bwd(const acc_embed_desc* desc, const int64_t* ids, const void* dY, void* dW, void* workspace, size_t ws_bytes, void* stream) {
  EmbedPlan plan;
  int rc = plan_embed(desc, &plan);
  if (rc != ACC_OK) return rc;
  if (!ids || !dY || !dW) return ACC_ERR_INVALID_ARG;
  if (!aligned16(ids) || !aligned16(dY) || !aligned16(dW) || !aligned16(workspace)) return ACC_ERR_ALIGN;
  if (!workspace || ws_bytes < plan.bytes) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  char* ws = (char*)workspace;
  EmbedParams p = plan.p;
  p.ids = ids; p.dy = dY; p.dw = dW;
  p.order = (int*)(ws + plan.order);
  p.rows = (int2*)(ws + plan.rows);
  p.list = (int2*)(ws + plan.list);
  p.total = (int*)(ws + plan.total);
  p.parts = (float*)(ws + plan.parts);
  L.launch_lds(embed_group_kernel, dim3(kBuckets), dim3(1024), (size_t)round_up(p.bins * p.waves * 4, 8) + 16 * kWaveList * 8, p);
  const dim3 sums((unsigned)(p.grad_groups + plan.zero_groups));
  const int64_t most = 1 << 23;   // parts of a launch
  auto typed = [&](auto value, auto grad) {
    using T = decltype(value);
    using TD = decltype(grad);
    L(embed_bwd_kernel<T, TD>, sums, dim3(256), p, plan.across);
    for (int64_t at = 0; at < plan.part_groups; at += most)
      L(embed_parts_kernel<TD>, dim3((unsigned)(plan.part_groups - at < most ? plan.part_groups - at : most)), dim3(256), p, (uint32_t)at);
  };
  auto of = [&](auto value) { desc->dw_dtype == ACC_BF16 ? typed(value, bf16{}) : typed(value, float{}); };
  if (desc->io_dtype == ACC_BF16) of(bf16{});
  else of(float{});
  return L.status();
}

size_t acc_grad_norm_workspace_bytes(const acc_grad_tensor* tensors, int64_t count, const acc_grad_factors* factors, int64_t pairs) {
  NormPlan plan;
  return plan_norm(tensors, count, factors, pairs, &plan) == ACC_OK ? plan.bytes : 0;
}

int acc_grad_norm(const acc_grad_tensor* tensors, int64_t count, const acc_grad_factors* factors, int64_t pairs, float max_norm, float* out,
                  void* workspace, size_t ws_bytes, void* stream) {
  NormPlan plan;
  int rc = plan_norm(tensors, count, factors, pairs, &plan);
  if (rc != ACC_OK) return rc;
  if (!out || !(max_norm >= 0.f)) return ACC_ERR_INVALID_ARG;
  if ((uintptr_t)out % 4 || !aligned16(workspace)) return ACC_ERR_ALIGN;
  if (!workspace || ws_bytes < plan.bytes) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  double* partial = (double*)workspace;
  float* parts = (float*)((char*)workspace + plan.parts);
  grad_tables(tensors, count, [&](const GradList& g, int64_t groups) {
    L(grad_squares_kernel, dim3((unsigned)groups), dim3(256), g, partial);
    partial += groups;
  });
  gram_batches(factors, pairs, [&](GramBatch& b, int32_t dtype) {
    b.l.g.parts = parts;
    const dim3 grid((unsigned)b.groups);
    if (dtype == ACC_BF16) L.launch_lds(gram_kernel<bf16>, grid, dim3(256), (size_t)4 * Tile32<bf16, 4>::BYTES, b.l.g);
    else L.launch_lds(gram_kernel<float>, grid, dim3(256), (size_t)8 * Tile32<float, 4>::BYTES, b.l.g);
    L(gram_sum_kernel, dim3((unsigned)b.sums), dim3(256), b.l, partial);
    partial += b.sums;
  });
  L(grad_norm_kernel, dim3(1), dim3(256), (const double*)workspace, plan.partials, max_norm, out);
  return L.status();
}

int acc_grad_scale(const acc_grad_tensor* tensors, int64_t count, const float* factor, void* stream) {
  int64_t groups;
  int rc = check_tensors(tensors, count, true, &groups);
  if (rc != ACC_OK) return rc;
  if (!factor) return ACC_ERR_INVALID_ARG;
  if ((uintptr_t)factor % 4) return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  grad_tables(tensors, count, [&](const GradList& g, int64_t groups) { L(grad_scale_kernel, dim3((unsigned)groups), dim3(256), g, factor); });
  return L.status();
}

}  // extern "C"
