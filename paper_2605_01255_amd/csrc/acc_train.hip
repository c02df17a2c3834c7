// Host side of the operators beside the compressed linear layer: 8-bit checkpoints of activations and what reads them.
// As in acc_api.hip nothing is allocated and nothing synchronised: every entry point only enqueues on the caller's stream.
#include "acc_act8.h"
#include "acc_ce.h"
#include "acc_gemm16.h"
#include "acc_gemm_ring.h"
#include "acc_host.h"

namespace acc {
namespace {

// ---- 8-bit checkpoints ------------------------------------------------------------------------------
bool valid_format(int32_t f) { return f == ACC_ACT8_E4M3 || f == ACC_ACT8_INT8; }

// Sizes and strides that the 8-bit calls share: rows of `c` elements, `ld` apart (0: dense), in a grid of less than 2^32 lanes.
int validate_rows(int64_t n, int64_t c, int64_t* ld) {
  if (n <= 0 || n > (int64_t)1 << 30 || c <= 0 || c > (1 << 21) || c % 8 || act_work_groups(n, c) >= 1 << 24) return ACC_ERR_SHAPE;
  if (!*ld) *ld = c;
  return *ld < c || *ld % 8 || *ld > ((int64_t)1 << 24) ? ACC_ERR_SHAPE : ACC_OK;
}

// f(a value of the element type, the format as a constant)
template <typename F> void with_act8(int32_t dtype, int32_t format, F&& f) {
  auto typed = [&](auto value) {
    if (format == ACC_ACT8_E4M3) f(value, std::integral_constant<int, ACC_ACT8_E4M3>{});
    else f(value, std::integral_constant<int, ACC_ACT8_INT8>{});
  };
  if (dtype == ACC_BF16) typed(bf16{});
  else typed(float{});
}

void act8_pack(int32_t dtype, int32_t format, const void* X, int64_t n, int64_t c, int64_t ld, void* Q, void* E, Launcher& L) {
  with_act8(dtype, format, [&](auto value, auto fmt) {
    using T = decltype(value);
    L(act8_pack_kernel<T, decltype(fmt)::value>, dim3((unsigned)act_work_groups(n, c)), dim3(256), (const T*)X, n, c, ld, (uint8_t*)Q, (uint8_t*)E);
  });
}

void act8_unpack(int32_t dtype, int32_t format, const void* Q, const void* E, int64_t n, int64_t c, int64_t ld, void* X, Launcher& L) {
  with_act8(dtype, format, [&](auto value, auto fmt) {
    using T = decltype(value);
    L(act8_unpack_kernel<T, decltype(fmt)::value>, dim3((unsigned)act_work_groups(n, c)), dim3(256), (const uint8_t*)Q, (const uint8_t*)E, n, c, ld, (T*)X);
  });
}

// ---- products over the tokens -------------------------------------------------------------------------
// C[M, N] (op)= At^T . B with At [K, M] and B [K, N]: both operands of the ring kernel by transposing reads.
template <int TM, int TN, int NS, typename TC, int SPLIT, bool SUM>
void ring_token_gemm(FastGemmParams& p, Launcher& L) {
  const unsigned grid = gemm_ring_plan(p, 32 * TM, 32 * TN);
  const int64_t splits = SPLIT ? ceil_div(p.K, p.k_per_split) : 1;
  p.tile_blocks = (int)grid;
  L.launch_lds(gemm_ring_kernel<TM, TN, NS, false, TC, SPLIT, SUM, false>, dim3(grid * (unsigned)splits), dim3(256),
               (size_t)gemm_ring_lds_bytes<TM, TN, NS>(), p);
}

// f(the tile's 16 x 16 blocks in both directions and its stages as constants): three stages where a compute unit has one work-group.
// 192 x 128 is the largest that pick_split_gemm has for this kernel.
template <typename F> void with_ring_tile(GemmTile tile, bool one_round, F&& f) {
  using std::integral_constant;
  switch (tile) {
    default: return one_round ? f(integral_constant<int, 6>{}, integral_constant<int, 4>{}, integral_constant<int, 3>{})
                              : f(integral_constant<int, 6>{}, integral_constant<int, 4>{}, integral_constant<int, 2>{});
    case GemmTile::k128: return one_round ? f(integral_constant<int, 4>{}, integral_constant<int, 4>{}, integral_constant<int, 3>{})
                                          : f(integral_constant<int, 4>{}, integral_constant<int, 4>{}, integral_constant<int, 2>{});
    case GemmTile::k128x64: return f(integral_constant<int, 4>{}, integral_constant<int, 2>{}, integral_constant<int, 3>{});
    case GemmTile::k64: return f(integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 3>{});
  }
}

// The form of a bfloat16 product over K tokens; the persistent kernel takes three K tiles and stores bfloat16.
SplitChoice plan_token_gemm(int64_t M, int64_t N, int64_t K, int64_t most_splits, bool bf16_c, bool sum) {
  return pick_split_gemm(M, N, K, most_splits, true, bf16_c && !sum && K > 128);
}
constexpr int64_t kTokenParts = 64;
// Bytes of the parts of a product over K tokens.
size_t token_parts_bytes(int32_t io, int32_t dtype, bool sum, int64_t M, int64_t N, int64_t K) {
  if (io != ACC_BF16) return 0;
  const SplitChoice c = plan_token_gemm(M, N, K, kTokenParts, dtype == ACC_BF16, sum);
  return c.splits > 1 ? (size_t)c.splits * M * N * sizeof(float) : 0;
}

template <typename TC, bool SUM>
void token_gemm(const void* A, const void* B, void* C, int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldb, int64_t ldc, Launcher& L,
                float* parts, const int* live, const float* scale, int least_rows) {
  FastGemmParams p = fast_params(A, B, C, M, N, K, lda, ldb, ldc, nullptr, 1.f, 1.f);
  p.live = live;
  p.scale = scale;
  p.least_rows = least_rows;
  const SplitChoice plan = plan_token_gemm(M, N, K, parts ? kTokenParts : 1, sizeof(TC) == 2, SUM);
  if (plan.splits > 1) {
    p.C = parts;
    p.ldc = N;
    p.k_per_split = plan.k_per_split;
    p.c_split_stride = M * N;
    with_ring_tile(plan.tile, plan.one_round, [&](auto tm, auto tn, auto ns) {
      ring_token_gemm<decltype(tm)::value, decltype(tn)::value, decltype(ns)::value, float, kPlain, false>(p, L);
    });
    L(add_parts_kernel<TC, SUM>, dim3((unsigned)ceil_div(M * N, 1024)), dim3(256), (const float*)parts, (int)plan.splits, M * N, N, ldc, (TC*)C);
    return;
  }
  if constexpr (sizeof(TC) == 2 && !SUM) {
    if (plan.tile == GemmTile::k256) {
      const unsigned slots = gemm_bf16_plan(p, 256, 256);
      L.launch_lds(gemm16_persist_kernel<false, true, false>, dim3(256), dim3(256), (size_t)160 * 1024, p, (int)slots);
      return;
    }
  }
  with_ring_tile(plan.tile, plan.one_round, [&](auto tm, auto tn, auto ns) {
    ring_token_gemm<decltype(tm)::value, decltype(tn)::value, decltype(ns)::value, TC, kNone, SUM>(p, L);
  });
}

// C[M, N] (op)= At^T . B, operands of `io`, C of `dtype`; rows of At and B 16-byte aligned and below 4 GiB in all.  parts: room of
// token_parts_bytes, or null: not in parts.  live: device count of the rows of both that take part, at most K; in bfloat16 least_rows of
// them are read at least, and in float32 what is behind them holds zeros.  scale (bfloat16): device factor.
void token_product(int32_t io, int32_t dtype, const void* A, int64_t lda, const void* B, int64_t ldb, void* C, int64_t ldc, int64_t M,
                   int64_t N, int64_t K, bool accumulate, Launcher& L, float* parts, const int* live = nullptr, const float* scale = nullptr,
                   int least_rows = 0) {
  if (io == ACC_BF16) {
    auto typed = [&](auto type) {
      using TC = decltype(type);
      if (accumulate) token_gemm<TC, true>(A, B, C, M, N, K, lda, ldb, ldc, L, parts, live, scale, least_rows);
      else token_gemm<TC, false>(A, B, C, M, N, K, lda, ldb, ldc, L, parts, live, scale, least_rows);
    };
    if (dtype == ACC_BF16) typed(bf16{});
    else typed(float{});
    return;
  }
  f32_product(F32Operand{A, lda, false, false}, F32Operand{B, ldb, false, false}, C, dtype, ldc, M, N, K, accumulate, L, false, live);
}

// Tokens of one such product: a buffer resource has to reach over the wider operand, whole K tiles of 64 tokens (so whole blocks too)
// included.  0: not even over one.
int64_t token_chunk(int64_t n, int64_t ld, int32_t io) {
  const int64_t most = kMaxOperandBytes / (ld * (int64_t)dtype_size(io)) / 64 * 64;
  return n <= most ? n : most;
}

// The checkpoint's values, then the parts of the product with them.  total == 0: rows too far apart, or too many.
struct Act8Plan {
  int64_t tokens;   // of one product
  size_t parts, total;
};
Act8Plan plan_act8(const acc_linear_desc* d, const Shape& s) {
  Act8Plan p{};
  p.tokens = token_chunk(s.n, s.ldy > s.d_in ? s.ldy : s.d_in, d->io_dtype);
  if (p.tokens == 0 || act_work_groups(s.n, s.d_in) >= 1 << 24) return p;
  p.parts = (size_t)round_up(p.tokens * s.d_in * (int64_t)dtype_size(d->io_dtype), 256);
  const bool w_oi = (d->flags & ACC_FLAG_W_OUT_IN) != 0;
  const int64_t M = w_oi ? s.d_out : s.d_in, N = w_oi ? s.d_in : s.d_out;
  size_t parts = 0;   // of the first product, and of those that are added to it
  for (bool sum : {(d->flags & ACC_FLAG_DW_ACCUMULATE) != 0, true}) {
    const size_t bytes = token_parts_bytes(d->io_dtype, d->dw_dtype, sum, M, N, p.tokens);
    if (bytes > parts && (!sum || (d->flags & ACC_FLAG_DW_ACCUMULATE) || p.tokens < s.n)) parts = bytes;
  }
  p.total = p.parts + parts;
  return p;
}

int validate_gated(const acc_gated_desc* d, int64_t* ldg, int64_t* ldh) {
  if (!d) return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(d->io_dtype) || !valid_format(d->format)) return ACC_ERR_DTYPE;
  *ldg = d->ldg;
  *ldh = d->ldh;
  const int rc = validate_rows(d->n, d->f, ldg);
  return rc != ACC_OK ? rc : validate_rows(d->n, d->f, ldh);
}

// ---- the vocabulary's cross entropy --------------------------------------------------------------------
constexpr int64_t kCePieceBytes = (int64_t)1 << 30;

struct CePlan {
  int64_t n, d, v, ldx, ldw;
  int64_t run;      // tokens of a run
  int64_t rows;     // of the dense matrices: a run, and 256 at least
  int64_t vp, ldz;  // columns of a piece, their row stride
  CeChoice sums;    // tile of the forward product
  int64_t strips;   // its waves' strips of columns, 128 wide on the persistent kernel, else 64
  SplitChoice dx_choice;   // of dX's sum over a piece
  int least_rows;
  size_t order, count, unit, targets, per_row, x, part, z, parts, dx, dw_parts;   // offsets into the workspace
  size_t forward, backward;                      // its bytes
};

// dX [n, d] is a sum over the whole piece: where its tiles leave compute units idle the sum is taken in parts, which the last kernel adds
// up (pick_split_gemm; in float32 parts of 512 columns at least, enough for four 64 x 64 tiles to a compute unit, two where
// there is one row of tiles: us a step with two / four, 1 x 2048 x 32000 313 / 321, 200 x 1024 x 16000 291 / 285, 1024 x 512 x 32000
// 1127 / 1109, 2048 x 1024 x 16000 1884 / 1826, 515 x 520 x 10007 244 / 244).
void plan_ce_dx(CePlan* p, bool b16) {
  p->dx_choice = pick_split_gemm(p->run, p->d, p->vp, 32, false, true);
  if (!b16) {
    int64_t splits = (p->run > 64 ? 1024 : 512) / (ceil_div(p->run, 64) * ceil_div(p->d, 64));
    if (splits > p->vp / 512) splits = p->vp / 512;
    if (splits < 1) splits = 1;
    p->dx_choice.k_per_split = round_up(ceil_div(p->vp, splits), 64);
    p->dx_choice.splits = ceil_div(p->vp, p->dx_choice.k_per_split);
  }
}

int plan_ce(const acc_ce_desc* d, CePlan* p) {
  if (!d || (d->flags & ~(uint32_t)ACC_FLAG_DW_ACCUMULATE) || d->reserved) return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(d->io_dtype) || !valid_dtype(d->dw_dtype)) return ACC_ERR_DTYPE;
  if (d->n <= 0 || d->n > (int64_t)1 << 30 || d->d <= 0 || d->d % 8 || d->d > (1 << 16) || d->v <= 0 || d->v > (1 << 21)) return ACC_ERR_SHAPE;
  if (d->piece < 0 || d->piece % 256 || d->piece > (1 << 22)) return ACC_ERR_SHAPE;
  p->n = d->n; p->d = d->d; p->v = d->v;
  p->ldx = d->ldx ? d->ldx : d->d;
  p->ldw = d->ldw ? d->ldw : d->d;
  for (int64_t ld : {p->ldx, p->ldw})
    if (ld < p->d || ld % 8 || ld > (1 << 18)) return ACC_ERR_SHAPE;
  const int64_t es = (int64_t)dtype_size(d->io_dtype);
  p->run = ((int64_t)2 << 30) / (p->d * es) / 256 * 256;
  if (p->run > 1 << 18) p->run = 1 << 18;
  const int64_t by_strips = ((int64_t)4 << 30) / (8 * ceil_div(p->v, 64)) / 256 * 256;   // 4 GiB of strips' sums
  if (p->run > by_strips) p->run = by_strips;
  if (p->run > p->n) p->run = p->n;
  p->rows = p->run < 256 ? 256 : p->run;
  // rows of dz that are there whatever the number of tokens that take part, zeros behind them: what the product over the tokens takes at
  // least, three K tiles where it may run on the persistent kernel
  p->least_rows = p->run <= 128 ? 64 : 192;
  // a piece: at most kCePieceBytes of dz, and of W what a buffer resource reaches
  int64_t vp = d->piece ? d->piece : kCePieceBytes / (p->rows * es) / 256 * 256;
  const int64_t most = ((int64_t)2 << 30) / (p->ldw * es) / 256 * 256;
  const int64_t most_z = ((int64_t)2 << 30) / (p->rows * 4) / 256 * 256;
  if (vp > most) vp = most;
  if (vp > most_z) vp = most_z;
  if (vp < 256) vp = 256;
  if (vp > p->v) vp = p->v;
  p->vp = vp;
  p->ldz = round_up(vp, 64);   // whole cache lines: rows that begin inside one cost the product with W twice the requests
  p->sums = pick_ce_tile(p->run, p->v, p->d);
  p->strips = ceil_div(p->v, p->sums.tile == CeTile::k256 ? 128 : 64);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t from = at;
    at += (size_t)round_up(bytes, 256);
    return from;
  };
  p->order = take(p->run * 4);
  p->count = take(4);
  p->unit = take(4);
  p->targets = take(p->rows * 8);
  p->per_row = take(3 * p->rows * 4);
  p->x = take(p->rows * p->d * es);
  // forward: bfloat16 logits never leave the accumulators, float ones do
  const size_t shared = at;
  p->part = take(p->strips * p->rows * 8);
  p->z = shared;
  if (d->io_dtype == ACC_F32) {
    at = shared;
    p->z = take(p->rows * p->ldz * 4);
  }
  p->forward = at;
  at = shared;   // backward: dz, then dX in float
  take(p->rows * p->ldz * es);
  plan_ce_dx(p, d->io_dtype == ACC_BF16);
  p->parts = take(p->dx_choice.splits * p->rows * p->d * 4);
  p->dx = take(p->vp < p->v ? p->rows * p->d * 4 : 0);
  int64_t dw = 0;
  for (bool sum : {(d->flags & ACC_FLAG_DW_ACCUMULATE) != 0, true}) {   // runs after the first are added
    if (sum && !(d->flags & ACC_FLAG_DW_ACCUMULATE) && p->run == p->n) continue;
    const int64_t bytes = (int64_t)token_parts_bytes(d->io_dtype, d->dw_dtype, sum, p->vp, p->d, p->run < p->least_rows ? p->least_rows : p->run);
    if (bytes > dw) dw = bytes;
  }
  p->dw_parts = take(dw);
  p->backward = at > p->forward ? at : p->forward;
  return ACC_OK;
}

// A run of tokens t0 .. t0 + n - 1 and the workspace of its call.
struct CeRun {
  const acc_ce_desc* desc;
  CePlan p;
  char* ws;
  int64_t t0, n;
  CeTokens tokens;
  size_t es() const { return dtype_size(desc->io_dtype); }
  const void* w_piece(const void* W, int64_t v0) const { return (const char*)W + (size_t)v0 * p.ldw * es(); }
  int64_t piece(int64_t v0) const { return p.v - v0 < p.vp ? p.v - v0 : p.vp; }
};

// last: as in CeTokens.
template <typename F>
int ce_runs(const acc_ce_desc* desc, const CePlan& p, const int64_t* targets, int64_t last, void* workspace, hipStream_t stream, F&& f) {
  Launcher L{stream};
  char* ws = (char*)workspace;
  for (int64_t t0 = 0; t0 < p.n; t0 += p.run) {
    const int64_t n = p.n - t0 < p.run ? p.n - t0 : p.run;
    const CeRun run{desc, p, ws, t0, n, CeTokens{targets + t0, (int)n, last, (int*)(ws + p.order), (int*)(ws + p.count)}};
    f(run, L);
  }
  return L.status();
}

// The tokens that take part, and what is read of them, into dense matrices.
void ce_gather(const CeRun& r, const void* X, const float* stats, const float* dloss, Launcher& L) {
  float* unit = (float*)(r.ws + r.p.unit);
  const bool units = dloss && r.desc->io_dtype == ACC_BF16;
  const bool here = r.n <= kCeSelectHere;
  if (!here) L(ce_select_kernel, dim3(1), dim3(1024), r.tokens, units ? dloss + r.t0 : nullptr, unit);
  auto typed = [&](auto value, auto select) {
    using T = decltype(value);
    L(ce_gather_kernel<T, decltype(select)::value>, dim3((unsigned)r.p.rows), dim3(256), r.tokens, (const T*)X + (size_t)r.t0 * r.p.ldx, r.p.ldx, (int)r.p.d,
      r.p.rows, (T*)(r.ws + r.p.x), r.p.v, stats ? stats + r.t0 : nullptr, dloss ? dloss + r.t0 : nullptr, units ? unit : nullptr, r.p.n,
      (int64_t*)(r.ws + r.p.targets), (float*)(r.ws + r.p.per_row));
  };
  auto of = [&](auto value) { here ? typed(value, std::true_type{}) : typed(value, std::false_type{}); };
  if (r.desc->io_dtype == ACC_BF16) of(bf16{});
  else of(float{});
}

// Z [rows, piece] = X . W_piece^T in float32.
void ce_logits_f32(const CeRun& r, const void* W, int64_t v0, Launcher& L) {
  f32_product(F32Operand{r.ws + r.p.x, r.p.d, true, false}, F32Operand{r.w_piece(W, v0), r.p.ldw, true, false}, r.ws + r.p.z, ACC_F32, r.p.ldz, r.n,
              r.piece(v0), r.p.d, false, L, true, r.tokens.count);
}

// X . W^T over columns v0 .. v0 + vp - 1, bfloat16, into sums of exponentials or the logits' gradient [rows, ldz].
// X: null for the gathered tokens, else the run's, all of them.
template <Epilogue EPI> void ce_product(const CeRun& r, const void* X, const void* W, int64_t v0, int64_t vp, Launcher& L) {
  FastGemmParams p = fast_params(X ? X : r.ws + r.p.x, r.w_piece(W, v0), r.ws + r.p.z, r.n, vp, r.p.d, X ? r.p.ldx : r.p.d, r.p.ldw, r.p.ldz, nullptr, 1.f, 0.f);
  float* per_row = (float*)(r.ws + r.p.per_row);
  p.live = X ? nullptr : r.tokens.count;
  p.ce = CeRows{X ? r.tokens.targets : (const int64_t*)(r.ws + r.p.targets), per_row + r.p.rows, per_row, per_row + 2 * r.p.rows,
                (f32x2*)(r.ws + r.p.part), X ? r.n : r.p.rows, v0};
  p.least_rows = r.p.least_rows;
  if (EPI == Epilogue::kGradient && p.M < p.least_rows) p.M = p.least_rows;   // for the grid
  auto ring = [&](auto tm, auto tn, auto ns) {
    constexpr int TM = decltype(tm)::value, TN = decltype(tn)::value, NS = decltype(ns)::value;
    const unsigned grid = gemm_ring_plan(p, 32 * TM, 32 * TN);
    L.launch_lds(gemm_ring_kernel<TM, TN, NS, true, bf16, kNone, false, true, EPI, true>, dim3(grid), dim3(256), (size_t)gemm_ring_lds_bytes<TM, TN, NS>(), p);
  };
  using std::integral_constant;
  const integral_constant<int, 2> two{};
  const integral_constant<int, 3> three{};
  const integral_constant<int, 4> four{};
  const CeChoice c = EPI == Epilogue::kExpSums ? r.p.sums : pick_ce_tile(r.p.run, r.p.vp, r.p.d);
  switch (c.tile) {
    case CeTile::k64x128: return ring(two, four, three);
    case CeTile::k128: return c.one_round ? ring(four, four, three) : ring(four, four, two);
    case CeTile::k192x128: return ring(integral_constant<int, 6>{}, four, two);
    case CeTile::k256: break;
  }
  gemm_ring_plan(p, 256, 256);
  if (p.super_m > 8) p.super_m = 8;
  if (p.K % 64) L.launch_lds(gemm16_persist_kernel<true, true, true, EPI>, dim3(256), dim3(256), (size_t)160 * 1024, p, 0);
  else L.launch_lds(gemm16_persist_kernel<true, false, true, EPI>, dim3(256), dim3(256), (size_t)160 * 1024, p, 0);
}

// The parts (float) of dz . W_piece for the rows with a token; their number.
int ce_input_gradient(const CeRun& r, const void* W, int64_t v0, Launcher& L) {
  const int64_t vp = r.piece(v0), stride = r.p.rows * r.p.d;
  const SplitChoice& c = r.p.dx_choice;
  const int splits = (int)ceil_div(vp, c.k_per_split);
  float* parts = (float*)(r.ws + r.p.parts);
  if (r.desc->io_dtype != ACC_BF16) {
    f32_split_product(F32Operand{r.ws + r.p.z, r.p.ldz, true, false}, F32Operand{r.w_piece(W, v0), r.p.ldw, false, false}, parts, r.p.d, r.n, r.p.d, vp,
                      c.k_per_split, stride, r.tokens.count, L);
    return splits;
  }
  FastGemmParams p = fast_params(r.ws + r.p.z, r.w_piece(W, v0), parts, r.n, r.p.d, round_up(vp, 8), r.p.ldz, r.p.ldw, r.p.d, nullptr, 1.f, 0.f);
  p.kb_rows = vp;
  p.live = r.tokens.count;
  p.k_per_split = c.k_per_split;
  p.c_split_stride = stride;
  if (c.tile == GemmTile::k256) {
    gemm_ring_plan(p, 256, 256);
    if (p.super_m > 8) p.super_m = 8;
    L.launch_lds(gemm16_persist_kernel<false, true, true, Epilogue::kParts>, dim3(256), dim3(256), (size_t)160 * 1024, p, 0);
    return splits;
  }
  with_ring_tile(c.tile, false, [&](auto tm, auto tn, auto ns) {
    constexpr int TM = decltype(tm)::value, TN = decltype(tn)::value, NS = decltype(ns)::value;
    const unsigned grid = gemm_ring_plan(p, 32 * TM, 32 * TN);
    p.tile_blocks = (int)grid;
    L.launch_lds(gemm_ring_kernel<TM, TN, NS, false, float, kPlain, false, true, Epilogue::kStore, true>, dim3(grid * (unsigned)splits), dim3(256),
                 (size_t)gemm_ring_lds_bytes<TM, TN, NS>(), p);
  });
  return splits;
}

}  // namespace
}  // namespace acc

using namespace acc;

extern "C" {

int acc_act8_pack(const acc_act8_desc* desc, const void* X, void* Q, void* E, void* stream) {
  if (!desc) return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(desc->io_dtype) || !valid_format(desc->format)) return ACC_ERR_DTYPE;
  int64_t ld = desc->ldx;
  int rc = validate_rows(desc->n, desc->c, &ld);
  if (rc != ACC_OK) return rc;
  if (!X || !Q || !E) return ACC_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(Q) || !aligned16(E)) return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  act8_pack(desc->io_dtype, desc->format, X, desc->n, desc->c, ld, Q, E, L);
  return L.status();
}

int acc_act8_unpack(const acc_act8_desc* desc, const void* Q, const void* E, void* X, void* stream) {
  if (!desc) return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(desc->io_dtype) || !valid_format(desc->format)) return ACC_ERR_DTYPE;
  int64_t ld = desc->ldx;
  int rc = validate_rows(desc->n, desc->c, &ld);
  if (rc != ACC_OK) return rc;
  if (!X || !Q || !E) return ACC_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(Q) || !aligned16(E)) return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  act8_unpack(desc->io_dtype, desc->format, Q, E, desc->n, desc->c, ld, X, L);
  return L.status();
}

int acc_linear_fwd_act8(const acc_linear_desc* desc, int format, const void* X, const void* W, void* Y, void* Q, void* E,
                        void* stream) {
  Shape s;
  int rc = validate_desc(desc, &s);
  if (rc != ACC_OK) return rc;
  if (!valid_format(format)) return ACC_ERR_DTYPE;
  const bool keep = !(desc->flags & ACC_FLAG_SKIP_SKETCH);
  if (keep && act_work_groups(s.n, s.d_in) >= 1 << 24) return ACC_ERR_SHAPE;
  if (!X || !W || !Y || (keep && (!Q || !E))) return ACC_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(W) || !aligned16(Y) || !aligned16(Q) || !aligned16(E)) return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  // the checkpoint first: it leaves X in the memory-side cache for the product, as the sketch does
  if (keep) act8_pack(desc->io_dtype, format, X, s.n, s.d_in, s.ldx, Q, E, L);
  exact_forward_gemm(desc, s, X, W, Y, L);
  return L.status();
}

size_t acc_linear_act8_workspace_bytes(const acc_linear_desc* desc) {
  Shape s;
  if (validate_desc(desc, &s) != ACC_OK) return 0;
  return plan_act8(desc, s).total;
}

int acc_linear_bwd_act8(const acc_linear_desc* desc, int format, const void* dY, const void* W, const void* Q, const void* E,
                        void* dX, void* dW, void* workspace, size_t ws_bytes, void* stream) {
  Shape s;
  int rc = validate_desc(desc, &s);
  if (rc != ACC_OK) return rc;
  if (!valid_format(format)) return ACC_ERR_DTYPE;
  if (desc->flags & ACC_FLAG_SKIP_SKETCH) return ACC_ERR_INVALID_ARG;
  if (!dY || (!dX && !dW) || (dX && !W) || (dW && (!Q || !E))) return ACC_ERR_INVALID_ARG;
  if (!aligned16(dY) || !aligned16(W) || !aligned16(Q) || !aligned16(E) || !aligned16(dX) || !aligned16(dW) || !aligned16(workspace))
    return ACC_ERR_ALIGN;
  const Act8Plan plan = plan_act8(desc, s);
  if (dW && !plan.total) return ACC_ERR_SHAPE;
  if (dW && (!workspace || ws_bytes < plan.total)) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  if (dX) exact_backward_gemm(desc, s, dY, W, dX, L);
  if (dW) {
    const bool w_oi = (desc->flags & ACC_FLAG_W_OUT_IN) != 0;
    const int64_t chunk = plan.tokens;
    float* parts = (float*)((char*)workspace + plan.parts);
    for (int64_t t0 = 0; t0 < s.n; t0 += chunk) {
      const int64_t nt = s.n - t0 < chunk ? s.n - t0 : chunk;
      const char* dy = (const char*)dY + (size_t)t0 * s.ldy * dtype_size(desc->io_dtype);
      act8_unpack(desc->io_dtype, format, (const char*)Q + t0 * s.d_in, (const char*)E + t0 / kActBlock * s.d_in, nt, s.d_in, s.d_in, workspace, L);
      const bool add = t0 > 0 || (desc->flags & ACC_FLAG_DW_ACCUMULATE);
      if (w_oi) token_product(desc->io_dtype, desc->dw_dtype, dy, s.ldy, workspace, s.d_in, dW, s.d_in, s.d_out, s.d_in, nt, add, L, nt == chunk ? parts : nullptr);
      else token_product(desc->io_dtype, desc->dw_dtype, workspace, s.d_in, dy, s.ldy, dW, s.d_out, s.d_in, s.d_out, nt, add, L, nt == chunk ? parts : nullptr);
    }
  }
  return L.status();
}

int acc_gated_fwd_act8(const acc_gated_desc* desc, const void* G, const void* U, void* H, void* Qg, void* Eg, void* Qu,
                       void* Eu, void* stream) {
  int64_t ldg, ldh;
  int rc = validate_gated(desc, &ldg, &ldh);
  if (rc != ACC_OK) return rc;
  if (!G || !U || !H || !Qg || !Eg || !Qu || !Eu) return ACC_ERR_INVALID_ARG;
  if (!aligned16(G) || !aligned16(U) || !aligned16(H) || !aligned16(Qg) || !aligned16(Eg) || !aligned16(Qu) || !aligned16(Eu))
    return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  with_act8(desc->io_dtype, desc->format, [&](auto value, auto fmt) {
    using T = decltype(value);
    L(gated_fwd_kernel<T, decltype(fmt)::value>, dim3((unsigned)act_work_groups(desc->n, desc->f)), dim3(256), (const T*)G, (const T*)U, desc->n, desc->f,
      ldg, ldh, (T*)H, (uint8_t*)Qg, (uint8_t*)Eg, (uint8_t*)Qu, (uint8_t*)Eu);
  });
  return L.status();
}

int acc_gated_bwd_act8(const acc_gated_desc* desc, const void* dH, const void* Qg, const void* Eg, const void* Qu,
                       const void* Eu, void* dG, void* dU, void* H, void* stream) {
  int64_t ldg, ldh;
  int rc = validate_gated(desc, &ldg, &ldh);
  if (rc != ACC_OK) return rc;
  if (!dH || !Qg || !Eg || !Qu || !Eu || !dG || !dU) return ACC_ERR_INVALID_ARG;
  if (!aligned16(dH) || !aligned16(Qg) || !aligned16(Eg) || !aligned16(Qu) || !aligned16(Eu) || !aligned16(dG) || !aligned16(dU) || !aligned16(H))
    return ACC_ERR_ALIGN;
  if ((rc = check_device()) != ACC_OK) return rc;
  Launcher L{(hipStream_t)stream};
  with_act8(desc->io_dtype, desc->format, [&](auto value, auto fmt) {
    using T = decltype(value);
    L(gated_bwd_kernel<T, decltype(fmt)::value>, dim3((unsigned)act_work_groups(desc->n, desc->f)), dim3(256), (const T*)dH, (const uint8_t*)Qg,
      (const uint8_t*)Eg, (const uint8_t*)Qu, (const uint8_t*)Eu, desc->n, desc->f, ldg, ldh, (T*)dG, (T*)dU, (T*)H);
  });
  return L.status();
}

size_t acc_linear_ce_workspace_bytes(const acc_ce_desc* desc, int is_backward) {
  CePlan p;
  if (plan_ce(desc, &p) != ACC_OK) return 0;
  return is_backward ? p.backward : p.forward;
}

int acc_linear_ce_fwd(const acc_ce_desc* desc, const void* X, const void* W, const int64_t* targets, float* loss, float* stats,
                      void* workspace, size_t ws_bytes, void* stream) {
  CePlan p;
  int rc = plan_ce(desc, &p);
  if (rc != ACC_OK) return rc;
  if (!X || !W || !targets || !loss || !stats) return ACC_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(W) || !aligned16(targets) || !aligned16(loss) || !aligned16(stats) || !aligned16(workspace)) return ACC_ERR_ALIGN;
  if (!workspace || ws_bytes < p.forward) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  return ce_runs(desc, p, targets, INT64_MAX, workspace, (hipStream_t)stream, [&](const CeRun& r, Launcher& L) {
    float* per_row = (float*)(r.ws + r.p.per_row);
    if (desc->io_dtype == ACC_BF16) {
      // Where one tile of the product holds all tokens nothing is saved by leaving some out.  (A token's logits are its own, so what
      // stands in the row of one without a loss reaches no other.)
      CeTokens tokens = r.tokens;
      const bool as_they_come = r.n <= 256;
      if (as_they_come) tokens.order = tokens.count = nullptr;
      else ce_gather(r, X, nullptr, nullptr, L);
      // of W what a buffer resource reaches: chunks past K go to its end, and have to lie outside
      const int64_t columns = ((int64_t)2 << 30) / (r.p.ldw * 2) / 256 * 256;
      for (int64_t v0 = 0; v0 < r.p.v; v0 += columns)
        ce_product<Epilogue::kExpSums>(r, as_they_come ? (const bf16*)X + (size_t)r.t0 * r.p.ldx : nullptr, W, v0, r.p.v - v0 < columns ? r.p.v - v0 : columns, L);
      int across = 16;   // rows of a work-group
      while (across > 1 && across / 2 >= r.n) across /= 2;
      L(ce_finish_kernel, dim3((unsigned)ceil_div(r.n, across)), dim3(256), tokens, (const f32x2*)(r.ws + r.p.part), (int)r.p.strips,
        as_they_come ? r.n : r.p.rows, across, r.p.v, (const float*)(per_row + r.p.rows), loss + r.t0, stats + r.t0, r.p.n);
      return;
    }
    ce_gather(r, X, nullptr, nullptr, L);
    for (int64_t v0 = 0; v0 < r.p.v; v0 += r.p.vp) {
      const int64_t vp = r.piece(v0);
      ce_logits_f32(r, W, v0, L);
      L(ce_piece_stats_kernel, dim3((unsigned)r.n), dim3(256), r.tokens, (const float*)(r.ws + r.p.z), r.p.ldz, v0, (int)vp, v0 == 0, v0 + vp == r.p.v,
        r.p.v, per_row, per_row + r.p.rows, per_row + 2 * r.p.rows, loss + r.t0, stats + r.t0, r.p.n);
    }
  });
}

int acc_linear_ce_bwd(const acc_ce_desc* desc, const void* X, const void* W, const int64_t* targets, const float* stats,
                      const float* dloss, void* dX, void* dW, void* workspace, size_t ws_bytes, void* stream) {
  CePlan p;
  int rc = plan_ce(desc, &p);
  if (rc != ACC_OK) return rc;
  if (!X || !W || !targets || !stats || !dloss || (!dX && !dW)) return ACC_ERR_INVALID_ARG;
  if (!aligned16(X) || !aligned16(W) || !aligned16(targets) || !aligned16(stats) || !aligned16(dloss) || !aligned16(dX) || !aligned16(dW) ||
      !aligned16(workspace))
    return ACC_ERR_ALIGN;
  if (!workspace || ws_bytes < p.backward) return ACC_ERR_WORKSPACE;
  if ((rc = check_device()) != ACC_OK) return rc;
  const bool b16 = desc->io_dtype == ACC_BF16;
  return ce_runs(desc, p, targets, p.v - 1, workspace, (hipStream_t)stream, [&](const CeRun& r, Launcher& L) {
    ce_gather(r, X, stats, dloss, L);
    float* per_row = (float*)(r.ws + r.p.per_row);
    float* dxf = (float*)(r.ws + r.p.dx);
    const float* unit = b16 ? (const float*)(r.ws + r.p.unit) : nullptr;
    char* dz = r.ws + r.p.z;
    for (int64_t v0 = 0; v0 < r.p.v; v0 += r.p.vp) {
      const int64_t vp = r.piece(v0);
      if (b16) {
        ce_product<Epilogue::kGradient>(r, nullptr, W, v0, vp, L);
      } else {
        ce_logits_f32(r, W, v0, L);
        L(ce_piece_grad_kernel, dim3((unsigned)r.p.rows), dim3(256), r.tokens, (float*)dz, r.p.ldz, v0, (int)vp, r.p.rows, (const int64_t*)(r.ws + r.p.targets), (const float*)per_row);
      }
      if (dX) {
        const int splits = ce_input_gradient(r, W, v0, L);
        const CeParts sum{(const float*)(r.ws + r.p.parts), splits, r.p.rows * r.p.d, v0 > 0 ? dxf : nullptr};
        const dim3 grid((unsigned)r.n);
        if (v0 + vp < r.p.v) L(ce_add_kernel, grid, dim3(256), r.tokens, sum, (int)r.p.d, dxf);
        else if (b16) L(ce_scatter_kernel<bf16>, grid, dim3(256), r.tokens, sum, unit, (int)r.p.d, (bf16*)dX + (size_t)r.t0 * r.p.ldx, r.p.ldx);
        else L(ce_scatter_kernel<float>, grid, dim3(256), r.tokens, sum, unit, (int)r.p.d, (float*)dX + (size_t)r.t0 * r.p.ldx, r.p.ldx);
      }
      if (dW) {
        char* dw = (char*)dW + (size_t)v0 * r.p.d * dtype_size(desc->dw_dtype);
        const bool add = r.t0 > 0 || (desc->flags & ACC_FLAG_DW_ACCUMULATE);
        token_product(desc->io_dtype, desc->dw_dtype, dz, r.p.ldz, r.ws + r.p.x, r.p.d, dw, r.p.d, vp, r.p.d, b16 && r.n < r.p.least_rows ? r.p.least_rows : r.n, add,
                      L, vp == r.p.vp && r.n == r.p.run ? (float*)(r.ws + r.p.dw_parts) : nullptr, r.tokens.count, unit, r.p.least_rows);
      }
    }
  });
}

}  // extern "C"
