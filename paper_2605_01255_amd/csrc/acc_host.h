// What the files with entry points share: validation, launches, and the products that one of them offers the others.
#pragma once
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <atomic>
#include <mutex>
#include <tuple>
#include <utility>

#include "acc_common.h"
#include "acc_gemm.h"

namespace acc {

inline bool valid_dtype(int32_t d) { return d == ACC_F32 || d == ACC_BF16; }
inline size_t dtype_size(int32_t d) { return d == ACC_BF16 ? 2 : 4; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Shape {
  int64_t n, d_in, d_out, r, ldx, ldw, ldy;
  int64_t ldf;  // row stride of the factors whose rows hold r elements
};

inline int validate_desc(const acc_linear_desc* d, Shape* s, uint32_t extra_flags = 0) {
  if (!d) return ACC_ERR_INVALID_ARG;
  if (d->flags & ~(uint32_t)(ACC_FLAG_SKIP_SKETCH | ACC_FLAG_ONE_LAUNCH | ACC_FLAG_W_OUT_IN | ACC_FLAG_DW_ACCUMULATE |
                             extra_flags))
    return ACC_ERR_INVALID_ARG;
  if (!valid_dtype(d->io_dtype) || !valid_dtype(d->factor_dtype) || !valid_dtype(d->dw_dtype))
    return ACC_ERR_DTYPE;
  if (d->n <= 0 || d->d_in <= 0 || d->d_out <= 0 || d->r <= 0) return ACC_ERR_SHAPE;
  if (d->r % 8 || d->d_in % 8 || d->d_out % 8) return ACC_ERR_SHAPE;  // 16-byte rows of every operand and factor
  // limits that keep every grid dimension and 32-bit tile count in range
  if (d->n > (int64_t)1 << 30 || d->d_in > (1 << 21) || d->d_out > (1 << 21) || d->r > (1 << 16))
    return ACC_ERR_SHAPE;
  if (d->row_offset % 4) return ACC_ERR_SHAPE;
  s->n = d->n; s->d_in = d->d_in; s->d_out = d->d_out; s->r = d->r;
  s->ldx = d->ldx ? d->ldx : d->d_in;
  const int64_t w_row = (d->flags & ACC_FLAG_W_OUT_IN) ? d->d_in : d->d_out;  // elements per row of W
  s->ldw = d->ldw ? d->ldw : w_row;
  s->ldy = d->ldy ? d->ldy : d->d_out;
  if (s->ldx < s->d_in || s->ldw < w_row || s->ldy < s->d_out) return ACC_ERR_SHAPE;
  if (s->ldx % 8 || s->ldw % 8 || s->ldy % 8) return ACC_ERR_SHAPE;
  s->ldf = d->ldf ? d->ldf : d->r;
  if (s->ldf < s->r || s->ldf % 8 || s->ldf > ((int64_t)1 << 24)) return ACC_ERR_SHAPE;
  return ACC_OK;
}

// ACC_VERBOSE=1 in the environment prints the HIP error behind an ACC_ERR_HIP to stderr.
inline int hip_fail(hipError_t e, const char* what) {
  static const bool verbose = getenv("ACC_VERBOSE") != nullptr;
  if (verbose) fprintf(stderr, "libacc: %s: %s\n", what, hipGetErrorString(e));
  return ACC_ERR_HIP;
}

// The library only runs on gfx950; the answer is cached per device ordinal.
inline int check_device() {
  static std::atomic<int> cached[64];  // 0 unknown, 1 ok, -1 not gfx950
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev < 0 || dev >= 64) return ACC_ERR_HIP;
  if (cached[dev] == 0) {
    hipDeviceProp_t prop;
    e = hipGetDeviceProperties(&prop, dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDeviceProperties");
    cached[dev] = (strncmp(prop.gcnArchName, "gfx950", 6) == 0) ? 1 : -1;
    if (cached[dev] != 1) hip_fail(hipErrorInvalidDevice, prop.gcnArchName);
  }
  return cached[dev] == 1 ? ACC_OK : ACC_ERR_HIP;
}

inline RaisedLimits g_raised;

// Enqueues kernels on one stream and remembers the first launch error.
struct Launcher {
  hipStream_t st;
  hipError_t err = hipSuccess;
  template <typename... KArgs, typename... Args>
  void operator()(void (*kernel)(KArgs...), dim3 grid, dim3 block, Args... args) {
    launch_lds(kernel, grid, block, 0, args...);
  }
  // lds_bytes of dynamic LDS; above 64 KB the kernel's limit is raised first (no allocation involved).
  template <typename... KArgs, typename... Args>
  void launch_lds(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t lds_bytes, Args... args) {
    if (err != hipSuccess) return;
    if (lds_bytes > 64 * 1024) {
      int dev = 0;
      err = hipGetDevice(&dev);
      if (err != hipSuccess) return;
      if (!g_raised.has((const void*)kernel, dev)) {
        err = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_bytes);
        if (err != hipSuccess) return;
        g_raised.add((const void*)kernel, dev);
      }
    }
    std::tuple<KArgs...> vals{args...};
    void* ptrs[sizeof...(KArgs)];
    fill(ptrs, vals, std::index_sequence_for<KArgs...>{});
    err = hipLaunchKernel((const void*)kernel, grid, block, ptrs, lds_bytes, st);
  }
  template <typename T, size_t... I>
  static void fill(void** ptrs, T& vals, std::index_sequence<I...>) {
    ((ptrs[I] = (void*)&std::get<I>(vals)), ...);
  }
  int status() const { return err == hipSuccess ? ACC_OK : hip_fail(err, "kernel launch"); }
};

// The K4 reduction of a sketch, handed to the GEMM launched right after it (FastGemmParams::red_*)
// instead of taking a launch of its own.  count == 0: nothing pending.
struct ReduceJob {
  const float* part;
  void* out;
  int64_t count;
  int G;
  int out_bf16;
  int64_t row, ld;  // the result's rows hold `row` elements and are stored `ld` apart
};

inline FastGemmParams fast_params(const void* A, const void* B, void* C, int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldb,
                           int64_t ldc, const ReduceJob* job, float alpha, float beta) {
  FastGemmParams p{};
  p.alpha = alpha; p.beta = beta;
  p.A = (const bf16*)A; p.B = (const bf16*)B; p.C = C;
  p.M = M; p.N = N; p.K = K; p.lda = lda; p.ldb = ldb; p.ldc = ldc;
  if (job && job->count) {
    p.red_part = job->part; p.red_out = job->out; p.red_count = job->count; p.red_G = job->G;
    p.red_out_bf16 = job->out_bf16;
    p.red_row = job->row; p.red_ld = job->ld;
  }
  return p;
}

// An operand of the float32 kernel: X[rows, K] with K contiguous (kmajor), or Xt[K, rows] with the rows contiguous.
struct F32Operand {
  const void* ptr;
  int64_t ld;
  bool kmajor;
  bool b16;  // bfloat16 elements
};

// ---- products of acc_api.hip ----------------------------------------------------------------------------
// The exact products of a pass: Y = X . W and dX = dY . W^T.
void exact_forward_gemm(const acc_linear_desc* desc, const Shape& s, const void* X, const void* W, void* Y, Launcher& L,
                        const ReduceJob* job = nullptr);
void exact_backward_gemm(const acc_linear_desc* desc, const Shape& s, const void* dY, const void* W, void* dX, Launcher& L,
                         const ReduceJob* job = nullptr);
// C[M, N] (+)= A . B for float32 operands of any order, C of `dtype`.  `padded`: rows of a K-contiguous A and of C may be read and
// written up to a multiple of four, A's zeros behind K among them (any N and K then).  f32_split_product: the same with the K range in
// runs of k_per_split (a multiple of 32), each into a C of its own, split_stride apart.  live: device count of A's rows that need to
// take part (the K range, where A is transposed); those behind it hold what changes nothing, and may take part.
void f32_product(const F32Operand& a, const F32Operand& b, void* C, int32_t dtype, int64_t ldc, int64_t M, int64_t N, int64_t K,
                 bool accumulate, Launcher& L, bool padded = false, const int* live = nullptr);
void f32_split_product(const F32Operand& a, const F32Operand& b, float* C, int64_t ldc, int64_t M, int64_t N, int64_t K, int64_t k_per_split,
                       int64_t split_stride, const int* live, Launcher& L);
}  // namespace acc
