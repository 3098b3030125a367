// libgbmuf: the largest logits of a row, and distillation from them.  The interface is in include/gbmuf.h; this
// file holds the host side and the C ABI, the kernels are in top_logits.cuh and distill.cuh.

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "gbmuf.h"

#include "host_common.h"
#include "primitives.cuh"
#include "packed_math.cuh"
#include "linear_epilogue.cuh"
#include "softmax_math.cuh"
#include "row_pieces.cuh"
#include "top_logits.cuh"
#include "distill.cuh"
#include "ops_host.h"

namespace {

constexpr double kColdest = 1.0 / 1024, kHottest = 1024.0;

bool temperature_of(float T, Temperature* t) {
  if (!(T >= kColdest && T <= kHottest)) return false;
  const double c = 1.4426950408889634 / (double)T;                // log2 e / T
  t->hi = (float)c;
  t->lo = (float)(c - (double)t->hi);
  t->least = -200.0f * T;
  t->inverse = 1.0 / (double)T;
  return true;
}
const char kTemperatureText[] = "temperature must be 1/1024 .. 1024";

// As many CTAs per row as keep every SM busy with few rows, 8 at most, each with half a chunk at least.
int split_few(const gbmuf_ops* ops, long long rows, long long bytes, int blocks_per_sm) {
  const long long ctas = (long long)ops->num_sms * blocks_per_sm;
  int log = 0;
  while (log < 3 && rows << (log + 1) <= ctas && bytes >> (log + 1) >= kLossChunk / 2) ++log;
  return log;
}

template <typename T> cudaError_t launch_top(const gbmuf_ops* ops, TopParams& P, cudaStream_t st) {
  if (P.vocab <= kTopShort)
    return launch(top_short_kernel<T>, (unsigned)std::min<long long>(P.rows, (long long)ops->num_sms * 8), 1, kLossWorkers, 0, st, P);
  P.split = 1 << split_few(ops, P.rows, P.vocab * (long long)sizeof(T), kTopBlocksPerSm);
  // a cluster shares one row only; a block by itself goes through several
  const long long grid = P.split > 1 ? P.rows * P.split : std::min<long long>(P.rows, (long long)ops->num_sms * kTopBlocksPerSm);
  return launch(top_ring_kernel<T>, (unsigned)grid, (unsigned)P.split, kLossThreads, kTopSmem, st, P);
}

constexpr long long kDistillCacheBytes = 64ll << 20;      // of the 126 MB of L2: the gradient passes through as well

constexpr int kFewLanes = 2;                    // lists of up to 64 entries: two per lane

template <typename T, int LANES> cudaError_t launch_distill(const gbmuf_ops* ops, DistillParams& P, cudaStream_t st) {
  if (P.vocab <= 2048) {
    const auto kernel = P.vocab <= 256 ? distill_warp_kernel<T, 8, LANES> : P.vocab <= 1024 ? distill_warp_kernel<T, 32, LANES>
                                                                                             : distill_warp_kernel<T, 64, LANES>;
    return launch(kernel, (unsigned)((P.rows + 3) / 4), 1, 128, 0, st, P);
  }
  const long long bytes = P.vocab * (long long)sizeof(T), ctas = (long long)ops->num_sms * kLossBlocksPerSm;
  int log = split_few(ops, P.rows, bytes, kLossBlocksPerSm);
  // the slices that are fetched twice, for the gradient, should fit the L2 cache
  while (P.dlogits && log < 3 && (bytes - ((long long)kLossKept * kLossChunk << log)) * (ctas >> log) >= kDistillCacheBytes) ++log;
  P.split = 1 << log;
  const int clusters = (int)std::min<long long>(P.rows, ops->distill_clusters[log]);
  const auto kernel = P.hard == 0.0f || P.T == 1.0f ? distill_ring_kernel<T, 0, LANES>
                    : P.T == 2.0f ? distill_ring_kernel<T, 2, LANES> : P.T == 3.0f ? distill_ring_kernel<T, 3, LANES>
                    : P.T == 4.0f ? distill_ring_kernel<T, 4, LANES> : distill_ring_kernel<T, 1, LANES>;
  return launch(kernel, (unsigned)(clusters * P.split), (unsigned)P.split, kDistillThreads, kDistillSmem, st, P);
}

gbmuf_status check_rows(const gbmuf_ops* ops, int64_t rows, int64_t vocab, int32_t dtype, int32_t k) {
  if (!ops) return invalid("ops is NULL");
  if (rows < 0 || vocab < 0) return invalid("rows and vocab must not be negative");
  if (rows > kMostDim || vocab > kMostDim) return refuse(GBMUF_ERR_UNSUPPORTED, "rows and vocab must be at most 2^31 - 2^16");
  if (rows > 0 && vocab == 0) return invalid("vocab must not be 0");
  if (!is_dtype(dtype)) return invalid("dtype must be GBMUF_F32 or GBMUF_BF16");
  if (k < 1) return invalid("k must be 1 or more");
  if (k > kListMost) return refuse(GBMUF_ERR_UNSUPPORTED, "k must be at most " + std::to_string(kListMost));
  return GBMUF_OK;
}
// A [rows][k] matrix of indices.
const char* check_index(const void* p, int64_t rows, int64_t k, int64_t ld) {
  if (!p) return rows == 0 ? nullptr : "is NULL";
  if ((uintptr_t)p % 8 != 0) return "is not aligned to its element type";
  if (rows > 1 && ld < k) return "has a row stride below its columns";
  if (rows > 1 && ld > ((int64_t)1 << 40)) return "has an extent above 2^56 elements";
  return nullptr;
}

}  // namespace

namespace {

template <typename T, int LANES> cudaError_t raise_limits() {
  const void* const kernels[] = {(const void*)distill_ring_kernel<T, 0, LANES>, (const void*)distill_ring_kernel<T, 1, LANES>,
                                 (const void*)distill_ring_kernel<T, 2, LANES>, (const void*)distill_ring_kernel<T, 3, LANES>,
                                 (const void*)distill_ring_kernel<T, 4, LANES>};
  cudaError_t e = cudaSuccess;
  for (const void* k : kernels)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDistillSmem);
  return e;
}

}  // namespace

gbmuf_status gbmuf_setup_vocab_ops(gbmuf_ops* ops) {
  const int blocks = ops->num_sms * kLossBlocksPerSm;
  int unused[4];
  cudaError_t e = raise_limits<float, kFewLanes>();
  if (e == cudaSuccess) e = raise_limits<float, kListMost / 32>();
  if (e == cudaSuccess) e = raise_limits<__nv_bfloat16, kFewLanes>();
  if (e == cudaSuccess) e = raise_limits<__nv_bfloat16, kListMost / 32>();
  // all of them have the same threads, shared memory and launch bounds
  if (e == cudaSuccess) e = count_clusters(distill_ring_kernel<float, 1, kListMost / 32>, kDistillThreads, kDistillSmem, blocks, ops->distill_clusters);
  if (e == cudaSuccess) e = count_clusters(top_ring_kernel<float>, kLossThreads, kTopSmem, blocks, unused);
  if (e == cudaSuccess) e = count_clusters(top_ring_kernel<__nv_bfloat16>, kLossThreads, kTopSmem, blocks, unused);
  return launched("set-up of the vocabulary operators", e);
}

extern "C" {

gbmuf_status gbmuf_top_logits(gbmuf_ops* ops, const gbmuf_top_logits_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!ops || !a) return invalid("ops and args must not be NULL");
    if (gbmuf_status st = check_rows(ops, a->rows, a->vocab, a->dtype, a->k)) return st;
    if (a->rows > 0 && a->k > a->vocab) return invalid("k must be at most vocab");
    TopParams P{};
    if (!temperature_of(a->temperature, &P.temperature)) return invalid(kTemperatureText);
    CHECK_MATRIX("logits", a->logits, a->rows, a->vocab, a->ld_logits, a->dtype, false);
    CHECK_MATRIX("values", a->values, a->rows, (int64_t)a->k, a->ld_values, a->dtype, false);
    if (const char* why = check_index(a->index, a->rows, a->k, a->ld_index)) return invalid(std::string("index ") + why);
    if ((uintptr_t)a->lse % 4 != 0) return invalid("lse is not aligned to its element type");
    if (a->rows == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    P.logits = a->logits; P.values = a->values; P.index = reinterpret_cast<long long*>(a->index); P.lse = a->lse;
    P.rows = a->rows; P.vocab = a->vocab; P.ld = a->ld_logits; P.ld_values = a->ld_values; P.ld_index = a->ld_index;
    P.k = a->k; P.split = 1; P.status = ops->d_status;
    cudaError_t e = cudaSuccess;
    DISPATCH_DTYPE(a->dtype, T, e = launch_top<T>(ops, P, (cudaStream_t)stream));
    return launched("launch of the largest-logits kernel", e);
  });
}

gbmuf_status gbmuf_distillation(gbmuf_ops* ops, const gbmuf_distillation_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!ops || !a) return invalid("ops and args must not be NULL");
    if (gbmuf_status st = check_rows(ops, a->rows, a->vocab, a->dtype, a->k)) return st;
    if (!is_dtype(a->teacher_dtype)) return invalid("teacher_dtype must be GBMUF_F32 or GBMUF_BF16");
    DistillParams P{};
    if (!temperature_of(a->temperature, &P.temperature)) return invalid(kTemperatureText);
    if (!(a->hard_weight >= 0.0f && a->hard_weight <= 1.0f)) return invalid("hard_weight must be 0 .. 1");
    if (!(a->scale == a->scale)) return invalid("scale must not be NaN");
    CHECK_MATRIX("logits", a->logits, a->rows, a->vocab, a->ld_logits, a->dtype, false);
    CHECK_MATRIX("dlogits", a->dlogits, a->rows, a->vocab, a->ld_dlogits, a->dtype, true);
    CHECK_MATRIX("teacher_logits", a->teacher_logits, a->rows, (int64_t)a->k, a->ld_teacher, a->teacher_dtype, false);
    if (const char* why = check_index(a->teacher_index, a->rows, a->k, a->ld_index)) return invalid(std::string("teacher_index ") + why);
    if (a->hard_weight != 0.0f && a->rows > 0 && !a->targets) return invalid("hard_weight needs targets");
    if ((uintptr_t)a->targets % 8 != 0) return invalid("targets is not aligned to its element type");
    if (((uintptr_t)a->row_weight | (uintptr_t)a->loss | (uintptr_t)a->lse | (uintptr_t)a->teacher_lse) % 4 != 0)
      return invalid("teacher_lse, row_weight, loss or lse is not aligned to its element type");
    if (a->dlogits == a->logits && a->dlogits && a->ld_dlogits != a->ld_logits)
      return invalid("dlogits in place of the logits needs their row stride");
    if (a->rows == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    P.logits = a->logits; P.teacher = a->teacher_logits; P.index = reinterpret_cast<const long long*>(a->teacher_index);
    P.teacher_lse = a->teacher_lse; P.targets = reinterpret_cast<const long long*>(a->targets); P.row_weight = a->row_weight;
    P.loss = a->loss; P.lse = a->lse; P.dlogits = a->dlogits;
    P.rows = a->rows; P.vocab = a->vocab; P.ld = a->ld_logits; P.ld_d = a->ld_dlogits;
    P.ld_teacher = a->ld_teacher; P.ld_index = a->ld_index; P.ignore_index = a->ignore_index;
    P.k = a->k; P.split = 1; P.teacher_bf16 = a->teacher_dtype == GBMUF_BF16;
    P.T = a->temperature; P.hard = a->hard_weight; P.scale = a->scale; P.status = ops->d_status;
    cudaError_t e = cudaSuccess;
    DISPATCH_DTYPE(a->dtype, T, e = a->k <= 32 * kFewLanes ? launch_distill<T, kFewLanes>(ops, P, (cudaStream_t)stream)
                                                        : launch_distill<T, kListMost / 32>(ops, P, (cudaStream_t)stream));
    return launched("launch of the distillation kernel", e);
  });
}

}  // extern "C"
