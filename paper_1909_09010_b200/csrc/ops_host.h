// Host side shared by the translation units of the local-step operators: the handle, errors, launches,
// checks of arguments.
#ifndef GBMUF_CSRC_OPS_HOST_H
#define GBMUF_CSRC_OPS_HOST_H

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <string>

#include "gbmuf.h"

#include "host_common.h"

struct gbmuf_ops {
  int device = 0;
  int num_sms = 0;
  int max_smem = 0;              // opt-in dynamic shared memory per block
  int32_t* d_status = nullptr;
  int tc_clusters[4] = {};       // clusters of 1, 2, 4, 8 CTAs of the linear-layer kernel that fit at once
  int loss_clusters[2][4] = {};  // clusters of 1, 2, 4, 8 CTAs of the cross-entropy kernel (fp32, bf16) that fit at once
  int distill_clusters[4] = {};         // the same of the distillation kernel
};
// What gbmuf_ops_create does for the kernels of vocab_ops.cu.
__attribute__((visibility("hidden"))) gbmuf_status gbmuf_setup_vocab_ops(gbmuf_ops* ops);

namespace {

gbmuf_status refuse(gbmuf_status st, const std::string& msg) {
  gbmuf_set_thread_error(msg);
  return st;
}
gbmuf_status invalid(const std::string& msg) { return refuse(GBMUF_ERR_INVALID_ARG, msg); }
gbmuf_status cuda_refuse(const char* what, cudaError_t e) {
  return refuse(GBMUF_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}
// No C++ exception (an allocation that fails) leaves an entry point.
template <typename F> gbmuf_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return GBMUF_ERR_ALLOC;
  }
}

// Every kernel of this file is launched as a programmatic dependent of the work before it in the
// stream: its blocks may become resident while that ends, and it waits (grid_dependency_wait) before
// it touches memory.  In clusters of `cluster` blocks.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), unsigned grid, unsigned cluster, int threads, uint32_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem;
  cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
gbmuf_status launched(const char* what, cudaError_t e) { return e == cudaSuccess ? GBMUF_OK : cuda_refuse(what, e); }

size_t size_of(int32_t dtype) { return dtype == GBMUF_F32 ? 4 : 2; }
constexpr int64_t kMostDim = 0x7fffffff - 0xffff;     // indices stay in 32 bits past the last tile
bool is_dtype(int32_t d) { return d == GBMUF_F32 || d == GBMUF_BF16; }

// A [rows][cols] operand: NULL only where allowed, aligned to its elements, rows that do not
// overlap, extent within 63 bits.  Empty ones are not looked at.
const char* check_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, bool optional) {
  if (!p) return optional || rows == 0 || cols == 0 ? nullptr : "is NULL";
  if ((uintptr_t)p % size_of(dtype) != 0) return "is not aligned to its element type";
  if (rows > 0 && cols > 0 && ld < cols) return "has a row stride below its columns";
  if ((rows > 1 && ld > ((int64_t)1 << 40)) || (__int128)rows * std::max(ld, cols) > ((__int128)1 << 56)) return "has an extent above 2^56 elements";
  return nullptr;
}
#define CHECK_MATRIX(name, p, rows, cols, ld, dtype, optional)                                   \
  if (const char* why = check_matrix(p, rows, cols, ld, dtype, optional)) return invalid(std::string(name " ") + why)

#define DISPATCH_DTYPE(dtype, T, ...)                       \
  if ((dtype) == GBMUF_F32) { using T = float; __VA_ARGS__; } \
  else { using T = __nv_bfloat16; __VA_ARGS__; }

// How many clusters of 1, 2, 4 and 8 blocks of a kernel the GPU holds at once.
template <typename K> cudaError_t count_clusters(K kernel, int threads, uint32_t smem, int blocks, int (&clusters)[4]) {
  cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  for (int i = 0; i < 4 && e == cudaSuccess; ++i) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1u << i; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(blocks >> i << i)); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&clusters[i], kernel, &cfg);
    if (clusters[i] < 1) clusters[i] = 1;
  }
  return e;
}

}  // namespace

#endif  // GBMUF_CSRC_OPS_HOST_H
