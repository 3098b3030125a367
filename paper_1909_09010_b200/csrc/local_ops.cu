// libgbmuf: the operators of a worker's local step -- linear layers with their gradients, the loss,
// the gradient norm and clipping.  The interface is the last section of include/gbmuf.h; this file
// holds the host side and the C ABI, the kernels live in the headers it includes:
//   linear_epilogue.cuh  activations, and what happens to a finished sum of a matrix product
//   linear_simt.cuh      matrix products on the fp32 units for any strides, column sums
//   cross_entropy.cuh    cross-entropy over a vocabulary with its gradient
//   grad_clip.cuh        norms over many tensors and the clipped copies

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <limits>
#include <new>
#include <numeric>
#include <string>
#include <vector>

#include "gbmuf.h"

#include "host_common.h"
#include "primitives.cuh"
#include "linear_epilogue.cuh"
#include "linear_simt.cuh"
#include "cross_entropy.cuh"
#include "grad_clip.cuh"

struct gbmuf_ops {
  int device = 0;
  int num_sms = 0;
  int32_t* d_status = nullptr;
};

struct gbmuf_clip {
  int device = 0, groups = 0, num_sms = 0;
  int64_t count = 0;             // tensors with elements
  long long chunks = 0;
  int blocks = 0;
  void* table = nullptr;         // [ClipTensor][slots][partial sums]
  size_t table_bytes = 0, slots_off = 0, partial_off = 0;
  WorkMarks work;
};

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

size_t size_of(int32_t dtype) { return dtype == GBMUF_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == GBMUF_F32 || d == GBMUF_BF16; }

// A [rows][cols] operand: NULL only where allowed, aligned to its elements, rows that do not
// overlap, extent within 63 bits.  Empty ones are not looked at.
const char* check_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, bool optional) {
  if (!p) return optional || rows == 0 || cols == 0 ? nullptr : "is NULL";
  if ((uintptr_t)p % size_of(dtype) != 0) return "is not aligned to its element type";
  if (rows > 0 && cols > 0 && ld < cols) return "has a row stride below its columns";
  if (ld > ((int64_t)1 << 40)) return "has a row stride above 2^40";
  return nullptr;
}
#define CHECK_MATRIX(name, p, rows, cols, ld, dtype, optional)                                   \
  if (const char* why = check_matrix(p, rows, cols, ld, dtype, optional)) return invalid(std::string(name " ") + why)

gbmuf_status check_sizes(const gbmuf_ops* ops, int64_t rows, int64_t n_in, int64_t n_out, int32_t dtype, int32_t act) {
  if (!ops) return invalid("ops is NULL");
  if (rows < 0 || n_in < 0 || n_out < 0) return invalid("rows, n_in and n_out must not be negative");
  if (rows > 0x7fffffff || n_in > 0x7fffffff || n_out > 0x7fffffff)
    return refuse(GBMUF_ERR_UNSUPPORTED, "rows, n_in and n_out must be below 2^31");
  if (!is_dtype(dtype)) return invalid("dtype must be GBMUF_F32 or GBMUF_BF16");
  if (act < GBMUF_ACT_NONE || act > GBMUF_ACT_SIGMOID) return invalid("unknown activation");
  return GBMUF_OK;
}

template <int KIND, typename T, typename TO>
void launch_simt(const gbmuf_ops* ops, const SimtParams& P, cudaStream_t st) {
  const long long tiles = ((P.C + 63) / 64) * ((P.R + 63) / 64);
  const int grid = (int)std::min<long long>(tiles, (long long)ops->num_sms * 8);
  linear_simt_kernel<KIND, T, TO><<<grid, 256, 0, st>>>(P);
}

gbmuf_status check_forward(const gbmuf_ops* ops, const gbmuf_linear_forward_args* a) {
  if (!a) return invalid("args is NULL");
  if (gbmuf_status st = check_sizes(ops, a->rows, a->n_in, a->n_out, a->dtype, a->activation)) return st;
  CHECK_MATRIX("x", a->x, a->rows, a->n_in, a->ld_x, a->dtype, false);
  CHECK_MATRIX("w", a->w, a->n_out, a->n_in, a->ld_w, a->dtype, false);
  CHECK_MATRIX("bias", a->bias, 1, a->n_out, a->n_out, a->dtype, true);
  CHECK_MATRIX("residual", a->residual, a->rows, a->n_out, a->ld_residual, a->dtype, true);
  CHECK_MATRIX("y", a->y, a->rows, a->n_out, a->ld_y, a->dtype, false);
  CHECK_MATRIX("z", a->z, a->rows, a->n_out, a->ld_z, a->dtype, true);
  return GBMUF_OK;
}

gbmuf_status check_backward_input(const gbmuf_ops* ops, const gbmuf_linear_backward_input_args* a) {
  if (!a) return invalid("args is NULL");
  if (gbmuf_status st = check_sizes(ops, a->rows, a->n_in, a->n_out, a->dtype, a->activation)) return st;
  CHECK_MATRIX("dz", a->dz, a->rows, a->n_out, a->ld_dz, a->dtype, false);
  CHECK_MATRIX("w", a->w, a->n_out, a->n_in, a->ld_w, a->dtype, false);
  CHECK_MATRIX("residual", a->residual, a->rows, a->n_in, a->ld_residual, a->dtype, true);
  CHECK_MATRIX("z_prev", a->z_prev, a->rows, a->n_in, a->ld_z_prev, a->dtype, a->dz_prev == nullptr);
  CHECK_MATRIX("dx", a->dx, a->rows, a->n_in, a->ld_dx, a->dtype, a->dz_prev != nullptr);
  CHECK_MATRIX("dz_prev", a->dz_prev, a->rows, a->n_in, a->ld_dz_prev, a->dtype, true);
  return GBMUF_OK;
}

gbmuf_status check_backward_weight(const gbmuf_ops* ops, const gbmuf_linear_backward_weight_args* a) {
  if (!a) return invalid("args is NULL");
  if (gbmuf_status st = check_sizes(ops, a->rows, a->n_in, a->n_out, a->dtype, 0)) return st;
  if (!is_dtype(a->grad_dtype)) return invalid("grad_dtype must be GBMUF_F32 or GBMUF_BF16");
  CHECK_MATRIX("dz", a->dz, a->rows, a->n_out, a->ld_dz, a->dtype, false);
  CHECK_MATRIX("x", a->x, a->rows, a->n_in, a->ld_x, a->dtype, a->dw == nullptr);
  CHECK_MATRIX("dw", a->dw, a->n_out, a->n_in, a->ld_dw, a->grad_dtype, a->dbias != nullptr);
  CHECK_MATRIX("dbias", a->dbias, 1, a->n_out, a->n_out, a->grad_dtype, true);
  return GBMUF_OK;
}

gbmuf_status launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? GBMUF_OK : cuda_refuse(what, e);
}

#define DISPATCH_DTYPE(dtype, T, ...)                       \
  if ((dtype) == GBMUF_F32) { using T = float; __VA_ARGS__; } \
  else { using T = __nv_bfloat16; __VA_ARGS__; }

template <typename T, typename TO>
void backward_weight(const gbmuf_ops* ops, const gbmuf_linear_backward_weight_args* a, cudaStream_t st) {
  if (a->dw && a->n_in > 0) {
    SimtParams P{};
    P.a = a->dz; P.sa_r = 1; P.sa_k = a->ld_dz;
    P.b = a->x; P.sb_c = 1; P.sb_k = a->ld_x;
    P.R = a->n_out; P.C = a->n_in; P.K = a->rows;
    P.E.out0 = a->dw; P.E.ld_out0 = a->ld_dw; P.E.accumulate = a->accumulate;
    launch_simt<kWeightGrad, T, TO>(ops, P, st);
  }
  if (a->dbias) {
    const int grid = (int)std::min<long long>((a->n_out + 31) / 32, 65535);
    column_sum_kernel<T, TO><<<grid, 256, 0, st>>>(static_cast<const T*>(a->dz), a->ld_dz, a->rows, a->n_out,
                                                   static_cast<TO*>(a->dbias), a->accumulate);
  }
}

}  // namespace

extern "C" {

gbmuf_status gbmuf_ops_create(int32_t device, gbmuf_ops** out) {
  return guarded([&]() -> gbmuf_status {
    if (!out) return invalid("out is NULL");
    if (device < 0) return invalid("device must not be negative");
    DeviceGuard guard(device);
    if (!guard.ok) { cudaGetLastError(); return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed"); }
    gbmuf_ops* ops = new gbmuf_ops;
    ops->device = device;
    cudaError_t e = cudaDeviceGetAttribute(&ops->num_sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaMalloc(&ops->d_status, 256);
    if (e == cudaSuccess) e = cudaMemset(ops->d_status, 0, 256);
    if (e != cudaSuccess) {
      cudaGetLastError();
      cudaFree(ops->d_status);
      delete ops;
      return cuda_refuse("set-up of the local-step operators", e);
    }
    *out = ops;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_ops_device_status(gbmuf_ops* ops, void* stream, int32_t* out) {
  return guarded([&]() -> gbmuf_status {
    if (!ops || !out) return invalid("ops and out must not be NULL");
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    cudaStream_t st = (cudaStream_t)stream;
    if (is_capturing(st)) return refuse(GBMUF_ERR_BAD_STATE, "the status word cannot be read inside a stream capture");
    int32_t v = 0;
    cudaError_t e = cudaMemcpyAsync(&v, ops->d_status, sizeof(v), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaMemsetAsync(ops->d_status, 0, sizeof(v), st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return cuda_refuse("read of the device status word", e);
    *out = v;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_ops_destroy(gbmuf_ops* ops) {
  if (!ops) return GBMUF_OK;
  cudaError_t e = cudaSuccess;
  {
    DeviceGuard guard(ops->device);
    e = guard.ok ? cudaFree(ops->d_status) : cudaErrorInvalidDevice;
  }
  delete ops;
  return e == cudaSuccess ? GBMUF_OK : GBMUF_ERR_CUDA;
}

gbmuf_status gbmuf_linear_forward_workspace(gbmuf_ops* ops, const gbmuf_linear_forward_args* a, int64_t* bytes) {
  return guarded([&]() -> gbmuf_status {
    if (!bytes) return invalid("bytes is NULL");
    if (gbmuf_status st = check_forward(ops, a)) return st;
    *bytes = 0;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_linear_forward(gbmuf_ops* ops, const gbmuf_linear_forward_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (gbmuf_status st = check_forward(ops, a)) return st;
    if (a->rows == 0 || a->n_out == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    SimtParams P{};
    P.a = a->x; P.sa_r = a->ld_x; P.sa_k = 1;
    P.b = a->w; P.sb_c = a->ld_w; P.sb_k = 1;
    P.R = a->rows; P.C = a->n_out; P.K = a->n_in;
    P.E.bias = a->bias; P.E.residual = a->residual; P.E.ld_residual = a->ld_residual;
    P.E.out0 = a->y; P.E.ld_out0 = a->ld_y; P.E.out1 = a->z; P.E.ld_out1 = a->ld_z; P.E.act = a->activation;
    DISPATCH_DTYPE(a->dtype, T, (launch_simt<kForward, T, T>(ops, P, (cudaStream_t)stream)));
    return launched("launch of the linear-layer kernel");
  });
}

gbmuf_status gbmuf_linear_backward_input_workspace(gbmuf_ops* ops, const gbmuf_linear_backward_input_args* a,
                                                   int64_t* bytes) {
  return guarded([&]() -> gbmuf_status {
    if (!bytes) return invalid("bytes is NULL");
    if (gbmuf_status st = check_backward_input(ops, a)) return st;
    *bytes = 0;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_linear_backward_input(gbmuf_ops* ops, const gbmuf_linear_backward_input_args* a,
                                         void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (gbmuf_status st = check_backward_input(ops, a)) return st;
    if (a->rows == 0 || a->n_in == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    SimtParams P{};
    P.a = a->dz; P.sa_r = a->ld_dz; P.sa_k = 1;
    P.b = a->w; P.sb_c = 1; P.sb_k = a->ld_w;
    P.R = a->rows; P.C = a->n_in; P.K = a->n_out;
    P.E.residual = a->residual; P.E.ld_residual = a->ld_residual; P.E.z_in = a->z_prev; P.E.ld_z_in = a->ld_z_prev;
    P.E.out0 = a->dx; P.E.ld_out0 = a->ld_dx; P.E.out1 = a->dz_prev; P.E.ld_out1 = a->ld_dz_prev;
    P.E.act = a->activation;
    DISPATCH_DTYPE(a->dtype, T, (launch_simt<kInputGrad, T, T>(ops, P, (cudaStream_t)stream)));
    return launched("launch of the input-gradient kernel");
  });
}

gbmuf_status gbmuf_linear_backward_weight_workspace(gbmuf_ops* ops, const gbmuf_linear_backward_weight_args* a,
                                                    int64_t* bytes) {
  return guarded([&]() -> gbmuf_status {
    if (!bytes) return invalid("bytes is NULL");
    if (gbmuf_status st = check_backward_weight(ops, a)) return st;
    *bytes = 0;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_linear_backward_weight(gbmuf_ops* ops, const gbmuf_linear_backward_weight_args* a,
                                          void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (gbmuf_status st = check_backward_weight(ops, a)) return st;
    if (a->n_out == 0 || (a->accumulate && a->rows == 0)) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    DISPATCH_DTYPE(a->dtype, T,
                   DISPATCH_DTYPE(a->grad_dtype, TO, (backward_weight<T, TO>(ops, a, (cudaStream_t)stream))));
    return launched("launch of the weight-gradient kernels");
  });
}

gbmuf_status gbmuf_activation_backward(gbmuf_ops* ops, int64_t rows, int64_t cols, int32_t dtype,
                                       int32_t activation, const void* dy, int64_t ld_dy, const void* z,
                                       int64_t ld_z, void* dz, int64_t ld_dz, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (gbmuf_status st = check_sizes(ops, rows, cols, 0, dtype, activation)) return st;
    CHECK_MATRIX("dy", dy, rows, cols, ld_dy, dtype, false);
    CHECK_MATRIX("z", z, rows, cols, ld_z, dtype, false);
    CHECK_MATRIX("dz", dz, rows, cols, ld_dz, dtype, false);
    if (rows == 0 || cols == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    const int grid = (int)std::min<long long>((rows * cols + 255) / 256, (long long)ops->num_sms * 16);
    DISPATCH_DTYPE(dtype, T, (activation_backward_kernel<T><<<grid, 256, 0, (cudaStream_t)stream>>>(
        static_cast<const T*>(dy), ld_dy, static_cast<const T*>(z), ld_z, static_cast<T*>(dz), ld_dz, rows, cols,
        activation)));
    return launched("launch of the activation-gradient kernel");
  });
}

gbmuf_status gbmuf_cross_entropy(gbmuf_ops* ops, const gbmuf_cross_entropy_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!ops || !a) return invalid("ops and args must not be NULL");
    if (a->rows < 0 || a->vocab < 0) return invalid("rows and vocab must not be negative");
    if (a->rows > 0x7fffffff || a->vocab > 0x7fffffff)
      return refuse(GBMUF_ERR_UNSUPPORTED, "rows and vocab must be below 2^31");
    if (a->rows > 0 && a->vocab == 0) return invalid("vocab must not be 0");
    if (!is_dtype(a->dtype)) return invalid("dtype must be GBMUF_F32 or GBMUF_BF16");
    if (!(a->scale == a->scale)) return invalid("scale must not be NaN");
    CHECK_MATRIX("logits", a->logits, a->rows, a->vocab, a->ld_logits, a->dtype, false);
    CHECK_MATRIX("dlogits", a->dlogits, a->rows, a->vocab, a->ld_dlogits, a->dtype, true);
    if (a->rows > 0 && !a->targets) return invalid("targets is NULL");
    if ((uintptr_t)a->targets % 8 != 0) return invalid("targets is not aligned to its element type");
    if (((uintptr_t)a->row_weight | (uintptr_t)a->loss | (uintptr_t)a->lse) % 4 != 0)
      return invalid("row_weight, loss or lse is not aligned to its element type");
    if (a->dlogits == a->logits && a->dlogits && a->ld_dlogits != a->ld_logits)
      return invalid("dlogits in place of the logits needs their row stride");
    if (a->rows == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    LossParams P{};
    P.logits = a->logits; P.targets = a->targets; P.row_weight = a->row_weight;
    P.loss = a->loss; P.lse = a->lse; P.dlogits = a->dlogits;
    P.rows = a->rows; P.vocab = a->vocab; P.ld = a->ld_logits; P.ld_d = a->ld_dlogits;
    P.ignore_index = a->ignore_index; P.scale = a->scale; P.status = ops->d_status;
    const int grid = (int)std::min<long long>(a->rows, (long long)ops->num_sms * 8);
    DISPATCH_DTYPE(a->dtype, T, (cross_entropy_kernel<T><<<grid, 256, 0, (cudaStream_t)stream>>>(P)));
    return launched("launch of the cross-entropy kernel");
  });
}

gbmuf_status gbmuf_clip_set_tensors(gbmuf_clip* h, int64_t count, const gbmuf_grad_tensor* tensors) {
  return guarded([&]() -> gbmuf_status {
    if (!h) return invalid("handle is NULL");
    if (count < 0 || count > (1 << 24)) return invalid("count must be 0 .. 2^24");
    if (count > 0 && !tensors) return invalid("tensors is NULL");
    std::vector<int64_t> order;
    for (int64_t i = 0; i < count; ++i) {
      const gbmuf_grad_tensor& t = tensors[i];
      if (t.rows < 0 || t.cols < 0 || t.rows > ((int64_t)1 << 40) || t.cols > ((int64_t)1 << 40) ||
          (t.cols > 0 && t.rows > ((int64_t)1 << 40) / t.cols))
        return invalid("a tensor's rows or cols are negative, or it has more than 2^40 elements");
      if (t.group < 0 || t.group >= h->groups) return invalid("a tensor's group is outside 0 .. groups-1");
      if (!is_dtype(t.dtype)) return invalid("dtype must be GBMUF_F32 or GBMUF_BF16");
      if (t.out && t.out_dtype != GBMUF_F32 && t.out_dtype != t.dtype)
        return invalid("out must be fp32 or of the gradient's type");
      CHECK_MATRIX("grad", t.grad, t.rows, t.cols, t.ld_grad, t.dtype, false);
      CHECK_MATRIX("out", t.out, t.rows, t.cols, t.ld_out, t.out ? t.out_dtype : t.dtype, true);
      if (t.out == t.grad && t.out && (t.out_dtype != t.dtype || (t.rows > 1 && t.ld_out != t.ld_grad)))
        return invalid("out in place of the gradient needs its type and row stride");
      if (t.rows > 0 && t.cols > 0) order.push_back(i);
    }
    std::stable_sort(order.begin(), order.end(),
                     [&](int64_t i, int64_t j) { return tensors[i].group < tensors[j].group; });
    std::vector<ClipTensor> table(order.size());
    std::vector<long long> group_first(h->groups, -1), group_end(h->groups, -1);
    std::vector<int> group_run(h->groups, 0);
    long long chunks = 0;
    int run = -1;
    for (size_t i = 0; i < order.size(); ++i) {
      const gbmuf_grad_tensor& t = tensors[order[i]];
      if (i == 0 || tensors[order[i - 1]].group != t.group) ++run;
      ClipTensor& d = table[i];
      d.grad = t.grad; d.out = t.out; d.n = t.rows * t.cols; d.cols = t.cols;
      // a tensor of one row, or of rows that follow one another, is one run of elements
      d.ld_grad = t.rows == 1 ? t.cols : t.ld_grad;
      d.ld_out = t.rows == 1 ? t.cols : t.ld_out;
      d.dtype = t.dtype; d.out_dtype = t.out_dtype; d.group = t.group; d.run = run; d.chunk0 = chunks;
      if (group_first[t.group] < 0) { group_first[t.group] = chunks; group_run[t.group] = run; }
      chunks += (d.n + kClipChunk - 1) / kClipChunk;
      group_end[t.group] = chunks;
    }
    const int blocks = (int)std::max<long long>(1, std::min<long long>(chunks, (long long)h->num_sms * 4));
    std::vector<int> slots(2 * (size_t)h->groups, 0);
    auto block_of = [&](long long c) {      // the block whose chunks [b C / G, (b + 1) C / G) hold c
      long long b = c * blocks / chunks;
      while (chunks * (b + 1) / blocks <= c) ++b;
      while (chunks * b / blocks > c) --b;
      return (int)b;
    };
    for (int g = 0; g < h->groups; ++g)
      if (group_first[g] >= 0) {
        const int b0 = block_of(group_first[g]), b1 = block_of(group_end[g] - 1);
        slots[2 * g] = b0 + group_run[g];
        slots[2 * g + 1] = b1 - b0 + 1;
      }
    DeviceGuard guard(h->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    const size_t slots_off = (table.size() * sizeof(ClipTensor) + 255) / 256 * 256;
    const size_t partial_off = slots_off + (slots.size() * sizeof(int) + 255) / 256 * 256;
    const size_t bytes = partial_off + ((size_t)blocks + h->groups) * sizeof(double);
    cudaError_t e = h->work.wait();
    if (e != cudaSuccess) return cuda_refuse("wait for the handle's earlier work", e);
    if (bytes > h->table_bytes) {
      void* fresh = nullptr;
      e = cudaMalloc(&fresh, bytes);
      if (e != cudaSuccess) { cudaGetLastError(); return refuse(GBMUF_ERR_ALLOC, "table of the gradient tensors"); }
      cudaFree(h->table);
      h->table = fresh;
      h->table_bytes = bytes;
    }
    std::vector<unsigned char> image(partial_off, 0);
    if (!table.empty()) memcpy(image.data(), table.data(), table.size() * sizeof(ClipTensor));
    if (!slots.empty()) memcpy(image.data() + slots_off, slots.data(), slots.size() * sizeof(int));
    h->count = 0;                            // no usable table until the upload has succeeded
    h->chunks = 0;
    if (!image.empty()) e = cudaMemcpy(h->table, image.data(), image.size(), cudaMemcpyHostToDevice);
    if (e != cudaSuccess) return cuda_refuse("upload of the gradient tensors' table", e);
    h->count = (int64_t)table.size(); h->chunks = chunks; h->blocks = blocks;
    h->slots_off = slots_off; h->partial_off = partial_off;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_clip_create(int32_t device, int32_t groups, int64_t count, const gbmuf_grad_tensor* tensors,
                               gbmuf_clip** out) {
  return guarded([&]() -> gbmuf_status {
    if (!out) return invalid("out is NULL");
    if (device < 0) return invalid("device must not be negative");
    if (groups < 1 || groups > 65536) return invalid("groups must be 1 .. 65536");
    DeviceGuard guard(device);
    if (!guard.ok) { cudaGetLastError(); return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed"); }
    gbmuf_clip* h = new gbmuf_clip;
    h->device = device; h->groups = groups;
    gbmuf_status st = GBMUF_OK;
    const cudaError_t e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) { cudaGetLastError(); st = cuda_refuse("device properties", e); }
    if (st == GBMUF_OK) st = gbmuf_clip_set_tensors(h, count, tensors);
    if (st != GBMUF_OK) { cudaFree(h->table); delete h; return st; }
    *out = h;
    return GBMUF_OK;
  });
}

static gbmuf_status clip_run(gbmuf_clip* h, bool scale, float max_norm, float* norms, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!h) return invalid("handle is NULL");
    if (!norms || (uintptr_t)norms % 4 != 0) return invalid("norms must be a device pointer to fp32");
    if (!(max_norm == max_norm)) return invalid("max_norm must not be NaN");
    DeviceGuard guard(h->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    cudaStream_t st = (cudaStream_t)stream;
    ClipParams P{};
    unsigned char* const base = static_cast<unsigned char*>(h->table);
    P.tensors = reinterpret_cast<const ClipTensor*>(base);
    P.slots = reinterpret_cast<const int*>(base + h->slots_off);
    P.partial = reinterpret_cast<double*>(base + h->partial_off);
    P.norms = norms; P.chunks = h->chunks; P.count = (int)h->count; P.groups = h->groups; P.blocks = h->blocks;
    P.max_norm = max_norm;
    if (h->chunks > 0) clip_norm_kernel<<<h->blocks, 256, 0, st>>>(P);
    if (scale) clip_scale_kernel<<<h->blocks, 256, 0, st>>>(P);
    else clip_finish_kernel<<<std::min(h->groups, h->num_sms), 256, 0, st>>>(P);
    const gbmuf_status rc = launched("launch of the gradient-norm kernels");
    if (rc == GBMUF_OK) h->work.note(st);
    return rc;
  });
}

gbmuf_status gbmuf_clip_norms(gbmuf_clip* h, float* norms, void* stream) {
  return clip_run(h, false, 0.0f, norms, stream);
}
gbmuf_status gbmuf_clip_scale(gbmuf_clip* h, float max_norm, float* norms, void* stream) {
  return clip_run(h, true, max_norm, norms, stream);
}

gbmuf_status gbmuf_clip_destroy(gbmuf_clip* h) {
  if (!h) return GBMUF_OK;
  gbmuf_status rc = GBMUF_OK;
  {
    DeviceGuard guard(h->device);
    if (guard.ok) {
      if (h->work.wait() != cudaSuccess) rc = GBMUF_ERR_CUDA;
      h->work.release();
      cudaFree(h->table);
    } else {
      rc = GBMUF_ERR_CUDA;
    }
  }
  delete h;
  return rc;
}

}  // extern "C"
