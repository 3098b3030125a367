// libgbmuf: the operators of a worker's local step -- linear layers with their gradients, the loss,
// the gradient norm and clipping.  The interface is the last section of include/gbmuf.h; this file
// holds the host side and the C ABI, the kernels live in the headers it includes:
//   packed_math.cuh      two fp32 operations per instruction
//   linear_epilogue.cuh  activations, and what happens to a finished sum of a matrix product
//   linear_tc.cuh        matrix products on the tensor cores
//   linear_pack.cuh      operands that cannot be read in place: other alignments, fp32 as bf16 parts
//   linear_rows.cuh      the layer for a few rows, on the fp32 units
//   column_sum.cuh       column sums (bias gradients), gradient of an activation by itself
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
#include <type_traits>
#include <vector>

#include "gbmuf.h"

#include "host_common.h"
#include "primitives.cuh"
#include "packed_math.cuh"
#include "linear_epilogue.cuh"
#include "linear_pack.cuh"
#include "linear_tc.cuh"
#include "linear_rows.cuh"
#include "column_sum.cuh"
#include "cross_entropy.cuh"
#include "grad_clip.cuh"

struct gbmuf_ops {
  int device = 0;
  int num_sms = 0;
  int max_smem = 0;              // opt-in dynamic shared memory per block
  int32_t* d_status = nullptr;
  int tc_clusters[4] = {};       // clusters of 1, 2, 4, 8 CTAs of the linear-layer kernel that fit at once
  int loss_clusters[2][4] = {};  // clusters of 1, 2, 4, 8 CTAs of the cross-entropy kernel (fp32, bf16) that fit at once
};

struct gbmuf_clip {
  int device = 0, groups = 0, num_sms = 0;
  bool ready = false;            // the table holds what set_tensors was last given
  int64_t count = 0;             // tensors with elements
  long long chunks = 0;
  int blocks = 0;
  int32_t* d_status = nullptr;
  void* table = nullptr;         // [ClipEntry][slots][partial sums]
  size_t table_bytes = 0, slots_off = 0, partial_off = 0;
  bool in_graph = false;         // a stream capture has recorded the table's address and sizes
  std::vector<void*> earlier;    // tables that graphs may still read
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

gbmuf_status check_sizes(const gbmuf_ops* ops, int64_t rows, int64_t n_in, int64_t n_out, int32_t dtype, int32_t act) {
  if (!ops) return invalid("ops is NULL");
  if (rows < 0 || n_in < 0 || n_out < 0) return invalid("rows, n_in and n_out must not be negative");
  if (rows > kMostDim || n_in > kMostDim || n_out > kMostDim)
    return refuse(GBMUF_ERR_UNSUPPORTED, "rows, n_in and n_out must be at most 2^31 - 2^16");
  if (!is_dtype(dtype)) return invalid("dtype must be GBMUF_F32 or GBMUF_BF16");
  if (act < GBMUF_ACT_NONE || act > GBMUF_ACT_SIGMOID) return invalid("unknown activation");
  return GBMUF_OK;
}

#define DISPATCH_DTYPE(dtype, T, ...)                       \
  if ((dtype) == GBMUF_F32) { using T = float; __VA_ARGS__; } \
  else { using T = __nv_bfloat16; __VA_ARGS__; }

// An operand as it lies in memory: [outer][inner] of the call's type, row stride ld; k_inner: the
// summed index is the inner one.
struct Operand {
  const void* p;
  long long outer, inner, ld;
  bool k_inner;
};
// A product of two operands: result [R][C], K terms.
struct Product {
  Operand a, b;
  long long R, C, K;
  int32_t dtype;
  Epilogue E;
};

bool in_place(const Operand& o, int32_t dtype) {
  return dtype == GBMUF_BF16 && (uintptr_t)o.p % 16 == 0 && (o.outer <= 1 || (o.ld % 8 == 0 && o.ld < ((long long)1 << 38)));
}
long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }
long long packed_bytes(const Operand& o, int32_t dtype) {
  return in_place(o, dtype) ? 0 : round_up((dtype == GBMUF_F32 ? 3 : 1) * o.outer * round_up(o.inner, 8) * 2, 256);
}
long long product_workspace(const Product& q) {
  return q.K == 0 || q.R == 0 || q.C == 0 ? 0 : packed_bytes(q.a, q.dtype) + packed_bytes(q.b, q.dtype);
}

PackJob pack_job(const gbmuf_ops* ops, const Operand& o, int32_t dtype, void* dst) {
  PackJob j{};
  if (in_place(o, dtype)) return j;
  j.src = o.p; j.dst = static_cast<__nv_bfloat16*>(dst); j.ld = o.ld; j.outer = o.outer; j.inner = o.inner; j.ld_dst = round_up(o.inner, 8);
  j.vec = (uintptr_t)o.p % 16 == 0 && (o.outer <= 1 || o.ld * (long long)size_of(dtype) % 16 == 0);
  j.blocks = (int)std::min<long long>((o.outer * (j.ld_dst / 8) + 255) / 256, (long long)ops->num_sms * 16);
  return j;
}

// Tensor map of an operand (packed at `packed` if it cannot be read in place): [parts][outer][inner],
// boxes of 64 inner elements by `box` outer ones.
gbmuf_status operand_map(const Operand& o, int32_t dtype, const void* packed, int box, CUtensorMap* map) {
  const EncodeTiledFn encode = encode_tiled_fn();
  if (!encode) return refuse(GBMUF_ERR_CUDA, "the driver does not provide cuTensorMapEncodeTiled");
  const bool here = in_place(o, dtype);
  const long long ld = here && o.outer > 1 ? o.ld : round_up(o.inner, 8);
  const cuuint64_t dim[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)(dtype == GBMUF_F32 ? 3 : 1)};
  const cuuint64_t stride[2] = {(cuuint64_t)ld * 2, dtype == GBMUF_F32 ? (cuuint64_t)(o.outer * ld) * 2 : (cuuint64_t)ld * 2};
  const cuuint32_t boxes[3] = {64, (cuuint32_t)box, 1}, one[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(here ? o.p : packed), dim, stride, boxes,
                            one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return refuse(GBMUF_ERR_CUDA, "cuTensorMapEncodeTiled failed with code " + std::to_string((int)r));
  return GBMUF_OK;
}

// Whether the epilogue's matrices can be accessed two bf16 columns at a time.
int may_pair(const Product& q) {
  const Epilogue& E = q.E;
  const void* const p[] = {E.residual, E.z_in, E.out0, E.out1};
  const long long ld[] = {E.ld_residual, E.ld_z_in, E.ld_out0, E.ld_out1};
  bool ok = q.C % 2 == 0;
  for (int i = 0; i < 4; ++i) ok = ok && (!p[i] || ((uintptr_t)p[i] % 4 == 0 && (q.R == 1 || ld[i] % 2 == 0)));
  return ok;
}

// Tile width, CTAs that share a tile's steps, CTAs that share a tile: the choice with the least time
// by a model whose eight constants were fitted to 180 measured products of 12 to 100,000 rows, columns
// and terms in both types (its choice was 0.8 % above the best one on average, 15 % at worst; no sum along
// a vocabulary among them).  The 1.45 for pairs with a strided A says what was measured, not why.
struct TcShape { int bn, split, pair; };
TcShape choose_shape(const gbmuf_ops* ops, const Product& q, int parts, bool rows_64, bool a_strided) {
  TcShape best{64, 1, 1};
  double best_t = 1e300;
  const long long ksteps = (q.K + 63) / 64;
  for (int pair = 1; pair <= 2; ++pair)
    for (int bn = pair == 2 ? 128 : rows_64 ? 64 : 32; bn <= (parts == 3 && pair == 1 ? 128 : 256); bn *= 2)
      for (int log = 0; log <= (pair == 2 ? 0 : 3); ++log) {
        const int split = 1 << log;
        const long long tiles = ((q.C + 128 * pair - 1) / (128 * pair)) * ((q.R + bn - 1) / bn);
        const long long fit = ops->tc_clusters[pair == 2 ? 1 : log];
        if (split > 1 && (split * 2 > ksteps || tiles > fit)) break;
        const double waves = (double)((tiles + fit - 1) / fit);
        // a step takes as long as its operands take to arrive, the epilogue as long as the tile is wide
        double step = std::max(100.0, parts * tc_stage_bytes(bn, pair) / 126.0);
        if (pair == 2 && a_strided) step *= 1.45;
        const double sums = 1000.0 + (double)((ksteps + split - 1) / split) * step, epilogue = 15.0 * bn / split;
        double t = split > 1 ? waves * (sums + 1100.0 + 19.0 * bn) : waves * std::max(sums, epilogue);
        t += epilogue + (pair == 2 ? 2000.0 : 0.0);
        if (t < best_t) { best_t = t; best = {bn, split, pair}; }
      }
  return best;
}

template <int KIND, typename T, typename TO, int PARTS, int BN, int PAIR>
gbmuf_status launch_tc(const gbmuf_ops* ops, TcParams& P, const CUtensorMap& ma, const CUtensorMap& mb, cudaStream_t st) {
  const auto kernel = linear_tc_kernel<KIND, T, TO, PARTS, BN, PAIR>;
  P.stages = std::min<int>(kTcMaxStages, (ops->max_smem - 1024 - (int)kTcHead) / (int)tc_stage_bytes(BN, PAIR));
  const uint32_t smem = tc_smem_bytes(BN, PAIR, P.stages);
  static std::atomic<uint64_t> ready{0};                  // devices on which the limit has been raised
  const uint64_t bit = 1ull << (ops->device & 63);
  if (!(ready.load() & bit)) {
    const cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ops->max_smem);
    if (e != cudaSuccess) return cuda_refuse("shared-memory limit of the linear-layer kernel", e);
    if (ops->device < 64) ready.fetch_or(bit);
  }
  const int at_once = P.split > 1 ? P.tiles : std::min(P.tiles, ops->num_sms / PAIR);     // a split tile: one per cluster
  P.tile_step = at_once; P.step_c = at_once / P.tiles_r; P.step_r = at_once % P.tiles_r;
  const unsigned grid = (unsigned)(at_once * PAIR * P.split);
  return launched("launch of the linear-layer kernel", launch(kernel, grid, (unsigned)(PAIR * P.split), kTcThreads, smem, st, ma, mb, P));
}

// Runs a product: operands that cannot be read in place are packed into the workspace first.
template <int KIND, typename T, typename TO, int PARTS>
gbmuf_status run_product(const gbmuf_ops* ops, Product q, void* workspace, int64_t workspace_bytes, cudaStream_t st) {
  const long long need = product_workspace(q);
  if (need > workspace_bytes || (need > 0 && (!workspace || (uintptr_t)workspace % 256 != 0)))
    return invalid("workspace must be 256-byte aligned device memory of at least " + std::to_string(need) + " bytes");
  q.E.pairs = may_pair(q);
  TcParams P{};
  P.E = q.E; P.status = ops->d_status; P.R = (int)q.R; P.C = (int)q.C;
  P.ksteps = (int)((q.K + kTcK - 1) / kTcK);
  const TcShape shape = choose_shape(ops, q, PARTS, KIND == kWeightGrad, KIND != kForward);
  P.split = shape.split;
  P.tiles_r = (int)((q.R + shape.bn - 1) / shape.bn);
  const long long tiles = (long long)P.tiles_r * ((q.C + 128 * shape.pair - 1) / (128 * shape.pair));
  if (tiles > 0x3fffffff) return refuse(GBMUF_ERR_UNSUPPORTED, "more than 2^30 tiles");
  P.tiles = (int)tiles;
  CUtensorMap ma{}, mb{};
  if (q.K > 0) {
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    void* const pa = ws;
    void* const pb = ws + packed_bytes(q.a, q.dtype);
    const PackJob ja = pack_job(ops, q.a, q.dtype, pa), jb = pack_job(ops, q.b, q.dtype, pb);
    if (ja.blocks + jb.blocks > 0) {
      const cudaError_t e = launch(q.dtype == GBMUF_F32 ? pack_kernel<float> : pack_kernel<__nv_bfloat16>, (unsigned)(ja.blocks + jb.blocks), 1,
                                   256, 0, st, ja, jb);
      if (e != cudaSuccess) return cuda_refuse("launch of the operand-packing kernel", e);
    }
    if (gbmuf_status rc = operand_map(q.a, q.dtype, pa, q.a.k_inner ? 128 : 64, &ma)) return rc;
    if (gbmuf_status rc = operand_map(q.b, q.dtype, pb, q.b.k_inner ? shape.bn / shape.pair : 64, &mb)) return rc;
  }
  if (shape.pair == 2)
    return shape.bn == 128 ? launch_tc<KIND, T, TO, PARTS, 128, 2>(ops, P, ma, mb, st)
                           : launch_tc<KIND, T, TO, PARTS, 256, 2>(ops, P, ma, mb, st);
  if constexpr (KIND != kWeightGrad)
    if (shape.bn == 32) return launch_tc<KIND, T, TO, PARTS, 32, 1>(ops, P, ma, mb, st);
  if constexpr (PARTS == 1)
    if (shape.bn == 256) return launch_tc<KIND, T, TO, PARTS, 256, 1>(ops, P, ma, mb, st);
  return shape.bn == 64 ? launch_tc<KIND, T, TO, PARTS, 64, 1>(ops, P, ma, mb, st)
                        : launch_tc<KIND, T, TO, PARTS, 128, 1>(ops, P, ma, mb, st);
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


Product forward_product(const gbmuf_linear_forward_args* a) {
  Product q{};
  q.a = {a->w, a->n_out, a->n_in, a->ld_w, true};
  q.b = {a->x, a->rows, a->n_in, a->ld_x, true};
  q.R = a->rows; q.C = a->n_out; q.K = a->n_in; q.dtype = a->dtype;
  q.E.bias = a->bias; q.E.residual = a->residual; q.E.ld_residual = a->ld_residual;
  q.E.out0 = a->y; q.E.ld_out0 = a->ld_y; q.E.out1 = a->z; q.E.ld_out1 = a->ld_z; q.E.act = a->activation;
  return q;
}

// Whether the few-rows kernel takes a layer.
bool few_rows(const gbmuf_linear_forward_args* a) {
  const int64_t most = a->dtype == GBMUF_F32 ? 16 : 8;
  const int64_t rows = a->rows <= 1 ? 1 : a->rows <= 2 ? 2 : a->rows <= 4 ? 4 : a->rows <= 8 ? 8 : 16;
  return a->rows <= most && rows * ((a->n_in + 7) / 8 * 8) * (int64_t)size_of(a->dtype) <= kRowsMostBytes;
}

template <typename T, int ROWS> gbmuf_status launch_rows(const gbmuf_ops* ops, const RowsParams& P, bool vec, cudaStream_t st) {
  constexpr int NF = ROWS >= 16 ? 2 : 4, per_block = NF * kRowsThreads / 32;
  const uint32_t smem = (uint32_t)(ROWS * ((P.K + 7) / 8 * 8) * (int)sizeof(T));
  const auto kernel = vec ? linear_rows_kernel<T, ROWS, true> : linear_rows_kernel<T, ROWS, false>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsMostBytes);
    if (e != cudaSuccess) return cuda_refuse("shared-memory limit of the few-rows kernel", e);
  }
  const unsigned grid = (unsigned)std::min<long long>(((long long)P.C + per_block - 1) / per_block, ops->num_sms * 2);
  return launched("launch of the few-rows kernel", launch(kernel, grid, 1, kRowsThreads, smem, st, P));
}
template <typename T> gbmuf_status forward_rows(const gbmuf_ops* ops, const gbmuf_linear_forward_args* a, cudaStream_t st) {
  RowsParams P{};
  P.E = forward_product(a).E;
  P.x = a->x; P.w = a->w; P.ld_x = a->ld_x; P.ld_w = a->ld_w;
  P.R = (int)a->rows; P.C = (int)a->n_out; P.K = (int)a->n_in;
  const bool vec = (uintptr_t)a->w % 16 == 0 && (a->n_out == 1 || a->ld_w * (int64_t)sizeof(T) % 16 == 0);
  if (a->rows <= 1) return launch_rows<T, 1>(ops, P, vec, st);
  if (a->rows <= 2) return launch_rows<T, 2>(ops, P, vec, st);
  if (a->rows <= 4) return launch_rows<T, 4>(ops, P, vec, st);
  if (a->rows <= 8) return launch_rows<T, 8>(ops, P, vec, st);
  return launch_rows<T, 16>(ops, P, vec, st);
}

Product input_grad_product(const gbmuf_linear_backward_input_args* a) {
  Product q{};
  q.a = {a->w, a->n_out, a->n_in, a->ld_w, false};
  q.b = {a->dz, a->rows, a->n_out, a->ld_dz, true};
  q.R = a->rows; q.C = a->n_in; q.K = a->n_out; q.dtype = a->dtype;
  q.E.residual = a->residual; q.E.ld_residual = a->ld_residual; q.E.z_in = a->z_prev; q.E.ld_z_in = a->ld_z_prev;
  q.E.out0 = a->dx; q.E.ld_out0 = a->ld_dx; q.E.out1 = a->dz_prev; q.E.ld_out1 = a->ld_dz_prev;
  q.E.act = a->activation;
  return q;
}

Product weight_grad_product(const gbmuf_linear_backward_weight_args* a) {
  Product q{};
  q.a = {a->x, a->rows, a->n_in, a->ld_x, false};
  q.b = {a->dz, a->rows, a->n_out, a->ld_dz, false};
  q.R = a->dw ? a->n_out : 0; q.C = a->n_in; q.K = a->rows; q.dtype = a->dtype;
  q.E.out0 = a->dw; q.E.ld_out0 = a->ld_dw; q.E.accumulate = a->accumulate;
  return q;
}

template <typename T, typename TO>
cudaError_t column_sum(const gbmuf_linear_backward_weight_args* a, cudaStream_t st) {
  const bool vec = (uintptr_t)a->dz % 16 == 0 && a->n_out % (16 / sizeof(T)) == 0 &&
                   (a->rows <= 1 || a->ld_dz * sizeof(T) % 16 == 0);
  const int cols = vec ? 128 / (int)sizeof(T) : 32, rows_at_once = vec ? 32 : 8;
  // a cluster shares the rows of a column tile: as many CTAs as have four rows per thread, 8 at most
  unsigned share = 1;
  while (share < 8 && a->rows >= (long long)share * 2 * rows_at_once * 4) share *= 2;
  const long long tiles = (a->n_out + cols - 1) / cols;
  return launch(vec ? column_sum_kernel<T, TO, true> : column_sum_kernel<T, TO, false>, share * (unsigned)tiles, share, 256, 0, st,
                static_cast<const T*>(a->dz), (long long)a->ld_dz, (long long)a->rows, (long long)a->n_out, static_cast<TO*>(a->dbias),
                (int)a->accumulate);
}

constexpr long long kLossCacheBytes = 64ll << 20;   // of the 126 MB: the gradient passes through as well

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

// Short rows: a warp each.  Longer ones: a cluster of CTAs each, of more CTAs where there are too few
// rows to fill the GPU, or where the slices that are fetched twice would not fit the L2 cache.
template <typename T> cudaError_t launch_loss(const gbmuf_ops* ops, LossParams& P, cudaStream_t st) {
  if (P.vocab <= kWarpVocab) {
    const auto kernel = P.vocab <= 256 ? cross_entropy_warp_kernel<T, 8> : P.vocab <= 1024 ? cross_entropy_warp_kernel<T, 32>
                                                                                           : cross_entropy_warp_kernel<T, kWarpRegs>;
    return launch(kernel, (unsigned)((P.rows + 3) / 4), 1, 128, 0, st, P);
  }
  const long long bytes = P.vocab * (long long)sizeof(T), ctas = (long long)ops->num_sms * kLossBlocksPerSm;
  int log = 0;
  while (log < 3) {
    const long long twice = (bytes - ((long long)kLossKept * kLossChunk << log)) * (ctas >> log);
    const bool few = P.rows << (log + 1) <= ctas && bytes >> (log + 1) >= kLossChunk / 2;
    if (!few && twice < kLossCacheBytes) break;
    ++log;
  }
  P.split = 1 << log;
  const int clusters = (int)std::min<long long>(P.rows, ops->loss_clusters[sizeof(T) == 2][log]);
  return launch(cross_entropy_ring_kernel<T>, (unsigned)(clusters * P.split), (unsigned)P.split, kLossThreads, kLossSmem, st, P);
}

// Reads and clears a status word, once the stream has got there.
gbmuf_status read_status(int device, int32_t* word, void* stream, int32_t* out) {
  DeviceGuard guard(device);
  if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
  cudaStream_t st = (cudaStream_t)stream;
  if (is_capturing(st)) return refuse(GBMUF_ERR_BAD_STATE, "the status word cannot be read inside a stream capture");
  int32_t v = 0;
  cudaError_t e = cudaMemcpyAsync(&v, word, sizeof(v), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(word, 0, sizeof(v), st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return cuda_refuse("read of the device status word", e);
  *out = v;
  return GBMUF_OK;
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
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&ops->max_smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, device);
    const int pairs = ops->num_sms * kLossBlocksPerSm;
    if (e == cudaSuccess) e = count_clusters(cross_entropy_ring_kernel<float>, kLossThreads, kLossSmem, pairs, ops->loss_clusters[0]);
    if (e == cudaSuccess) e = count_clusters(cross_entropy_ring_kernel<__nv_bfloat16>, kLossThreads, kLossSmem, pairs, ops->loss_clusters[1]);
    if (e == cudaSuccess)
      e = count_clusters(linear_tc_kernel<kForward, __nv_bfloat16, __nv_bfloat16, 1, 128, 1>, kTcThreads, (uint32_t)ops->max_smem, ops->num_sms,
                         ops->tc_clusters);
    if (e == cudaSuccess) e = cudaMalloc(&ops->d_status, 256);
    if (e == cudaSuccess) e = cudaMemset(ops->d_status, 0, 256);
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);          // other streams do not wait for the default one
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
    return read_status(ops->device, ops->d_status, stream, out);
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
    *bytes = few_rows(a) ? 0 : product_workspace(forward_product(a));
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_linear_forward(gbmuf_ops* ops, const gbmuf_linear_forward_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (gbmuf_status st = check_forward(ops, a)) return st;
    if (a->rows == 0 || a->n_out == 0) return GBMUF_OK;
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    if (few_rows(a)) { DISPATCH_DTYPE(a->dtype, T, return forward_rows<T>(ops, a, (cudaStream_t)stream)); }
    const Product q = forward_product(a);
    DISPATCH_DTYPE(a->dtype, T, return run_product<kForward, T, T, (sizeof(T) == 4 ? 3 : 1)>(ops, q, a->workspace, a->workspace_bytes, (cudaStream_t)stream));
  });
}

gbmuf_status gbmuf_linear_backward_input_workspace(gbmuf_ops* ops, const gbmuf_linear_backward_input_args* a,
                                                   int64_t* bytes) {
  return guarded([&]() -> gbmuf_status {
    if (!bytes) return invalid("bytes is NULL");
    if (gbmuf_status st = check_backward_input(ops, a)) return st;
    *bytes = product_workspace(input_grad_product(a));
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
    const Product q = input_grad_product(a);
    DISPATCH_DTYPE(a->dtype, T, return run_product<kInputGrad, T, T, (sizeof(T) == 4 ? 3 : 1)>(ops, q, a->workspace, a->workspace_bytes, (cudaStream_t)stream));
  });
}

gbmuf_status gbmuf_linear_backward_weight_workspace(gbmuf_ops* ops, const gbmuf_linear_backward_weight_args* a,
                                                    int64_t* bytes) {
  return guarded([&]() -> gbmuf_status {
    if (!bytes) return invalid("bytes is NULL");
    if (gbmuf_status st = check_backward_weight(ops, a)) return st;
    *bytes = product_workspace(weight_grad_product(a));
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
    cudaStream_t st = (cudaStream_t)stream;
    if (a->dw && a->n_in > 0) {
      const Product q = weight_grad_product(a);
      gbmuf_status rc = GBMUF_OK;
      DISPATCH_DTYPE(a->dtype, T, DISPATCH_DTYPE(a->grad_dtype, TO,
          (rc = run_product<kWeightGrad, TO, TO, (sizeof(T) == 4 ? 3 : 1)>(ops, q, a->workspace, a->workspace_bytes, st))));
      if (rc != GBMUF_OK) return rc;
    }
    if (a->dbias) {
      cudaError_t e = cudaSuccess;
      DISPATCH_DTYPE(a->dtype, T, DISPATCH_DTYPE(a->grad_dtype, TO, (e = column_sum<T, TO>(a, st))));
      if (e != cudaSuccess) return cuda_refuse("launch of the bias-gradient kernel", e);
    }
    return GBMUF_OK;
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
    const unsigned grid = (unsigned)std::min<long long>((rows * cols + 255) / 256, (long long)ops->num_sms * 16);
    cudaError_t e = cudaSuccess;
    DISPATCH_DTYPE(dtype, T, e = launch(activation_backward_kernel<T>, grid, 1, 256, 0, (cudaStream_t)stream, static_cast<const T*>(dy),
                                        (long long)ld_dy, static_cast<const T*>(z), (long long)ld_z, static_cast<T*>(dz), (long long)ld_dz,
                                        (long long)rows, (long long)cols, (int)activation));
    return launched("launch of the activation-gradient kernel", e);
  });
}

gbmuf_status gbmuf_cross_entropy(gbmuf_ops* ops, const gbmuf_cross_entropy_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!ops || !a) return invalid("ops and args must not be NULL");
    if (a->rows < 0 || a->vocab < 0) return invalid("rows and vocab must not be negative");
    if (a->rows > kMostDim || a->vocab > kMostDim)
      return refuse(GBMUF_ERR_UNSUPPORTED, "rows and vocab must be at most 2^31 - 2^16");
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
    cudaError_t e = cudaSuccess;
    DISPATCH_DTYPE(a->dtype, T, e = launch_loss<T>(ops, P, (cudaStream_t)stream));
    return e == cudaSuccess ? GBMUF_OK : cuda_refuse("launch of the cross-entropy kernel", e);
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
    std::vector<ClipEntry> table;
    table.reserve(order.size());
    std::vector<long long> group_first(h->groups, -1), group_end(h->groups, -1);
    std::vector<int> group_run(h->groups, 0);
    long long chunks = 0;
    int run = -1;
    for (size_t i = 0; i < order.size(); ++i) {
      const gbmuf_grad_tensor& t = tensors[order[i]];
      if (i == 0 || tensors[order[i - 1]].group != t.group) ++run;
      // rows that follow one another are one run of elements, long rows are a run each; short
      // strided rows stay together and are read element by element
      const bool whole = t.rows == 1 || (t.ld_grad == t.cols && (!t.out || t.ld_out == t.cols));
      const bool split = !whole && t.cols >= 512;
      const int64_t runs = split ? t.rows : 1;
      if (group_first[t.group] < 0) { group_first[t.group] = chunks; group_run[t.group] = run; }
      if (runs + (int64_t)table.size() > (1 << 26)) return refuse(GBMUF_ERR_UNSUPPORTED, "more than 2^26 runs of elements");
      for (int64_t r = 0; r < runs; ++r) {
        ClipEntry d{};
        d.grad = static_cast<const char*>(t.grad) + r * t.ld_grad * (int64_t)size_of(t.dtype);
        d.out = t.out ? static_cast<char*>(t.out) + r * t.ld_out * (int64_t)size_of(t.out_dtype) : nullptr;
        d.n = split ? t.cols : t.rows * t.cols;
        d.cols = t.cols; d.ld_grad = t.ld_grad; d.ld_out = t.ld_out;
        d.dtype = t.dtype; d.out_dtype = t.out ? t.out_dtype : t.dtype; d.group = t.group; d.run = run; d.chunk0 = chunks;
        d.direct = !whole && !split;
        d.shift = d.direct ? 0 : (int32_t)((uintptr_t)d.grad % 16 / size_of(t.dtype));
        const int64_t ch = kClipSlot / (int64_t)size_of(t.dtype);
        chunks += (d.n + d.shift + ch - 1) / ch;
        table.push_back(d);
      }
      group_end[t.group] = chunks;
    }
    const int blocks = (int)std::max<long long>(1, std::min<long long>(chunks, (long long)h->num_sms * kClipBlocksPerSm));
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
    const size_t slots_off = (table.size() * sizeof(ClipEntry) + 255) / 256 * 256;
    const size_t partial_off = slots_off + (slots.size() * sizeof(int) + 255) / 256 * 256;
    const size_t bytes = partial_off + ((size_t)blocks + h->groups) * sizeof(double);
    cudaError_t e = h->work.wait();
    if (e != cudaSuccess) return cuda_refuse("wait for the handle's earlier work", e);
    if (bytes > h->table_bytes || h->in_graph) {
      if (h->in_graph) h->earlier.reserve(h->earlier.size() + 1);
      void* fresh = nullptr;
      e = cudaMalloc(&fresh, bytes);
      if (e != cudaSuccess) { cudaGetLastError(); return refuse(GBMUF_ERR_ALLOC, "table of the gradient tensors"); }
      if (h->in_graph) h->earlier.push_back(h->table); else cudaFree(h->table);
      h->table = fresh;
      h->table_bytes = bytes;
      h->in_graph = false;
    }
    std::vector<unsigned char> image(partial_off, 0);
    if (!table.empty()) memcpy(image.data(), table.data(), table.size() * sizeof(ClipEntry));
    if (!slots.empty()) memcpy(image.data() + slots_off, slots.data(), slots.size() * sizeof(int));
    h->ready = false;                        // until the upload has succeeded
    if (!image.empty()) e = cudaMemcpy(h->table, image.data(), image.size(), cudaMemcpyHostToDevice);
    // a copy from pageable memory may return before it has landed, and streams other than the default one
    // would not wait for it
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
    if (e != cudaSuccess) return cuda_refuse("upload of the gradient tensors' table", e);
    h->count = (int64_t)table.size(); h->chunks = chunks; h->blocks = blocks;
    h->slots_off = slots_off; h->partial_off = partial_off; h->ready = true;
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
    cudaError_t e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaFuncSetAttribute((const void*)clip_norm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kClipSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute((const void*)clip_scale_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kClipSmem);
    if (e == cudaSuccess) e = cudaMalloc(&h->d_status, 256);
    if (e == cudaSuccess) e = cudaMemset(h->d_status, 0, 256);         // set_tensors waits for it
    if (e != cudaSuccess) { cudaGetLastError(); st = cuda_refuse("set-up of the clipping handle", e); }
    if (st == GBMUF_OK) st = gbmuf_clip_set_tensors(h, count, tensors);
    if (st != GBMUF_OK) { cudaFree(h->d_status); cudaFree(h->table); delete h; return st; }
    *out = h;
    return GBMUF_OK;
  });
}

static gbmuf_status clip_run(gbmuf_clip* h, bool scale, float max_norm, float* norms, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!h) return invalid("handle is NULL");
    if (!norms || (uintptr_t)norms % 4 != 0) return invalid("norms must be a device pointer to fp32");
    if (!(max_norm == max_norm)) return invalid("max_norm must not be NaN");
    if (!h->ready) return refuse(GBMUF_ERR_BAD_STATE, "the last set_tensors failed");
    DeviceGuard guard(h->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    cudaStream_t st = (cudaStream_t)stream;
    ClipParams P{};
    unsigned char* const base = static_cast<unsigned char*>(h->table);
    P.status = h->d_status;
    P.entries = reinterpret_cast<const ClipEntry*>(base);
    P.slots = reinterpret_cast<const int*>(base + h->slots_off);
    P.partial = reinterpret_cast<double*>(base + h->partial_off);
    P.norms = norms; P.chunks = h->chunks; P.count = (int)h->count; P.groups = h->groups; P.blocks = h->blocks;
    P.max_norm = max_norm;
    cudaError_t e = cudaSuccess;
    if (h->chunks > 0) e = launch(clip_norm_kernel, (unsigned)h->blocks, 1, kClipThreads, kClipSmem, st, P);
    if (e == cudaSuccess)
      e = scale ? launch(clip_scale_kernel, (unsigned)h->blocks, 1, kClipThreads, kClipSmem, st, P)
                : launch(clip_finish_kernel, (unsigned)std::min(h->groups, h->num_sms), 1, kClipWorkers, 0, st, P);
    if (e != cudaSuccess) return cuda_refuse("launch of the gradient-norm kernels", e);
    if (!h->work.note(st)) h->in_graph = true;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_clip_norms(gbmuf_clip* h, float* norms, void* stream) {
  return clip_run(h, false, 0.0f, norms, stream);
}
gbmuf_status gbmuf_clip_scale(gbmuf_clip* h, float max_norm, float* norms, void* stream) {
  return clip_run(h, true, max_norm, norms, stream);
}

gbmuf_status gbmuf_clip_device_status(gbmuf_clip* h, void* stream, int32_t* out) {
  return guarded([&]() -> gbmuf_status {
    if (!h || !out) return invalid("handle and out must not be NULL");
    return read_status(h->device, h->d_status, stream, out);
  });
}

gbmuf_status gbmuf_clip_selftest_wait_timeout(gbmuf_clip* h, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (!h) return invalid("handle is NULL");
    DeviceGuard guard(h->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    clip_expired_wait_kernel<<<1, 32, 0, (cudaStream_t)stream>>>(h->d_status);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) h->work.note((cudaStream_t)stream);
    return launched("launch of the wait-timeout self-test", e);
  });
}

gbmuf_status gbmuf_clip_destroy(gbmuf_clip* h) {
  if (!h) return GBMUF_OK;
  gbmuf_status rc = GBMUF_OK;
  {
    DeviceGuard guard(h->device);
    if (guard.ok) {
      if (h->work.wait() != cudaSuccess) rc = GBMUF_ERR_CUDA;
      h->work.release();
      cudaFree(h->d_status);
      cudaFree(h->table);
      for (void* t : h->earlier) cudaFree(t);
    } else {
      rc = GBMUF_ERR_CUDA;
    }
  }
  delete h;
  return rc;
}

}  // extern "C"
