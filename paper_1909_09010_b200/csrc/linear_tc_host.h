// Host side of the tensor-core products: operands, tensor maps, launch shapes.
// Included after linear_tc.cuh and linear_pack.cuh.
#ifndef GBMUF_CSRC_LINEAR_TC_HOST_H
#define GBMUF_CSRC_LINEAR_TC_HOST_H

#include "ops_host.h"

namespace {

// An operand as it lies in memory: [outer][inner] of the call's type, row stride ld; k_inner: the
// summed index is the inner one.  ready: it has been packed, as bf16 parts [1 or 3][outer][ld], `part`
// elements apart (0: outer * ld).
struct Operand {
  const void* p;
  long long outer, inner, ld;
  bool k_inner, ready;
  long long part;
};
// A product of two operands: result [R][C], K terms.
struct Product {
  Operand a, b;
  long long R, C, K;
  int32_t dtype;
  Epilogue E;
};

bool in_place(const Operand& o, int32_t dtype) {
  return o.ready || (dtype == GBMUF_BF16 && (uintptr_t)o.p % 16 == 0 && (o.outer <= 1 || (o.ld % 8 == 0 && o.ld < ((long long)1 << 38))));
}
long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }
long long packed_bytes(const Operand& o, int32_t dtype, bool always = false) {
  return !always && in_place(o, dtype) ? 0 : round_up((dtype == GBMUF_F32 ? 3 : 1) * o.outer * round_up(o.inner, 8) * 2, 256);
}
long long product_workspace(const Product& q) {
  return q.K == 0 || q.R == 0 || q.C == 0 ? 0 : packed_bytes(q.a, q.dtype) + packed_bytes(q.b, q.dtype);
}

// always: a part of a matrix that as a whole cannot be read in place.
PackJob pack_job(const gbmuf_ops* ops, const Operand& o, int32_t dtype, void* dst, bool always = false) {
  PackJob j{};
  if (!always && in_place(o, dtype)) return j;
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
  const long long ld = here && (o.outer > 1 || o.ready) ? o.ld : round_up(o.inner, 8);
  const cuuint64_t dim[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)(dtype == GBMUF_F32 ? 3 : 1)};
  const cuuint64_t stride[2] = {(cuuint64_t)ld * 2, dtype == GBMUF_F32 ? (cuuint64_t)(o.part ? o.part : o.outer * ld) * 2 : (cuuint64_t)ld * 2};
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

// at_once: tiles that are worked on side by side.
template <int KIND, typename T, typename TO, int PARTS, int BN, int PAIR>
gbmuf_status launch_tc_at(const gbmuf_ops* ops, TcParams& P, int at_once, const CUtensorMap& ma, const CUtensorMap& mb, cudaStream_t st,
                          const CUtensorMap& out = CUtensorMap{}) {
  const auto kernel = linear_tc_kernel<KIND, T, TO, PARTS, BN, PAIR>;
  constexpr uint32_t OUT = kTcOut<KIND, PARTS, BN>;
  P.stages = std::min<int>(kTcMaxStages, (ops->max_smem - 1024 - (int)(kTcHead + OUT)) / (int)tc_stage_bytes(BN, PAIR));
  const uint32_t smem = tc_smem_bytes(BN, PAIR, P.stages) + OUT;
  static std::atomic<uint64_t> ready{0};                  // devices on which the limit has been raised
  const uint64_t bit = 1ull << (ops->device & 63);
  if (!(ready.load() & bit)) {
    const cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ops->max_smem);
    if (e != cudaSuccess) return cuda_refuse("shared-memory limit of the linear-layer kernel", e);
    if (ops->device < 64) ready.fetch_or(bit);
  }
  P.tile_step = at_once; P.step_slow = at_once / P.tiles_fast; P.step_fast = at_once % P.tiles_fast;
  const unsigned grid = (unsigned)(at_once * PAIR * P.split);
  return launched("launch of the linear-layer kernel", launch(kernel, grid, (unsigned)(PAIR * P.split), kTcThreads, smem, st, ma, mb, out, P));
}
template <int KIND, typename T, typename TO, int PARTS, int BN, int PAIR>
gbmuf_status launch_tc(const gbmuf_ops* ops, TcParams& P, const CUtensorMap& ma, const CUtensorMap& mb, cudaStream_t st) {
  const int at_once = P.split > 1 ? P.tiles : std::min(P.tiles, ops->num_sms / PAIR);     // a split tile: one per cluster
  return launch_tc_at<KIND, T, TO, PARTS, BN, PAIR>(ops, P, at_once, ma, mb, st);
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_TC_HOST_H
