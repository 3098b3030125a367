// libgbmuf: the softmax layer with its cross-entropy and all gradients, in pieces of the vocabulary, without
// the logits in memory.  The interface is in include/gbmuf.h; this file holds the host side and the C ABI,
// the kernels are those of linear_tc.cuh with the epilogues of linear_loss.cuh.

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
#include "linear_pack.cuh"
#include "softmax_math.cuh"
#include "linear_loss.cuh"
#include "linear_tc.cuh"
#include "linear_rows.cuh"
#include "linear_tc_host.h"

namespace {

typedef gbmuf_linear_cross_entropy_args Args;

// The gradient of a piece's logits is written once and read twice, by the two products.  Smaller pieces would stay
// in the L2 cache, but every piece costs three launches and their last waves (2,048 x 1,024 x 100,000: pieces of 9,472
// words 1,543 us, 18,944 1,494, 56,832 1,533; 1,024 x 512 x 267,735: 9,472 1,454, 28,416 1,286, 56,832 1,254).
constexpr long long kPieceBytes = 128ll << 20;
constexpr long long kPieceLeast = 2048;           // words: fewer leave the products too short

gbmuf_status check(const gbmuf_ops* ops, const Args* a) {
  if (!ops || !a) return invalid("ops and args must not be NULL");
  if (a->rows < 0 || a->n_in < 0 || a->vocab < 0) return invalid("rows, n_in and vocab must not be negative");
  if (a->rows > kMostDim || a->n_in > kMostDim || a->vocab > kMostDim)
    return refuse(GBMUF_ERR_UNSUPPORTED, "rows, n_in and vocab must be at most 2^31 - 2^16");
  if (a->rows > 0 && a->vocab == 0) return invalid("vocab must not be 0");
  if (!is_dtype(a->dtype) || !is_dtype(a->grad_dtype)) return invalid("dtype and grad_dtype must be GBMUF_F32 or GBMUF_BF16");
  if (!(a->scale == a->scale)) return invalid("scale must not be NaN");
  if (a->piece < 0) return invalid("piece must not be negative");
  CHECK_MATRIX("x", a->x, a->rows, a->n_in, a->ld_x, a->dtype, false);
  CHECK_MATRIX("w", a->w, a->vocab, a->n_in, a->ld_w, a->dtype, false);
  CHECK_MATRIX("bias", a->bias, 1, a->vocab, a->vocab, a->dtype, true);
  CHECK_MATRIX("dx", a->dx, a->rows, a->n_in, a->ld_dx, a->dtype, true);
  CHECK_MATRIX("dw", a->dw, a->vocab, a->n_in, a->ld_dw, a->grad_dtype, true);
  CHECK_MATRIX("dbias", a->dbias, 1, a->vocab, a->vocab, a->grad_dtype, true);
  if (a->rows > 0 && !a->targets) return invalid("targets is NULL");
  if ((uintptr_t)a->targets % 8 != 0) return invalid("targets is not aligned to its element type");
  if (((uintptr_t)a->row_weight | (uintptr_t)a->loss | (uintptr_t)a->lse) % 4 != 0)
    return invalid("row_weight, loss or lse is not aligned to its element type");
  return GBMUF_OK;
}

// Row tiles whose CTAs fill at least nine tenths of the GPU when each keeps to one row tile.
int rows_at_once(int tiles, int fit) {
  int t = std::min(tiles, fit);
  while (fit / t * t * 10 < fit * 9) --t;
  return t;
}
// ---- launch shapes.  Time of 64 terms of a tile of 128 pair x bn.  bf16: what its operands take to arrive (98 bytes a
// nanosecond and CTA of a pair, 110 of a single one) or its products to be formed (386 ns for 256 columns at the
// rate of a library product), whichever is longer; measured at 2,048 x 1,024 x 14,336: pairs of 256 400 ns, of 128
// 250, single CTAs of 256 460, of 128 290.  fp32, six products: as measured at 2,048 x 512 x 20,000, bound by the
// products for pairs of 256, by the shared memory that feeds them for the others.
double step_time(int parts, int bn, int pair) {
  if (parts == 3) return bn >= 256 ? 1800.0 : bn == 128 ? (pair == 2 ? 1100.0 : 1200.0) : bn == 64 ? 820.0 : 700.0;
  return std::max((double)tc_stage_bytes(bn, pair) / (pair == 2 ? 98.0 : 110.0), 386.0 * bn / 256.0);
}
struct Shape { int bn, pair, slices; double ns; };
enum Purpose { kStatistics, kGradient, kWeight, kTerm };
// The shape with the least time: rows R and columns C of the result, K terms.  fp32 sums leave the accumulator as they
// go, so there the epilogue (15 ns a column; 45 of the gradient, with its three parts) does not overlap the next tile's
// sums where there are two accumulators.  kStatistics: whole rounds of the column tiles only.  kTerm: the terms are cut
// into slices where tiles are few, as many as fill one to three waves.
Shape choose(const gbmuf_ops* ops, Purpose why, long long R, long long C, long long K, int parts) {
  Shape best{64, 1, 1, 1e300};
  const long long steps = (K + 63) / 64;
  for (int pair = 1; pair <= 2; ++pair)
    for (int bn = pair == 2 ? 128 : why == kTerm ? 64 : 32; bn <= (parts == 3 && (pair == 1 || why == kGradient) ? 128 : 256); bn *= 2) {
      const long long across = (C + 128 * pair - 1) / (128 * pair), tiles = std::max<long long>(1, across * ((R + bn - 1) / bn));
      long long fit = ops->num_sms / pair;
      if (why == kStatistics) { const long long t = rows_at_once((int)std::min<long long>(std::max<long long>(across, 1), 1 << 20), (int)fit); fit = fit / t * t; }
      const double step = step_time(parts, bn, pair), epilogue = (parts == 3 && why == kGradient ? 45.0 : 15.0) * bn;
      for (int w = 1; w <= (why == kTerm ? 3 : 1); ++w) {
        const long long n = why == kTerm ? std::max<long long>(1, std::min(steps / 4, w * fit / tiles)) : 1;
        const double sums = (double)((steps + n - 1) / n) * step;
        const bool hidden = parts == 1 || bn <= 128;
        const double tile = 1000.0 + (hidden ? std::max(sums, epilogue) : sums + epilogue);
        double t = ((tiles * n + fit - 1) / fit) * tile + (hidden ? epilogue : 0.0) + 0.001 * (n - 1) * R * C;
        if (pair == 2) t = (parts == 1 ? 0.95 : 1.0) * t + 2000.0;           // a third less through L2: power for the products
        if (t < best.ns) best = {bn, pair, (int)n, t};
      }
    }
  return best;
}
TcShape tc_shape(const Shape& s) { return {s.bn, 1, s.pair}; }

struct Plan {
  int parts;                                      // bf16 parts of an operand
  bool grad, x_ready, w_ready;                    // ready: read in place
  bool bias_once, few, twice, relative;           // few: the statistics of a few rows, on the fp32 units; relative: weights over the largest one
  int few_blocks;
  long long rows;                                 // of the gradients' products
  long long piece, pieces, ld_x, ld_w, ld_d, ld_acc, ld_partial, rows_padded, strips;
  TcShape stats, tc;                              // of the two products that form the logits
  Shape term;
  long long x_off, w_off, target_off, slot_off, max_off, pair_off, word_off, weight_off, d_off, partial_off, acc_off, bytes;
};

Operand operand_x(const Args* a) { return {a->x, a->rows, a->n_in, a->ld_x, true, false, 0}; }
Operand operand_w(const Args* a, long long v0, long long words) {
  return {static_cast<const char*>(a->w) + v0 * a->ld_w * (long long)size_of(a->dtype), words, a->n_in, a->ld_w, true, false, 0};
}
int row_tiles(const TcShape& s, long long rows) { return (int)((rows + 128 * s.pair - 1) / (128 * s.pair)); }
// Row tiles of the next launch of the statistics, with `left` rows to do.
int stats_rows(const gbmuf_ops* ops, const TcShape& s, long long left) { return rows_at_once(row_tiles(s, left), ops->num_sms / s.pair); }
int stats_slots(const gbmuf_ops* ops, const TcShape& s, int tiles_c, long long words) {
  return (int)std::min<long long>(ops->num_sms / s.pair / tiles_c, (words + s.bn - 1) / s.bn) * (kTcFinishers / 4);
}

// The time of a piece by that model, and a little for its launches.
double piece_time(const gbmuf_ops* ops, const Plan& p, const Args* a, long long words) {
  double ns = choose(ops, kGradient, p.rows, words, a->n_in, p.parts).ns + 5000.0;
  if (a->dw) ns += choose(ops, kWeight, words, a->n_in, p.rows, p.parts).ns;
  if (a->dx) ns += choose(ops, kTerm, p.rows, a->n_in, words, p.parts).ns;
  return ns;
}
// Words of a piece: what fits kPieceBytes (gradient and packed weights each), or a little less where that leaves fewer
// CTAs without a tile.
long long choose_piece(const gbmuf_ops* ops, const Plan& p, const Args* a) {
  long long wide = p.grad ? p.rows : 1;           // of what is in memory of a word: its gradient, its weights packed
  if (!p.w_ready) wide = std::max(wide, round_up(a->n_in, 8));
  const long long most = std::max(kPieceLeast, kPieceBytes / (2 * p.parts * wide) / 256 * 256);
  if (a->vocab <= most) return a->vocab;
  const long long least = (a->vocab + most - 1) / most;
  long long best = most;
  double best_t = 1e300;
  for (long long n = least; n <= least + std::min<long long>(least / 2 + 2, 16); ++n) {
    const long long piece = round_up((a->vocab + n - 1) / n, 256);
    if (piece < kPieceLeast && n > least) break;
    const long long whole = a->vocab / piece, rest = a->vocab % piece;
    const double t = whole * piece_time(ops, p, a, piece) + (rest ? piece_time(ops, p, a, rest) : 0.0);
    if (t < best_t) { best_t = t; best = piece; }
  }
  return best;
}

Plan make_plan(const gbmuf_ops* ops, const Args* a) {
  Plan p{};
  p.parts = a->dtype == GBMUF_F32 ? 3 : 1;
  p.grad = a->dx || a->dw || a->dbias;
  // as the linear layer's rule for a few rows
  const int64_t most = a->dtype == GBMUF_F32 ? 16 : 8, rounded = a->rows <= 1 ? 1 : a->rows <= 2 ? 2 : a->rows <= 4 ? 4 : a->rows <= 8 ? 8 : 16;
  p.few = a->rows <= most && rounded * ((a->n_in + 7) / 8 * 8) * (int64_t)size_of(a->dtype) <= kRowsMostBytes;
  p.twice = p.grad && p.parts == 1 && a->row_weight && a->rows <= kLossTwice;
  p.rows = p.twice ? 2 * a->rows : a->rows;
  p.relative = p.grad && p.parts == 1 && a->row_weight && !p.twice;      // more rows than `few` has
  p.x_ready = !p.twice && in_place(operand_x(a), a->dtype);
  p.w_ready = in_place(operand_w(a, 0, a->vocab), a->dtype);
  const bool products = p.grad || !p.few;         // operands of the tensor cores are needed
  p.piece = a->piece ? std::min<long long>(a->piece, a->vocab) : p.grad || (!p.w_ready && products) ? choose_piece(ops, p, a) : a->vocab;
  p.pieces = (a->vocab + p.piece - 1) / p.piece;
  p.ld_x = p.x_ready && a->rows > 1 ? a->ld_x : round_up(a->n_in, 8);      // the stride of a single row says nothing
  p.ld_w = p.w_ready && a->vocab > 1 ? a->ld_w : round_up(a->n_in, 8);
  p.ld_d = round_up(p.rows, 64);                 // whole strips of rows are stored
  p.ld_acc = round_up(a->n_in, 4);
  p.rows_padded = round_up(p.rows, kLossRowPad);
  const long long together = p.w_ready ? a->vocab : p.piece;
  p.stats = tc_shape(choose(ops, kStatistics, together, a->rows, a->n_in, p.parts));
  p.tc = tc_shape(choose(ops, kGradient, p.rows, p.piece, a->n_in, p.parts));
  long long at = 0;
  auto take = [&](long long bytes) { const long long here = at; at += round_up(bytes, 256); return here; };
  p.x_off = take(p.x_ready || !products ? 0 : packed_bytes(operand_x(a), a->dtype, true) * (p.twice ? 2 : 1));
  p.w_off = take(p.w_ready || !products ? 0 : packed_bytes(operand_w(a, 0, p.piece), a->dtype, true));
  p.target_off = take(a->rows * 4);
  const int per_block = (rounded >= 16 ? 2 : 4) * kRowsThreads / 32;
  p.few_blocks = (int)std::min<long long>((a->vocab + per_block - 1) / per_block, ops->num_sms * 2);
  long long slots = p.few ? p.few_blocks * a->rows : 0;
  for (long long r = 0; r < a->rows && !p.few;) {
    const int t = stats_rows(ops, p.stats, a->rows - r);
    const long long n = std::min<long long>(a->rows - r, 128ll * p.stats.pair * t);
    slots += n * stats_slots(ops, p.stats, t, together) * (p.w_ready ? 1 : p.pieces);
    r += n;
  }
  p.slot_off = take(slots * 8);
  if (p.relative) p.max_off = take(((a->rows + 31) / 32 + 1) * 4);      // the factor comes first
  if (p.grad) {
    p.pair_off = take(p.rows_padded / 2 * (long long)sizeof(RowPair));
    p.word_off = take(p.rows_padded * 4);
    p.weight_off = take(p.rows_padded * 4);
    p.d_off = take(p.piece * p.ld_d * 2 * p.parts);
    if (a->dbias) {
      // the strips' sums of all words, added up once at the end, unless that takes too much room
      p.strips = (p.rows + p.tc.bn - 1) / p.tc.bn * (kTcFinishers / 4);
      p.bias_once = p.strips * a->vocab * 4 <= kPieceBytes;
      p.ld_partial = p.bias_once ? a->vocab : p.piece;
      p.partial_off = take(p.strips * p.ld_partial * 4);
    }
    if (a->dx) {
      p.term = choose(ops, kTerm, p.rows, a->n_in, p.piece, p.parts);
      p.acc_off = take(p.term.slices * p.rows * p.ld_acc * 4);
    }
  }
  p.bytes = at;
  return p;
}

// Tensor map of a piece's gradient [parts][words][rows], for stores of 32 rows by 32 words.
gbmuf_status gradient_map(const TcParams& P, int parts, CUtensorMap* map) {
  const EncodeTiledFn encode = encode_tiled_fn();
  if (!encode) return refuse(GBMUF_ERR_CUDA, "the driver does not provide cuTensorMapEncodeTiled");
  const cuuint64_t dim[3] = {(cuuint64_t)P.R, (cuuint64_t)P.E.words, (cuuint64_t)parts};
  const cuuint64_t stride[2] = {(cuuint64_t)P.E.ld_out0 * 2, (cuuint64_t)P.E.part * 2};
  const cuuint32_t box[3] = {32, 32, 1}, one[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, P.E.out0, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return refuse(GBMUF_ERR_CUDA, "cuTensorMapEncodeTiled failed with code " + std::to_string((int)r));
  return GBMUF_OK;
}
template <int KIND, typename T, int PARTS>
gbmuf_status launch_logits(const gbmuf_ops* ops, const TcShape& s, TcParams& P, int at_once, const Operand& a, const Operand& b,
                           int32_t dtype, cudaStream_t st) {
  CUtensorMap ma{}, mb{}, out{};
  if (KIND == kLossGrad)
    if (gbmuf_status rc = gradient_map(P, PARTS, &out)) return rc;
  if (P.ksteps > 0) {
    if (gbmuf_status rc = operand_map(a, dtype, nullptr, 128, &ma)) return rc;
    if (gbmuf_status rc = operand_map(b, dtype, nullptr, s.bn / s.pair, &mb)) return rc;
  }
  if (s.pair == 2) {
    if constexpr (KIND != kLossGrad || PARTS == 1)
      if (s.bn == 256) return launch_tc_at<KIND, T, T, PARTS, 256, 2>(ops, P, at_once, ma, mb, st, out);
    return launch_tc_at<KIND, T, T, PARTS, 128, 2>(ops, P, at_once, ma, mb, st, out);
  }
  if (s.bn == 32) return launch_tc_at<KIND, T, T, PARTS, 32, 1>(ops, P, at_once, ma, mb, st, out);
  if constexpr (PARTS == 1)
    if (s.bn == 256) return launch_tc_at<KIND, T, T, PARTS, 256, 1>(ops, P, at_once, ma, mb, st, out);
  return s.bn == 64 ? launch_tc_at<KIND, T, T, PARTS, 64, 1>(ops, P, at_once, ma, mb, st, out)
                    : launch_tc_at<KIND, T, T, PARTS, 128, 1>(ops, P, at_once, ma, mb, st, out);
}

// The two products with the gradient of a piece's logits.
template <int KIND, typename T, typename TO, int PARTS>
gbmuf_status launch_loss_product(const gbmuf_ops* ops, int bn, int pair, TcParams& P, int at_once, const Operand& a, const Operand& b,
                                 int32_t dtype, cudaStream_t st) {
  CUtensorMap ma{}, mb{};
  if (gbmuf_status rc = operand_map(a, dtype, nullptr, 64, &ma)) return rc;
  if (gbmuf_status rc = operand_map(b, dtype, nullptr, b.k_inner ? bn / pair : 64, &mb)) return rc;
  if (pair == 2)
    return bn == 128 ? launch_tc_at<KIND, T, TO, PARTS, 128, 2>(ops, P, at_once, ma, mb, st)
                     : launch_tc_at<KIND, T, TO, PARTS, 256, 2>(ops, P, at_once, ma, mb, st);
  if constexpr (KIND == kLossWeight)
    if (bn == 32) return launch_tc_at<KIND, T, TO, PARTS, 32, 1>(ops, P, at_once, ma, mb, st);
  if constexpr (PARTS == 1)
    if (bn == 256) return launch_tc_at<KIND, T, TO, PARTS, 256, 1>(ops, P, at_once, ma, mb, st);
  return bn == 64 ? launch_tc_at<KIND, T, TO, PARTS, 64, 1>(ops, P, at_once, ma, mb, st)
                  : launch_tc_at<KIND, T, TO, PARTS, 128, 1>(ops, P, at_once, ma, mb, st);
}

// twice: and once more behind it
gbmuf_status pack(const gbmuf_ops* ops, const Operand& o, int32_t dtype, void* dst, bool twice, cudaStream_t st) {
  const PackJob j = pack_job(ops, o, dtype, dst, true);       // a piece of a single word might do in place, its matrix does not
  if (j.blocks == 0) return GBMUF_OK;
  PackJob again{};
  if (twice) {
    again = j;
    again.dst = j.dst + j.outer * j.ld_dst;
  }
  return launched("launch of the operand-packing kernel",
                  launch(dtype == GBMUF_F32 ? pack_kernel<float> : pack_kernel<__nv_bfloat16>, (unsigned)(j.blocks + again.blocks), 1, 256, 0, st, j, again));
}

// A few rows: one read of the weights on the fp32 units, as in the linear layer.
template <typename T, int ROWS> cudaError_t launch_rows_loss(const RowsParams& P, bool vec, unsigned grid, cudaStream_t st) {
  const uint32_t smem = (uint32_t)(ROWS * ((P.K + 7) / 8 * 8) * (int)sizeof(T));
  const auto kernel = vec ? linear_rows_kernel<T, ROWS, true, true> : linear_rows_kernel<T, ROWS, false, true>;
  if (smem > 48 * 1024 - 4096) {                  // 4 KB: what it has besides
    const cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsMostBytes);
    if (e != cudaSuccess) return e;
  }
  return launch(kernel, grid, 1, kRowsThreads, smem, st, P);
}
template <typename T> cudaError_t rows_loss(const Args* a, RowsParams& P, unsigned grid, cudaStream_t st) {
  P.x = a->x; P.w = a->w; P.ld_x = a->ld_x; P.ld_w = a->ld_w;
  P.R = (int)a->rows; P.C = (int)a->vocab; P.K = (int)a->n_in;
  const bool vec = (uintptr_t)a->w % 16 == 0 && (a->vocab == 1 || a->ld_w * (int64_t)sizeof(T) % 16 == 0);
  if (a->rows <= 1) return launch_rows_loss<T, 1>(P, vec, grid, st);
  if (a->rows <= 2) return launch_rows_loss<T, 2>(P, vec, grid, st);
  if (a->rows <= 4) return launch_rows_loss<T, 4>(P, vec, grid, st);
  if (a->rows <= 8 || sizeof(T) == 2) return launch_rows_loss<T, 8>(P, vec, grid, st);
  if constexpr (sizeof(T) == 4) return launch_rows_loss<T, 16>(P, vec, grid, st);
  return cudaErrorInvalidValue;
}

template <typename T> gbmuf_status run(const gbmuf_ops* ops, const Args* a, cudaStream_t st) {
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
  const Plan p = make_plan(ops, a);
  if (p.bytes > a->workspace_bytes || !a->workspace || (uintptr_t)a->workspace % 256 != 0)
    return invalid("workspace must be 256-byte aligned device memory of at least " + std::to_string(p.bytes) + " bytes");
  char* const ws = static_cast<char*>(a->workspace);
  const long long N = a->rows, G = p.rows, V = a->vocab, H = a->n_in, size = (long long)sizeof(T);
  Operand x = operand_x(a);
  if (!p.x_ready && (p.grad || !p.few)) {
    if (gbmuf_status rc = pack(ops, x, a->dtype, ws + p.x_off, p.twice, st)) return rc;
    x.p = ws + p.x_off;
  }
  x.ld = p.ld_x;
  x.ready = true;
  x.part = N * x.ld;
  long long packed = -1;                          // the piece that lies packed
  auto weights = [&](long long v0, long long words, Operand& w) -> gbmuf_status {
    w = operand_w(a, v0, words);
    if (!p.w_ready) {
      if (packed != v0)
        if (gbmuf_status rc = pack(ops, w, a->dtype, ws + p.w_off, false, st)) return rc;
      packed = v0;
      w.p = ws + p.w_off;
    }
    w.ld = p.ld_w;
    w.ready = true;
    return GBMUF_OK;
  };
  auto tc_params = [&](const TcShape& s, long long R, long long C, bool stats) {
    TcParams P{};
    P.status = ops->d_status; P.R = (int)R; P.C = (int)C; P.split = 1;
    P.ksteps = (int)((H + kTcK - 1) / kTcK);
    const int tiles_r = (int)((R + s.bn - 1) / s.bn), tiles_c = (int)((C + 128 * s.pair - 1) / (128 * s.pair));
    P.tiles_fast = stats ? tiles_c : tiles_r;
    P.tiles = tiles_r * tiles_c;
    return P;
  };
  const TcShape& s = p.stats;
  const long long most_tiles = std::max((V / s.bn + 1) * (N / 128 + 1), (V / 128 + 1) * (G / p.tc.bn + 1));
  if (most_tiles > 0x3fffffff) return refuse(GBMUF_ERR_UNSUPPORTED, "more than 2^30 tiles of logits");
  float* const factor = p.relative ? reinterpret_cast<float*>(ws + p.max_off) : nullptr;
  // ---- statistics: every CTA keeps to one row tile, so its threads keep a row's running maximum and sum.  Rows in ranges
  // that fill the GPU; do_ranges(f): f(first row, rows, row tiles, the range's slots)
  const long long step = p.w_ready ? V : p.piece, steps = (V + step - 1) / step;
  auto do_ranges = [&](auto f) -> gbmuf_status {
    float2* slots = reinterpret_cast<float2*>(ws + p.slot_off);
    for (long long r0 = 0; r0 < N;) {
      const int t = p.few ? 1 : stats_rows(ops, s, N - r0);
      const long long n = p.few ? N : std::min<long long>(N - r0, 128ll * s.pair * t);
      if (gbmuf_status rc = f(r0, n, t, slots)) return rc;
      if (!p.few) slots += n * stats_slots(ops, s, t, step) * steps;
      r0 += n;
    }
    return GBMUF_OK;
  };
  if (p.few) {
    RowsParams P{};
    P.E.bias = a->bias; P.E.loss_rows = a->targets;
    P.E.target_logit = reinterpret_cast<float*>(ws + p.target_off);
    P.E.partial = ws + p.slot_off; P.E.ld_partial = N;
    const cudaError_t e = rows_loss<T>(a, P, (unsigned)p.few_blocks, st);
    if (e != cudaSuccess) return cuda_refuse("launch of the few-rows loss kernel", e);
  }
  for (long long v0 = 0; v0 < V && !p.few; v0 += step) {      // weights that have to be packed are packed once for all rows
    const long long words = std::min(step, V - v0);
    Operand w;
    if (gbmuf_status rc = weights(v0, words, w)) return rc;
    if (gbmuf_status rc = do_ranges([&](long long r0, long long n, int t, float2* slots) -> gbmuf_status {
      Operand xr = x;
      xr.p = static_cast<const char*>(x.p) + r0 * x.ld * 2;
      xr.outer = n;
      TcParams P = tc_params(s, words, n, true);
      P.E.bias = a->bias ? static_cast<const char*>(a->bias) + v0 * size : nullptr;
      P.E.loss_rows = a->targets + r0;
      P.E.target_logit = reinterpret_cast<float*>(ws + p.target_off) + r0;
      P.E.partial = slots + v0 / step * stats_slots(ops, s, t, step) * n;
      P.E.ld_partial = n;
      P.E.first_word = (int)v0;
      if (factor) {                              // r0 is a multiple of 128
        P.E.weight_max = factor + 1 + r0 / 32;
        P.E.loss_weights = a->row_weight + r0; P.E.scale = a->scale; P.E.vocab = V; P.E.ignore_index = a->ignore_index;
      }
      const int here = stats_slots(ops, s, t, words);
      return launch_logits<kLossStats, T, PARTS>(ops, s, P, here / (kTcFinishers / 4) * t, xr, w, a->dtype, st);
    })) {
      return rc;
    }
  }
  long long groups = (N + 31) / 32;
  if (factor && groups > kLossMostGroups) {        // 2,000,000 x 16, 300 words: read by every join block 1,160 us, this 60
    const cudaError_t e = launch(loss_max_kernel, 1, 1, 1024, 0, st, factor + 1, groups);
    if (e != cudaSuccess) return cuda_refuse("launch of the loss's weight kernel", e);
    groups = 1;
  }
  if (gbmuf_status rc = do_ranges([&](long long r0, long long n, int t, float2* slots) -> gbmuf_status {
    JoinParams J{};
    J.L.targets = a->targets + r0; J.L.row_weight = a->row_weight ? a->row_weight + r0 : nullptr;
    J.L.loss = a->loss ? a->loss + r0 : nullptr; J.L.lse = a->lse ? a->lse + r0 : nullptr;
    J.L.rows = n; J.L.vocab = V; J.L.ignore_index = a->ignore_index; J.L.scale = a->scale; J.L.status = ops->d_status;
    J.slots = slots;
    J.target_logit = reinterpret_cast<const float*>(ws + p.target_off) + r0;
    if (p.grad) {
      J.pairs = reinterpret_cast<RowPair*>(ws + p.pair_off) + r0 / 2;
      J.targets = reinterpret_cast<int*>(ws + p.word_off) + r0;
      J.weights = reinterpret_cast<float*>(ws + p.weight_off) + r0;
    }
    if (factor) { J.weight_max = factor + 1; J.factor = factor; J.groups = groups; }
    J.ld = n; J.twice = p.twice;
    J.count = p.few ? p.few_blocks : (int)((steps - 1) * stats_slots(ops, s, t, step)) + stats_slots(ops, s, t, V - (steps - 1) * step);
    J.rows_padded = r0 + n == N ? p.rows_padded - r0 : n;
    const cudaError_t e = launch(loss_join_kernel, (unsigned)((J.rows_padded + 31) / 32), 1, 32 * kJoinShares, 0, st, J);
    return e == cudaSuccess ? GBMUF_OK : cuda_refuse("launch of the loss's join kernel", e);
  })) {
    return rc;
  }
  if (!p.grad) return GBMUF_OK;
  // ---- gradients, a piece of the vocabulary at a time
  x.outer = G;
  for (long long i = 0, v0 = 0; v0 < V; ++i, v0 += p.piece) {
    const long long words = std::min(p.piece, V - v0);
    const bool last = v0 + words == V;
    Operand w;
    if (gbmuf_status rc = weights(v0, words, w)) return rc;
    void* const d = ws + p.d_off;
    TcParams P = tc_params(p.tc, G, words, false);
    P.E.bias = a->bias ? static_cast<const char*>(a->bias) + v0 * size : nullptr;
    P.E.loss_rows = ws + p.pair_off;
    P.E.loss_targets = reinterpret_cast<const int*>(ws + p.word_off);
    P.E.loss_weights = reinterpret_cast<const float*>(ws + p.weight_off);
    P.E.partial = a->dbias ? reinterpret_cast<float*>(ws + p.partial_off) + (p.bias_once ? v0 : 0) : nullptr;
    P.E.ld_partial = p.ld_partial;
    P.E.first_word = (int)v0; P.E.words = (int)words;
    P.E.rest_from = p.twice ? (int)N : 0x7fffffff;
    P.E.out0 = d; P.E.ld_out0 = p.ld_d; P.E.part = words * p.ld_d;
    const int at_once = std::min(P.tiles, ops->num_sms / p.tc.pair);
    if (gbmuf_status rc = launch_logits<kLossGrad, T, PARTS>(ops, p.tc, P, at_once, w, x, a->dtype, st)) return rc;
    if (a->dbias && (!p.bias_once || last)) {
      const long long first = p.bias_once ? 0 : v0, n = v0 + words - first;
      cudaError_t e = cudaSuccess;
      DISPATCH_DTYPE(a->grad_dtype, TO, e = launch(loss_bias_kernel<TO>, (unsigned)((n + 255) / 256), 1, 256, 0, st,
                                                   reinterpret_cast<const float*>(ws + p.partial_off), p.ld_partial, (int)p.strips, n,
                                                   static_cast<TO*>(a->dbias) + first, (int)a->accumulate, a->scale, (const float*)factor));
      if (e != cudaSuccess) return cuda_refuse("launch of the loss's bias-gradient kernel", e);
    }
    if (H == 0) continue;
    // dw = d^T x: columns along the lanes, d's rows next to one another
    Operand xw = x, dw_b{d, words, G, p.ld_d, true, true, 0}, dx_b{d, words, G, p.ld_d, false, true, 0};
    xw.k_inner = false;
    if (a->dw) {
      const TcShape shape = tc_shape(choose(ops, kWeight, words, a->n_in, G, p.parts));
      TcParams W = tc_params(shape, words, H, false);
      W.ksteps = (int)((G + kTcK - 1) / kTcK);
      W.E.out0 = static_cast<char*>(a->dw) + v0 * a->ld_dw * (long long)size_of(a->grad_dtype); W.E.ld_out0 = a->ld_dw;
      W.E.accumulate = a->accumulate;
      W.E.scale = a->scale;
      W.E.factor = factor;
      W.E.pairs = a->grad_dtype == GBMUF_BF16 && (uintptr_t)W.E.out0 % 4 == 0 && H % 2 == 0 && (words == 1 || a->ld_dw % 2 == 0);
      gbmuf_status rc = GBMUF_OK;
      DISPATCH_DTYPE(a->grad_dtype, TO, (rc = launch_loss_product<kLossWeight, TO, TO, PARTS>(
          ops, shape.bn, shape.pair, W, std::min(W.tiles, ops->num_sms / shape.pair), xw, dw_b, a->dtype, st)));
      if (rc != GBMUF_OK) return rc;
    }
    if (a->dx) {
      // dx += d w, in fp32
      Operand wk = w;
      wk.k_inner = false;
      TcShape shape{p.term.bn, 1, p.term.pair};
      TcParams D = tc_params(shape, G, H, false);
      D.ksteps = (int)((words + kTcK - 1) / kTcK);
      D.slices = p.term.slices;
      D.tiles_c = D.tiles / D.tiles_fast;
      D.tiles *= D.slices;
      D.E.out0 = ws + p.acc_off; D.E.ld_out0 = p.ld_acc; D.E.part = G * p.ld_acc; D.E.accumulate = i > 0;
      if (gbmuf_status rc = launch_loss_product<kLossTerm, T, float, PARTS>(ops, shape.bn, shape.pair, D, std::min(D.tiles, ops->num_sms / shape.pair),
                                                                            wk, dx_b, a->dtype, st))
        return rc;
      if (last) {
        const cudaError_t e = launch(loss_dx_kernel<T>, (unsigned)std::min<long long>(N, ops->num_sms * 8), 1, 256, 0, st,
                                     reinterpret_cast<const float*>(ws + p.acc_off), p.ld_acc, G * p.ld_acc, p.term.slices,
                                     static_cast<T*>(a->dx), (long long)a->ld_dx, N, (int)H, a->scale, (const float*)factor, p.twice);
        if (e != cudaSuccess) return cuda_refuse("launch of the loss's input-gradient kernel", e);
      }
    }
  }
  return GBMUF_OK;
}

}  // namespace

extern "C" {

gbmuf_status gbmuf_linear_cross_entropy_workspace(gbmuf_ops* ops, const gbmuf_linear_cross_entropy_args* a, int64_t* bytes) {
  return guarded([&]() -> gbmuf_status {
    if (!bytes) return invalid("bytes is NULL");
    if (gbmuf_status st = check(ops, a)) return st;
    *bytes = a->rows == 0 ? 0 : make_plan(ops, a).bytes;
    return GBMUF_OK;
  });
}

gbmuf_status gbmuf_linear_cross_entropy(gbmuf_ops* ops, const gbmuf_linear_cross_entropy_args* a, void* stream) {
  return guarded([&]() -> gbmuf_status {
    if (gbmuf_status st = check(ops, a)) return st;
    if (a->rows == 0) {                            // empty sums
      if (a->accumulate || a->vocab == 0 || (!a->dw && !a->dbias)) return GBMUF_OK;
      gbmuf_linear_backward_weight_args z{};
      z.n_in = a->n_in; z.n_out = a->vocab; z.dw = a->dw; z.dbias = a->dbias; z.ld_dw = a->ld_dw;
      z.ld_dz = a->vocab; z.ld_x = a->n_in;
      z.dtype = a->dtype; z.grad_dtype = a->grad_dtype;
      return gbmuf_linear_backward_weight(ops, &z, stream);
    }
    DeviceGuard guard(ops->device);
    if (!guard.ok) return refuse(GBMUF_ERR_CUDA, "cudaSetDevice failed");
    DISPATCH_DTYPE(a->dtype, T, return run<T>(ops, a, (cudaStream_t)stream));
  });
}

}  // extern "C"
