// A product whose operands lie ready as bf16 parts, for the other translation units.
#ifndef GBMUF_CSRC_READY_PRODUCT_H
#define GBMUF_CSRC_READY_PRODUCT_H

#include <stdint.h>

#include "gbmuf.h"

// out[rows][cols] = sum over `terms` of a(term, col) b(row, term).  a is [terms][cols]; b is [terms][rows]
// (weight_grad) or [rows][terms].  Operands: [outer][inner] with row stride ld, 16-byte aligned, ld a
// multiple of 8; fp32 ones as three bf16 parts, outer * ld elements apart.
//   weight_grad: out is of out_dtype; accumulate != 0 adds to what it holds.
//   else: + residual.  Either out alone, of dtype; or, for dtype bf16 and out_dtype fp32, residual and out
//   in fp32 and `rounded` in bf16, each of which may be NULL (residual may be out).
struct gbmuf_ready_product {
  bool weight_grad;
  int32_t dtype, out_dtype, accumulate;
  const void *a, *b;
  int64_t a_outer, a_inner, a_ld, b_outer, b_inner, b_ld;
  int64_t rows, cols, terms;
  const void* residual;
  void *out, *rounded;
  int64_t ld_residual, ld_out, ld_rounded;
};
struct gbmuf_ops;
__attribute__((visibility("hidden"))) gbmuf_status gbmuf_run_ready_product(const gbmuf_ops* ops, const gbmuf_ready_product& r,
                                                                           void* stream);

#endif  // GBMUF_CSRC_READY_PRODUCT_H
