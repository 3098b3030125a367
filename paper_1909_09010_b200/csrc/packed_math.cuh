// Two fp32 operations per instruction, single instructions of the special-function unit, and what the
// local-step kernels add to primitives.cuh.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_PACKED_MATH_CUH
#define GBMUF_CSRC_PACKED_MATH_CUH

namespace {

struct Two { unsigned long long u; };
__device__ __forceinline__ Two two(float x, float y) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void apart(Two t, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(t.u)); }
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
  return r;
}
__device__ __forceinline__ Two operator-(Two a, Two b) { return fma_two(b, two(-1.0f, -1.0f), a); }

__device__ __forceinline__ float exp2_unit(float y) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float rcp_unit(float y) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
// Minimum and maximum that give NaN for NaN.
__device__ __forceinline__ float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float min_nan(float x, float y) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}

// A bulk copy that says whether its source will be fetched again soon: the L2 cache then keeps it
// rather than what only passes through (cross-entropy of 2,048 x 267,735 bf16: 464 -> 422 us).
__device__ __forceinline__ void bulk_load_hint(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, bool again) {
  uint64_t keep, pass;
  asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep));
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pass));
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar), "l"(again ? keep : pass)
      : "memory");
}

// mbar_wait_bounded with the first try in line.
__device__ __noinline__ bool wait_slowly(uint32_t bar, uint32_t parity, int32_t* status) {
  return mbar_wait_bounded(bar, parity, status);
}
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, int32_t* status) {
  return mbar_try_wait(bar, parity) || wait_slowly(bar, parity, status);
}

}  // namespace

#endif  // GBMUF_CSRC_PACKED_MATH_CUH
