// Two fp32 operations per instruction, and single instructions of the special-function unit.
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

// mbar_wait_bounded with the first try in line.
__device__ __noinline__ bool wait_slowly(uint32_t bar, uint32_t parity, int32_t* status) {
  return mbar_wait_bounded(bar, parity, status);
}
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, int32_t* status) {
  return mbar_try_wait(bar, parity) || wait_slowly(bar, parity, status);
}

}  // namespace

#endif  // GBMUF_CSRC_PACKED_MATH_CUH
