// Element types, activations and the epilogue of the linear-layer kernels.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_LINEAR_EPILOGUE_CUH
#define GBMUF_CSRC_LINEAR_EPILOGUE_CUH

namespace {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Values beyond +-100 count as +-100 where an activation is flat there in fp32 (its exponentials
// are 0 or its limit is reached), so that infinities give the limits and not inf * 0; NaN stays.
__device__ __forceinline__ float clamp100(float z) { return z > 100.0f ? 100.0f : (z < -100.0f ? -100.0f : z); }

__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case GBMUF_ACT_RELU: return z < 0.0f ? 0.0f : z;
    // z Phi(z) with Phi(z) = erfc(-z / sqrt 2) / 2, which keeps its relative accuracy for z << 0
    case GBMUF_ACT_GELU: return (z < -100.0f ? -100.0f : z) * (0.5f * erfcf(-0.70710678118654752f * z));
    case GBMUF_ACT_SILU: return (z < -100.0f ? -100.0f : z) / (1.0f + expf(-z));
    case GBMUF_ACT_TANH: return tanhf(z);
    case GBMUF_ACT_SIGMOID: return 1.0f / (1.0f + expf(-z));
    default: return z;
  }
}

__device__ __forceinline__ float activate_slope(float z, int act) {
  switch (act) {
    case GBMUF_ACT_RELU: return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    case GBMUF_ACT_GELU: {
      const float c = clamp100(z);
      return 0.5f * erfcf(-0.70710678118654752f * c) + c * (0.39894228040143268f * expf(-0.5f * c * c));
    }
    case GBMUF_ACT_SILU: {
      const float c = clamp100(z), s = 1.0f / (1.0f + expf(-c));
      return s * (1.0f + c * (1.0f - s));
    }
    case GBMUF_ACT_TANH: { const float t = tanhf(z); return 1.0f - t * t; }
    case GBMUF_ACT_SIGMOID: { const float s = 1.0f / (1.0f + expf(-z)); return s * (1.0f - s); }
    default: return 1.0f;
  }
}

enum LinearKind { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

// What happens to a finished sum `acc` of row r, column c of the result.  T: the type of all
// operands but the weight gradient, which is TO.
//   forward      z = acc + bias[c]; out1 <- z; out0 <- act(z) + residual
//   input grad   d = acc + residual; out0 <- d; out1 <- d * act'(z_in)
//   weight grad  out0 <- acc (+ out0)
struct Epilogue {
  const void* bias;
  const void* residual;
  const void* z_in;
  void* out0;
  void* out1;
  long long ld_residual, ld_z_in, ld_out0, ld_out1;
  int act, accumulate;
};

template <int KIND, typename T, typename TO>
__device__ __forceinline__ void finish_element(const Epilogue& E, long long r, long long c, float acc) {
  if (KIND == kForward) {
    const float z = E.bias ? acc + to_f32(static_cast<const T*>(E.bias)[c]) : acc;
    if (E.out1) static_cast<T*>(E.out1)[r * E.ld_out1 + c] = from_f32<T>(z);
    float y = activate(z, E.act);
    if (E.residual) y += to_f32(static_cast<const T*>(E.residual)[r * E.ld_residual + c]);
    static_cast<T*>(E.out0)[r * E.ld_out0 + c] = from_f32<T>(y);
  } else if (KIND == kInputGrad) {
    float d = acc;
    if (E.residual) d += to_f32(static_cast<const T*>(E.residual)[r * E.ld_residual + c]);
    if (E.out0) static_cast<T*>(E.out0)[r * E.ld_out0 + c] = from_f32<T>(d);
    if (E.out1)
      static_cast<T*>(E.out1)[r * E.ld_out1 + c] =
          from_f32<T>(d * activate_slope(to_f32(static_cast<const T*>(E.z_in)[r * E.ld_z_in + c]), E.act));
  } else {
    TO* const p = static_cast<TO*>(E.out0) + r * E.ld_out0 + c;
    *p = from_f32<TO>(E.accumulate ? acc + to_f32(*p) : acc);
  }
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_EPILOGUE_CUH
