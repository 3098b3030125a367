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

// FAST (results that are rounded to bf16): exponentials and reciprocals from the special-function
// unit, a few units in 2^-22, where the accurate functions would make the epilogue the bound.
template <bool FAST> __device__ __forceinline__ float exp_of(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST> __device__ __forceinline__ float quotient(float x, float y) { return FAST ? __fdividef(x, y) : x / y; }
template <bool FAST> __device__ __forceinline__ float logistic(float z) {
  // __fdividef returns 0 for a divisor above 2^126: exp(100) is below
  return quotient<FAST>(1.0f, 1.0f + exp_of<FAST>(-(FAST ? clamp100(z) : z)));
}
// Phi(z) = erfc(-z / sqrt 2) / 2, and g = exp(-z^2 / 2).  FAST: Abramowitz and Stegun 7.1.26,
// erfc(x) = (a1 t + .. + a5 t^5) exp(-x^2), t = 1 / (1 + p x) for x >= 0, off by at most 1.5e-7.
template <bool FAST> __device__ __forceinline__ float normal_cdf(float z, float& g) {
  g = exp_of<FAST>(-0.5f * z * z);
  if (!FAST) return 0.5f * erfcf(-0.70710678118654752f * z);
  const float t = __fdividef(1.0f, fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.0f));
  float q = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  q = fmaf(t, q, 0.5f * 1.421413741f);
  q = fmaf(t, q, 0.5f * -0.284496736f);
  q = fmaf(t, q, 0.5f * 0.254829592f) * t * g;
  return z >= 0.0f ? 1.0f - q : q;
}
template <bool FAST> __device__ __forceinline__ float tanh_of(float z) {
  if (!FAST) return tanhf(z);
  const float s = z * z;                                   // below 0.15 the series: next term 17/315 z^7
  const float near = fmaf(z * s, fmaf(s, 2.0f / 15.0f, -1.0f / 3.0f), z);
  const float far = 1.0f - __fdividef(2.0f, 1.0f + __expf(2.0f * (z > 40.0f ? 40.0f : z)));
  return fabsf(z) < 0.15f ? near : far;
}

template <bool FAST> __device__ __forceinline__ float activate(float z, int act) {
  float g;
  switch (act) {
    case GBMUF_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case GBMUF_ACT_GELU: return (z < -100.0f ? -100.0f : z) * normal_cdf<FAST>(z > 100.0f ? 100.0f : z, g);
    case GBMUF_ACT_SILU: return (z < -100.0f ? -100.0f : z) * logistic<FAST>(z);
    case GBMUF_ACT_TANH: return tanh_of<FAST>(z);
    case GBMUF_ACT_SIGMOID: return logistic<FAST>(z);
    default: return z;
  }
}

template <bool FAST> __device__ __forceinline__ float activate_slope(float z, int act) {
  switch (act) {
    case GBMUF_ACT_RELU: return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    case GBMUF_ACT_GELU: {
      float g;
      const float c = clamp100(z), phi = normal_cdf<FAST>(c, g);
      return fmaf(c * 0.39894228040143268f, g, phi);
    }
    case GBMUF_ACT_SILU: {
      const float c = clamp100(z), s = logistic<FAST>(c);
      return s * (1.0f + c * (1.0f - s));
    }
    case GBMUF_ACT_TANH: { const float t = tanh_of<FAST>(z); return 1.0f - t * t; }
    case GBMUF_ACT_SIGMOID: { const float s = logistic<FAST>(z); return s * (1.0f - s); }
    default: return 1.0f;
  }
}
template <bool FAST, int N> __device__ __forceinline__ void activate_all(float (&v)[N], int act) {
  switch (act) {                                           // the choice outside the loop
#define EACH(A) case A: _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = activate<FAST>(v[i], A); break;
    EACH(GBMUF_ACT_RELU) EACH(GBMUF_ACT_GELU) EACH(GBMUF_ACT_SILU) EACH(GBMUF_ACT_TANH) EACH(GBMUF_ACT_SIGMOID)
#undef EACH
  }
}
// v *= act'(z)
template <bool FAST, int N> __device__ __forceinline__ void slope_all(float (&v)[N], const float (&z)[N], int act) {
  switch (act) {
#define EACH(A) case A: _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] *= activate_slope<FAST>(z[i], A); break;
    EACH(GBMUF_ACT_RELU) EACH(GBMUF_ACT_GELU) EACH(GBMUF_ACT_SILU) EACH(GBMUF_ACT_TANH) EACH(GBMUF_ACT_SIGMOID)
#undef EACH
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
  int pairs;           // bf16: every matrix above may be accessed two columns at a time
};

// Single elements.
template <int KIND, typename T, typename TO>
__device__ __forceinline__ void finish_element(const Epilogue& E, long long r, long long c, float acc) {
  constexpr bool FAST = sizeof(T) == 2;
  if (KIND == kForward) {
    const float z = E.bias ? acc + to_f32(static_cast<const T*>(E.bias)[c]) : acc;
    if (E.out1) static_cast<T*>(E.out1)[r * E.ld_out1 + c] = from_f32<T>(z);
    float y = activate<FAST>(z, E.act);
    if (E.residual) y += to_f32(static_cast<const T*>(E.residual)[r * E.ld_residual + c]);
    static_cast<T*>(E.out0)[r * E.ld_out0 + c] = from_f32<T>(y);
  } else if (KIND == kInputGrad) {
    float d = acc;
    if (E.residual) d += to_f32(static_cast<const T*>(E.residual)[r * E.ld_residual + c]);
    if (E.out0) static_cast<T*>(E.out0)[r * E.ld_out0 + c] = from_f32<T>(d);
    if (E.out1)
      static_cast<T*>(E.out1)[r * E.ld_out1 + c] =
          from_f32<T>(d * activate_slope<FAST>(to_f32(static_cast<const T*>(E.z_in)[r * E.ld_z_in + c]), E.act));
  } else {
    TO* const p = static_cast<TO*>(E.out0) + r * E.ld_out0 + c;
    *p = from_f32<TO>(E.accumulate ? acc + to_f32(*p) : acc);
  }
}

// N rows of a warp's 32 neighbouring columns: lane l holds column c (= c of lane 0 + l) of rows
// r .. r+N-1.  fp32 goes out as it is held, 128 bytes per row.  bf16 goes two columns at a time:
// lane pairs trade halves, so that the even lane has both columns of row r + j and the odd one those
// of row r + j + 1 (half the memory instructions of 16-bit accesses); a matrix whose alignment or odd
// width forbids that takes the 16-bit accesses.
__device__ __forceinline__ uint32_t trade_pairs(uint32_t u, int lane) {
  return __byte_perm(u, __shfl_xor_sync(~0u, u, 1), lane & 1 ? 0x3276 : 0x5410);
}
template <typename X, int N> struct Strip {
  uint32_t raw[N];

  // Asks for the values; unpack() has to come before the next use of the memory they came from.
  __device__ __forceinline__ void load(const void* base, long long ld, int r, int c, int R, int C, bool pairs, int lane) {
    if (sizeof(X) == 2 && pairs) {
      const int odd = lane & 1;
      const char* p = static_cast<const char*>(base) + ((r + odd) * ld + (c - odd)) * 2;
#pragma unroll
      for (int j = 0; j < N / 2; ++j)
        raw[j] = c - odd < C && r + odd + 2 * j < R ? *reinterpret_cast<const uint32_t*>(p + 4 * j * ld) : 0u;
    } else {
      const X* p = static_cast<const X*>(base) + r * ld + c;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (sizeof(X) == 2) raw[j] = c < C && r + j < R ? *reinterpret_cast<const uint16_t*>(p + j * ld) : 0u;
        else raw[j] = c < C && r + j < R ? *reinterpret_cast<const uint32_t*>(p + j * ld) : 0u;
      }
    }
  }
  __device__ __forceinline__ void unpack(float (&v)[N], bool pairs, int lane) const {
    if (sizeof(X) == 2 && pairs) {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const uint32_t u = trade_pairs(raw[j], lane);
        v[2 * j] = __uint_as_float(u << 16);
        v[2 * j + 1] = __uint_as_float(u & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = __uint_as_float(sizeof(X) == 2 ? raw[j] << 16 : raw[j]);
    }
  }
};
template <typename X, int N>
__device__ __forceinline__ void store_strip(const float (&v)[N], void* base, long long ld, int r, int c, int R, int C, bool pairs,
                                            int lane) {
  if (sizeof(X) == 2 && pairs) {
    const int odd = lane & 1;
    char* p = static_cast<char*>(base) + ((r + odd) * ld + (c - odd)) * 2;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      const uint32_t u = trade_pairs(*reinterpret_cast<const uint32_t*>(&h), lane);
      if (c - odd < C && r + odd + 2 * j < R) *reinterpret_cast<uint32_t*>(p + 4 * j * ld) = u;
    }
  } else {
    X* p = static_cast<X*>(base) + r * ld + c;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (c < C && r + j < R) p[j * ld] = from_f32<X>(v[j]);
  }
}

// The epilogue of N rows.  ask() requests what the epilogue reads, early; finish() takes the sums.
template <int KIND, typename T, typename TO, int N> struct Finisher {
  Strip<T, N> first, second;          // residual (or dw), z_in

  __device__ __forceinline__ void ask(const Epilogue& E, int r, int c, int R, int C, int lane) {
    if (KIND != kWeightGrad && E.residual) first.load(E.residual, E.ld_residual, r, c, R, C, E.pairs, lane);
    if (KIND == kInputGrad && E.out1) second.load(E.z_in, E.ld_z_in, r, c, R, C, E.pairs, lane);
  }
  // All lanes of a warp, whether or not their column exists.  bias: that of column c.
  __device__ __forceinline__ void finish(const Epilogue& E, int r, int c, int R, int C, int lane, float bias, float (&v)[N]) {
    constexpr bool FAST = sizeof(T) == 2;
    float x[N];
    if (KIND == kForward) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += bias;
      if (E.out1) store_strip<T>(v, E.out1, E.ld_out1, r, c, R, C, E.pairs, lane);
      activate_all<FAST>(v, E.act);
      if (E.residual) {
        first.unpack(x, E.pairs, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += x[i];
      }
      store_strip<T>(v, E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
    } else if (KIND == kInputGrad) {
      if (E.residual) {
        first.unpack(x, E.pairs, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += x[i];
      }
      if (E.out0) store_strip<T>(v, E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
      if (E.out1) {
        second.unpack(x, E.pairs, lane);
        slope_all<FAST>(v, x, E.act);
        store_strip<T>(v, E.out1, E.ld_out1, r, c, R, C, E.pairs, lane);
      }
    } else {
      if (E.accumulate) {
        Strip<TO, N> old;
        old.load(E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
        old.unpack(x, E.pairs, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += x[i];
      }
      store_strip<TO>(v, E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
    }
  }
};

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_EPILOGUE_CUH
