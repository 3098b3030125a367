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

// Activations and their slopes, two values at a time.  Values beyond +-100 count as +-100 where an
// activation is flat there in fp32 (its exponentials are 0 or its limit is reached), so that infinities
// give the limits and not inf * 0; NaN stays NaN.  A slope that goes to 0 is formed as a product of what
// goes to 0, not as a difference of numbers near 1, so that its last digits hold (fp32).
//
// FAST (results that are rounded to bf16): exponentials and reciprocals are single instructions of the
// special-function unit, off by a few units of 2^-22; the accurate functions took twice the
// instructions of everything else in the epilogue and made it the bound.
__device__ __forceinline__ float clamp100(float z) { return z > 100.0f ? 100.0f : (z < -100.0f ? -100.0f : z); }

template <bool FAST> __device__ __forceinline__ Two decay(float a, float b) {          // exp(-a), exp(-b)
  if (!FAST) return two(expf(-a), expf(-b));
  float x, y;
  apart(two(a, b) * two(-1.44269504f, -1.44269504f), x, y);
  return two(exp2_unit(x), exp2_unit(y));
}
template <bool FAST> __device__ __forceinline__ Two reciprocal(Two t) {
  float x, y;
  apart(t, x, y);
  return FAST ? two(rcp_unit(x), rcp_unit(y)) : two(1.0f / x, 1.0f / y);
}
template <bool FAST> __device__ __forceinline__ Two logistic(float a, float b) {
  return reciprocal<FAST>(decay<FAST>(a, b) + two(1.0f, 1.0f));
}
// For a, b >= 0: q = 1 - Phi = erfc(x / sqrt 2) / 2 (Phi the normal distribution function) and
// g = exp(-x^2 / 2).  FAST: Abramowitz and Stegun 7.1.26, erfc(x) = (a1 t + .. + a5 t^5) exp(-x^2),
// t = 1 / (1 + p x), off by at most 1.5e-7.
template <bool FAST> __device__ __forceinline__ Two normal_tail(float a, float b, Two& g) {
  if (!FAST) {
    g = two(expf(-0.5f * a * a), expf(-0.5f * b * b));
    return two(0.5f * erfcf(0.70710678118654752f * a), 0.5f * erfcf(0.70710678118654752f * b));
  }
  const Two x = two(a, b);
  float u, v;
  apart(x * x * two(-0.72134752f, -0.72134752f), u, v);
  g = two(exp2_unit(u), exp2_unit(v));
  constexpr float kP = 0.3275911f * 0.70710678118654752f;
  apart(fma_two(x, two(kP, kP), two(1.0f, 1.0f)), u, v);
  const Two t = two(rcp_unit(u), rcp_unit(v));
  auto both = [](float c) { return two(0.5f * c, 0.5f * c); };
  Two q = fma_two(t, both(1.061405429f), both(-1.453152027f));
  q = fma_two(t, q, both(1.421413741f));
  q = fma_two(t, q, both(-0.284496736f));
  q = fma_two(t, q, both(0.254829592f));
  return q * t * g;
}
template <bool FAST> __device__ __forceinline__ float tanh_of(float z) {
  if (!FAST) return tanhf(z);
  const float s = z * z;                                   // below 0.15 the series: next term 17/315 z^7
  const float near = fmaf(z * s, fmaf(s, 2.0f / 15.0f, -1.0f / 3.0f), z);
  const float far = fmaf(-2.0f, rcp_unit(1.0f + exp2_unit(2.88539008f * z)), 1.0f);
  return fabsf(z) < 0.15f ? near : far;
}

template <bool FAST, int ACT> __device__ __forceinline__ void activate_two(float& a, float& b) {
  if (ACT == GBMUF_ACT_RELU) {
    a = a < 0.0f ? 0.0f : a;
    b = b < 0.0f ? 0.0f : b;
  } else if (ACT == GBMUF_ACT_GELU) {                      // z Phi(z) = max(z, 0) - |z| q(|z|)
    const float x = min_nan(fabsf(a), 100.0f), y = min_nan(fabsf(b), 100.0f);
    Two g;
    apart(fma_two(two(-x, -y), normal_tail<FAST>(x, y, g), two(fmaxf(a, 0.0f), fmaxf(b, 0.0f))), a, b);
  } else if (ACT == GBMUF_ACT_SILU) {
    const Two s = logistic<FAST>(a, b);
    apart(two(max_nan(a, -100.0f), max_nan(b, -100.0f)) * s, a, b);
  } else if (ACT == GBMUF_ACT_TANH) {
    a = tanh_of<FAST>(a);
    b = tanh_of<FAST>(b);
  } else if (ACT == GBMUF_ACT_SIGMOID) {
    apart(logistic<FAST>(a, b), a, b);
  }
}
template <bool FAST, int ACT> __device__ __forceinline__ Two slope_two(float a, float b) {
  const Two one = two(1.0f, 1.0f);
  if (ACT == GBMUF_ACT_RELU) return two(a > 0.0f ? 1.0f : (a <= 0.0f ? 0.0f : a), b > 0.0f ? 1.0f : (b <= 0.0f ? 0.0f : b));
  if (ACT == GBMUF_ACT_GELU) {                             // Phi(z) + z phi(z), Phi = q or 1 - q by the sign
    const float x = min_nan(fabsf(a), 100.0f), y = min_nan(fabsf(b), 100.0f);
    Two g;
    float u, v, cu, cv;
    const Two q = normal_tail<FAST>(x, y, g);
    apart(q, u, v);
    apart(one - q, cu, cv);
    const Two phi = two(a < 0.0f ? u : cu, b < 0.0f ? v : cv);
    return fma_two(two(copysignf(x, a), copysignf(y, b)) * two(0.39894228f, 0.39894228f), g, phi);
  }
  if (ACT == GBMUF_ACT_SILU) {
    const Two s = logistic<FAST>(a, b);
    return s * fma_two(two(clamp100(a), clamp100(b)), one - s, one);
  }
  if (ACT == GBMUF_ACT_TANH) {                             // 4 e / (1 + e)^2, e = exp(-2 |z|)
    const Two e = decay<FAST>(2.0f * fabsf(a), 2.0f * fabsf(b)), r = reciprocal<FAST>(one + e);
    return e * two(4.0f, 4.0f) * (r * r);
  }
  if (ACT == GBMUF_ACT_SIGMOID) {                          // e / (1 + e)^2, e = exp(-|z|)
    const Two e = decay<FAST>(fabsf(a), fabsf(b)), r = reciprocal<FAST>(one + e);
    return e * (r * r);
  }
  return one;
}

template <bool FAST, int N> __device__ __forceinline__ void activate_all(float (&v)[N], int act) {
  switch (act) {                                           // the choice outside the loop
#define EACH(A) case A: _Pragma("unroll") for (int i = 0; i < N; i += 2) activate_two<FAST, A>(v[i], v[i + 1]); break;
    EACH(GBMUF_ACT_RELU) EACH(GBMUF_ACT_GELU) EACH(GBMUF_ACT_SILU) EACH(GBMUF_ACT_TANH) EACH(GBMUF_ACT_SIGMOID)
#undef EACH
  }
}
// v *= act'(z)
template <bool FAST, int N> __device__ __forceinline__ void slope_all(float (&v)[N], const float (&z)[N], int act) {
  switch (act) {
#define EACH(A)                                                                                        \
  case A:                                                                                              \
    _Pragma("unroll") for (int i = 0; i < N; i += 2)                                                   \
      apart(two(v[i], v[i + 1]) * slope_two<FAST, A>(z[i], z[i + 1]), v[i], v[i + 1]);                 \
    break;
    EACH(GBMUF_ACT_RELU) EACH(GBMUF_ACT_GELU) EACH(GBMUF_ACT_SILU) EACH(GBMUF_ACT_TANH) EACH(GBMUF_ACT_SIGMOID)
#undef EACH
  }
}

enum LinearKind { kForward = 0, kInputGrad = 1, kWeightGrad = 2, kLossStats = 3, kLossGrad = 4, kLossWeight = 5, kLossTerm = 6 };

// What happens to a finished sum `acc` of row r, column c of the result.  T: the type of all
// operands but the weight gradient, which is TO.
//   forward      z = acc + bias[c]; out1 <- z; out0 <- act(z) + residual
//   input grad   d = acc + residual; out0 <- d; out1 <- d * act'(z_in)
//   weight grad  out0 <- acc (+ out0); loss weight: out0 <- factor scale acc (+ out0), of other operands
//   loss stats, loss grad, loss term: linear_loss.cuh
struct Epilogue {
  const void* bias;
  const void* residual;
  const void* z_in;
  void* out0;
  void* out1;
  long long ld_residual, ld_z_in, ld_out0, ld_out1;
  int act, accumulate;
  int pairs;           // bf16: every matrix above may be accessed two columns at a time
  // of the loss alone
  const void* loss_rows;     // kLossStats: int64 targets; kLossGrad: RowPair
  const int* loss_targets;   // kLossGrad
  const float* loss_weights; // kLossGrad; kLossStats: row weights, where weight_max is wanted
  float* target_logit;       // kLossStats
  void* partial;             // kLossStats: float2 [slots][ld_partial]; kLossGrad: float [strips][ld_partial] or NULL
  long long ld_partial;
  long long part;            // kLossGrad, fp32: elements from one bf16 part of out0 to the next; kLossTerm: from one slice's
  int first_word, words;     // of the vocabulary's piece
  int rest_from;             // kLossGrad, bf16: rows from here on are the first ones again, of which the rounding's rest is stored
  float scale;               // kLossWeight: of the sums; kLossStats: of the weights
  const float* factor;       // kLossWeight, bf16 operands: of the sums too, in device memory, or NULL
  float* weight_max;         // kLossStats, bf16: the largest weight of each 32 rows, or NULL
  long long vocab, ignore_index;     // kLossStats, for weight_max
};

// N rows of a warp's 32 neighbouring columns: lane l holds column c (= c of lane 0 + l) of rows
// r .. r+N-1.  fp32 goes out as it is held, 128 bytes per row.  bf16 goes two columns at a time:
// lane pairs trade halves, so that the even lane has both columns of row r + j and the odd one those
// of row r + j + 1 (half the memory instructions of 16-bit accesses); a matrix whose alignment or odd
// width forbids that takes the 16-bit accesses.  WHOLE: all rows and columns exist, no tests.
__device__ __forceinline__ uint32_t trade_pairs(uint32_t u, int lane) {
  return __byte_perm(u, __shfl_xor_sync(~0u, u, 1), lane & 1 ? 0x3276 : 0x5410);
}
template <typename X, int N> struct Strip {
  uint32_t raw[sizeof(X) == 2 ? N / 2 : N];          // bf16: two rows to a word

  // Asks for the values; unpack() has to come before the next use of the memory they came from.  One
  // pointer walks down the rows: an address per row from scratch would be a third of the epilogue.
  template <bool WHOLE>
  __device__ __forceinline__ void load(const void* base, long long ld, int r, int c, int R, int C, bool pairs, int lane) {
    if (sizeof(X) == 2 && pairs) {
      const int odd = lane & 1;
      const char* p = static_cast<const char*>(base) + ((r + odd) * ld + (c - odd)) * 2;
#pragma unroll
      for (int j = 0; j < N / 2; ++j, p += 4 * ld)
        raw[j] = WHOLE || (c - odd < C && r + odd + 2 * j < R) ? *reinterpret_cast<const uint32_t*>(p) : 0u;
    } else {
      const X* p = static_cast<const X*>(base) + r * ld + c;
#pragma unroll
      for (int j = 0; j < N; ++j, p += ld) {
        const bool there = WHOLE || (c < C && r + j < R);
        if constexpr (sizeof(X) == 2) {
          const uint32_t h = there ? *reinterpret_cast<const uint16_t*>(p) : 0u;
          raw[j / 2] = j & 1 ? raw[j / 2] | h << 16 : h;
        } else {
          raw[j] = there ? *reinterpret_cast<const uint32_t*>(p) : 0u;
        }
      }
    }
  }
  __device__ __forceinline__ void unpack(float (&v)[N], bool pairs, int lane) const {
    if constexpr (sizeof(X) == 2) {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const uint32_t u = pairs ? trade_pairs(raw[j], lane) : raw[j];
        v[2 * j] = __uint_as_float(u << 16);
        v[2 * j + 1] = __uint_as_float(u & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = __uint_as_float(raw[j]);
    }
  }
};
template <typename X, bool WHOLE, int N>
__device__ __forceinline__ void store_strip(const float (&v)[N], void* base, long long ld, int r, int c, int R, int C, bool pairs,
                                            int lane) {
  if (sizeof(X) == 2 && pairs) {
    const int odd = lane & 1;
    char* p = static_cast<char*>(base) + ((r + odd) * ld + (c - odd)) * 2;
#pragma unroll
    for (int j = 0; j < N / 2; ++j, p += 4 * ld) {
      __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      const uint32_t u = trade_pairs(*reinterpret_cast<const uint32_t*>(&h), lane);
      if (WHOLE || (c - odd < C && r + odd + 2 * j < R)) *reinterpret_cast<uint32_t*>(p) = u;
    }
  } else {
    X* p = static_cast<X*>(base) + r * ld + c;
#pragma unroll
    for (int j = 0; j < N; ++j, p += ld)
      if (WHOLE || (c < C && r + j < R)) *p = from_f32<X>(v[j]);
  }
}

// The epilogue of N rows.  ask() requests what the epilogue reads, early; finish() takes the sums.
template <int KIND, typename T, typename TO, int N> struct Finisher {
  Strip<T, N> first, second;          // residual (or dw), z_in
  float factor;                       // kLossWeight

  template <bool WHOLE>
  __device__ __forceinline__ void ask_(const Epilogue& E, int r, int c, int R, int C, int lane) {
    if ((KIND == kForward || KIND == kInputGrad) && E.residual) first.template load<WHOLE>(E.residual, E.ld_residual, r, c, R, C, E.pairs, lane);
    if (KIND == kInputGrad && E.out1) second.template load<WHOLE>(E.z_in, E.ld_z_in, r, c, R, C, E.pairs, lane);
  }
  template <bool WHOLE>
  __device__ __forceinline__ void finish_(const Epilogue& E, int r, int c, int R, int C, int lane, float bias, float (&v)[N]) {
    constexpr bool FAST = sizeof(T) == 2;
    float x[N];
    if (KIND == kForward) {
#pragma unroll
      for (int i = 0; i < N; i += 2) apart(two(v[i], v[i + 1]) + two(bias, bias), v[i], v[i + 1]);
      if (E.out1) store_strip<T, WHOLE>(v, E.out1, E.ld_out1, r, c, R, C, E.pairs, lane);
      activate_all<FAST>(v, E.act);
      if (E.residual) {
        first.unpack(x, E.pairs, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += x[i];
      }
      store_strip<T, WHOLE>(v, E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
    } else if (KIND == kInputGrad) {
      if (E.residual) {
        first.unpack(x, E.pairs, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += x[i];
      }
      if (E.out0) store_strip<T, WHOLE>(v, E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
      if (E.out1) {
        second.unpack(x, E.pairs, lane);
        slope_all<FAST>(v, x, E.act);
        store_strip<T, WHOLE>(v, E.out1, E.ld_out1, r, c, R, C, E.pairs, lane);
      }
    } else {
      if (KIND == kLossWeight) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] * factor * E.scale;
      }
      if (E.accumulate) {
        Strip<TO, N> old;
        old.template load<WHOLE>(E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
        old.unpack(x, E.pairs, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += x[i];
      }
      store_strip<TO, WHOLE>(v, E.out0, E.ld_out0, r, c, R, C, E.pairs, lane);
    }
  }
  // All lanes of a warp, whether or not their column exists.  bias: that of column c.
  __device__ __forceinline__ void ask(const Epilogue& E, int r, int c, int R, int C, int lane) {
    if (whole(r, c, R, C, lane)) ask_<true>(E, r, c, R, C, lane); else ask_<false>(E, r, c, R, C, lane);
  }
  __device__ __forceinline__ void finish(const Epilogue& E, int r, int c, int R, int C, int lane, float bias, float (&v)[N]) {
    if (whole(r, c, R, C, lane)) finish_<true>(E, r, c, R, C, lane, bias, v); else finish_<false>(E, r, c, R, C, lane, bias, v);
  }
  __device__ __forceinline__ static bool whole(int r, int c, int R, int C, int lane) { return r + N <= R && c - lane + 32 <= C; }
};

// The forward epilogue of a single element.
template <typename T> __device__ __forceinline__ void finish_element(const Epilogue& E, long long r, long long c, float acc) {
  const float z = E.bias ? acc + to_f32(static_cast<const T*>(E.bias)[c]) : acc;
  if (E.out1) static_cast<T*>(E.out1)[r * E.ld_out1 + c] = from_f32<T>(z);
  float y[2] = {z, z};
  activate_all<sizeof(T) == 2>(y, E.act);
  if (E.residual) y[0] += to_f32(static_cast<const T*>(E.residual)[r * E.ld_residual + c]);
  static_cast<T*>(E.out0)[r * E.ld_out0 + c] = from_f32<T>(y[0]);
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_EPILOGUE_CUH
