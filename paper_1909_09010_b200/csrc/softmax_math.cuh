// Exponentials of logits, and what the statistics of a row say about its loss.
// Part of libgbmuf (CUDA, sm_100a); included by the local-step operators' translation units.
#ifndef GBMUF_CSRC_SOFTMAX_MATH_CUH
#define GBMUF_CSRC_SOFTMAX_MATH_CUH

namespace {

struct LossParams {
  const void* logits;
  const int64_t* targets;
  const float* row_weight;
  float *loss, *lse;
  void* dlogits;
  long long rows, vocab, ld, ld_d;
  long long ignore_index;
  float scale;
  int32_t* status;
  int split;           // CTAs per row (ring kernel)
};

// e^t for t <= 0, two at a time: 2^y with y = t log2 e from the special-function unit.  bf16 logits (FAST): the
// rounding of y, 2^-24 of at most a few tens, is far below bf16.  fp32: what y lost (its rounding, and that of
// log2 e) is computed exactly as f and put back as the factor 1 + f ln 2.
template <bool FAST> __device__ __forceinline__ Two exp_of(Two t) {
  constexpr float kHi = 1.44269502f, kLo = 1.925963033e-8f, kLn2 = 0.693147181f;       // log2 e = kHi + kLo
  float y0, y1;
  if (FAST) {
    apart(t * two(kHi, kHi), y0, y1);
    return two(exp2_unit(y0), exp2_unit(y1));
  }
  apart(t, y0, y1);                                        // -inf would give inf - inf below; NaN stays
  t = two(max_nan(y0, -200.0f), max_nan(y1, -200.0f));
  const Two y = t * two(kHi, kHi);
  const Two f = fma_two(t, two(kLo, kLo), fma_two(t, two(kHi, kHi), y * two(-1.0f, -1.0f)));
  apart(y, y0, y1);
  const Two r = two(exp2_unit(y0), exp2_unit(y1));
  return fma_two(r, f * two(kLn2, kLn2), r);
}
// exp(x - m) for a fixed m; m = -inf counts as 0.  The difference comes first (and not x log2 e - m log2 e in one
// operation) so that x = m gives 1 exactly and no finite logit overflows.
template <bool FAST> struct Shift {
  float m;
  __device__ __forceinline__ void set(float top) { m = top == -INFINITY ? 0.0f : top; }
  __device__ __forceinline__ Two operator()(float x0, float x1) const { return exp_of<FAST>(two(x0, x1) + two(-m, -m)); }
  __device__ __forceinline__ float operator()(float x) const {
    float a, b;
    apart((*this)(x, x), a, b);
    return a;
  }
};

// What the statistics of a row say: its loss and whether its gradient is zero.
struct RowOutcome { float lse, loss; bool zero; };
__device__ __forceinline__ bool target_ignored(const LossParams& P, long long t, float w) { return t == P.ignore_index || w == 0.0f; }
__device__ __forceinline__ bool target_inside(const LossParams& P, long long t) { return t >= 0 && t < P.vocab; }
__device__ __forceinline__ RowOutcome row_outcome(const LossParams& P, float m, float sum, float x_target, long long t, float w) {
  RowOutcome o;
  const bool empty = m == -INFINITY && sum == 0.0f;
  const float l = logf(sum);
  o.lse = empty ? -INFINITY : m + l;
  const bool ignored = target_ignored(P, t, w), outside = !ignored && !target_inside(P, t);
  o.zero = ignored || outside || empty;
  // not lse - x_target: what the logits have in common would take digits from the logarithm
  o.loss = ignored ? 0.0f : outside ? NAN : empty ? INFINITY : w * ((m - x_target) + l);
  return o;
}
__device__ __forceinline__ void report_target(const LossParams& P, long long t, float w) {
  if (!target_ignored(P, t, w) && !target_inside(P, t)) atomicExch(P.status, (int32_t)GBMUF_ERR_INVALID_ARG);
}

// log z to 2^-24 or so whatever its size: the exponent's part in 64 bits, beside the logarithm of 0.7 .. 1.4.
__device__ __forceinline__ double log_of(float z) {
  if (!(z > 1e-37f && z < 3.4e38f)) return (double)logf(z);
  const uint32_t b = __float_as_uint(z), shifted = b - 0x3f350000u;           // sqrt 1/2
  const int e = (int)shifted >> 23;
  return (double)e * 0.69314718055994531 + (double)logf(__uint_as_float(b - ((uint32_t)e << 23)));
}
// exp((x - m) / T), as Shift: log2 e / T = hi + lo; below `least` (x - m) the result is 0 in fp32.
struct Temperature {
  float hi, lo, least;
  double inverse;            // 1 / T
};
template <bool FAST> struct TemperedShift {
  float m, hi, lo, least;
  __device__ __forceinline__ void at(const Temperature& t) { hi = t.hi; lo = t.lo; least = t.least; }
  __device__ __forceinline__ void set(float top) { m = top == -INFINITY ? 0.0f : top; }
  __device__ __forceinline__ Two operator()(float x0, float x1) const {
    Two t = two(x0, x1) + two(-m, -m);
    float y0, y1;
    if (FAST) {
      apart(t * two(hi, hi), y0, y1);
      return two(exp2_unit(y0), exp2_unit(y1));
    }
    apart(t, y0, y1);
    t = two(max_nan(y0, least), max_nan(y1, least));
    const Two y = t * two(hi, hi);
    const Two f = fma_two(t, two(lo, lo), fma_two(t, two(hi, hi), y * two(-1.0f, -1.0f)));
    apart(y, y0, y1);
    const Two r = two(exp2_unit(y0), exp2_unit(y1));
    return fma_two(r, f * two(0.693147181f, 0.693147181f), r);
  }
  __device__ __forceinline__ float operator()(float x) const {
    float a, b;
    apart((*this)(x, x), a, b);
    return a;
  }
};

}  // namespace

#endif  // GBMUF_CSRC_SOFTMAX_MATH_CUH
