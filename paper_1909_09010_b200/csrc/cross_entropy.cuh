// Cross-entropy of a softmax over a vocabulary, with its gradient.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_CROSS_ENTROPY_CUH
#define GBMUF_CSRC_CROSS_ENTROPY_CUH

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
};

// (m, s): s = sum of exp(x - m).  m = -inf: nothing but -inf so far, s = 0 (or NaN).
__device__ __forceinline__ void softmax_merge(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  if (top == -INFINITY) { s += s2; return; }
  s = s * expf(m - top) + s2 * expf(m2 - top);
  m = top;
}

// The weight a single logit enters with: 1, 0 for -inf, NaN for +inf and NaN.
__device__ __forceinline__ float softmax_unit(float x) { return x == -INFINITY ? 0.0f : 1.0f + (x - x); }

// What the statistics of a row say: its loss, the factor of its gradient and whether that is zero.
struct RowOutcome { float lse, loss, s; long long target; bool zero; };

__device__ __forceinline__ RowOutcome row_outcome(const LossParams& P, long long row, float m, float sum,
                                                  float x_target, long long t, float s) {
  RowOutcome o;
  const bool empty = m == -INFINITY && sum == 0.0f;
  o.lse = empty ? -INFINITY : m + logf(sum);
  o.s = s;
  o.target = t;
  const bool ignored = t == P.ignore_index || s == 0.0f;
  const bool outside = !ignored && (t < 0 || t >= P.vocab);
  o.zero = ignored || outside || empty;
  o.loss = ignored ? 0.0f : outside ? NAN : empty ? INFINITY : s * (o.lse - x_target);
  if (outside) atomicExch(P.status, (int32_t)GBMUF_ERR_INVALID_ARG);
  return o;
}

template <typename T>
__global__ void __launch_bounds__(256) cross_entropy_kernel(const LossParams P) {
  __shared__ float sm[8], ss[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
    float m = -INFINITY, s = 0.0f;
    for (long long v = threadIdx.x; v < P.vocab; v += 256) softmax_merge(m, s, to_f32(x[v]), softmax_unit(to_f32(x[v])));
    for (int d = 16; d > 0; d >>= 1) {
      const float m2 = __shfl_xor_sync(~0u, m, d), s2 = __shfl_xor_sync(~0u, s, d);
      softmax_merge(m, s, m2, s2);
    }
    if (lane == 0) { sm[warp] = m; ss[warp] = s; }
    __syncthreads();
    m = sm[0]; s = ss[0];
    for (int w = 1; w < 8; ++w) softmax_merge(m, s, sm[w], ss[w]);
    const long long t = P.targets[row];
    const float w = P.scale * (P.row_weight ? P.row_weight[row] : 1.0f);
    const float xt = t >= 0 && t < P.vocab ? to_f32(x[t]) : 0.0f;
    __syncthreads();                                       // dlogits may be the logits
    const RowOutcome o = row_outcome(P, row, m, s, xt, t, w);
    if (threadIdx.x == 0) {
      if (P.loss) P.loss[row] = o.loss;
      if (P.lse) P.lse[row] = o.lse;
    }
    if (P.dlogits) {
      T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
      const float inv = 1.0f / s;
      for (long long v = threadIdx.x; v < P.vocab; v += 256)
        d[v] = from_f32<T>(o.zero ? 0.0f : o.s * (expf(to_f32(x[v]) - m) * inv - (v == t ? 1.0f : 0.0f)));
    }
  }
}

}  // namespace

#endif  // GBMUF_CSRC_CROSS_ENTROPY_CUH
