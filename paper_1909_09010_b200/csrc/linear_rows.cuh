// The linear layer for a few rows (single tokens).
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_LINEAR_ROWS_CUH
#define GBMUF_CSRC_LINEAR_ROWS_CUH

namespace {

// For few rows the layer is one read of w [C][K].  All of x lies in shared memory; a warp takes NF
// rows of w (features) at a time, 16 bytes per lane and load, and keeps the NF x ROWS partial sums of
// its lane in registers, on the fp32 units: no operand is packed or split and any alignment will do
// (VEC false: element by element).  The 32 lanes' sums are joined by exchanging halves, so that
// NF x ROWS sums take about as many shuffles and not five each.
// Measured: 1 x 1,024 x 4,096 bf16 4.3 to 4.6 us (the tensor-core kernel 9.8); 8 x 512 x 267,735 fp32 97 to
// 99 us, 86 % of the copy rate (the tensor-core kernel, which has to pack the weights first, 478).
struct RowsParams {
  Epilogue E;
  const void *x, *w;
  long long ld_x, ld_w;
  int R, C, K;
};
constexpr int kRowsThreads = 512;
constexpr uint32_t kRowsMostBytes = 98304;       // of x: two blocks per SM

// W elements of NF features against ROWS rows of x.
template <typename T, int ROWS, int NF, int W>
__device__ __forceinline__ void rows_step(float (&acc)[NF * ROWS], const T (&u)[NF][W], const T* x, int kp) {
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    __align__(16) T xv[W];
    if constexpr (W > 1) *reinterpret_cast<uint4*>(xv) = *reinterpret_cast<const uint4*>(x + r * kp);
    else xv[0] = x[r * kp];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int j = 0; j < W; ++j) acc[f * ROWS + r] = fmaf(to_f32(u[f][j]), to_f32(xv[j]), acc[f * ROWS + r]);
  }
}

// LOSS: the layer is a softmax layer; its logits are not stored, a block leaves each row's maximum, the sum of the
// exponentials relative to it, and the target's logit (linear_loss.cuh joins the blocks).
template <typename T, int ROWS, bool VEC, bool LOSS = false>
__global__ void __launch_bounds__(kRowsThreads, 2) linear_rows_kernel(const RowsParams P) {
  constexpr int NF = ROWS >= 16 ? 2 : 4, NA = NF * ROWS, V = VEC ? 16 / (int)sizeof(T) : 1;
  extern __shared__ __align__(128) unsigned char smem[];
  grid_launch_dependents();
  grid_dependency_wait();
  T* const xs = reinterpret_cast<T*>(smem);
  const int kp = (P.K + 7) & ~7;                 // row stride in shared memory
  for (int i = threadIdx.x; i < ROWS * kp; i += kRowsThreads) {
    const int r = i / kp, k = i - r * kp;
    xs[i] = r < P.R && k < P.K ? static_cast<const T*>(P.x)[r * P.ld_x + k] : from_f32<T>(0.0f);
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, warps = gridDim.x * (kRowsThreads / 32);
  float m = -INFINITY, s = 0.0f;                 // LOSS: of this lane's row and words
  for (int c0 = (blockIdx.x * (kRowsThreads / 32) + (threadIdx.x >> 5)) * NF; c0 < P.C; c0 += warps * NF) {
    float acc[NA] = {};
    const T* w[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) w[f] = static_cast<const T*>(P.w) + (long long)(c0 + f < P.C ? c0 + f : c0) * P.ld_w;
    int k = lane * V;
    constexpr int AHEAD = ROWS <= 4 ? 2 : 1;     // steps whose loads are in flight together
    for (; k + (AHEAD - 1) * 32 * V + V <= P.K; k += AHEAD * 32 * V) {
      __align__(16) T u[AHEAD][NF][V];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const T* const p = w[f] + k + a * 32 * V;
          if constexpr (VEC) *reinterpret_cast<uint4*>(u[a][f]) = __ldcs(reinterpret_cast<const uint4*>(p));
          else u[a][f][0] = *p;
        }
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) rows_step<T, ROWS, NF, V>(acc, u[a], xs + k + a * 32 * V, kp);
    }
    if (AHEAD > 1)
      for (; k + V <= P.K; k += 32 * V) {
        __align__(16) T u[NF][V];
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          if constexpr (VEC) *reinterpret_cast<uint4*>(u[f]) = __ldcs(reinterpret_cast<const uint4*>(w[f] + k));
          else u[f][0] = w[f][k];
        }
        rows_step<T, ROWS, NF, V>(acc, u, xs + k, kp);
      }
    if (VEC) {                                   // the elements after the last whole 16 bytes
      const int e = P.K / V * V + lane;
      if (e < P.K) {
        T u[NF][1];
#pragma unroll
        for (int f = 0; f < NF; ++f) u[f][0] = w[f][e];
        rows_step<T, ROWS, NF, 1>(acc, u, xs + e, kp);
      }
    }
    // Exchange of halves: after the step with distance d a lane holds half as many sums, those whose
    // index has, at that bit, its own lane's bit d.
    int index = 0;
#pragma unroll
    for (int d = 16, n = NA / 2; d > 0; d >>= 1, n >>= 1) {
      if (n >= 1) {
        const bool upper = lane & d;
        if (upper) index += n;
#pragma unroll
        for (int i = 0; i < NA / 2; ++i)
          if (i < n) {
            const float give = upper ? acc[i] : acc[i + n], keep = upper ? acc[i + n] : acc[i];
            acc[i] = keep + __shfl_xor_sync(~0u, give, d);
          }
      } else {
        acc[0] += __shfl_xor_sync(~0u, acc[0], d);
      }
    }
    constexpr int SPARE = NA >= 32 ? 0 : 32 / NA - 1;      // lanes that hold the same sum
    const int c = c0 + index / ROWS, r = index % ROWS;
    if constexpr (!LOSS) {
      if ((lane & SPARE) == 0 && c < P.C && r < P.R) finish_element<T>(P.E, r, c, acc[0]);
    } else if (c < P.C && r < P.R) {
      const float z = P.E.bias ? acc[0] + to_f32(static_cast<const T*>(P.E.bias)[c]) : acc[0];
      if ((lane & SPARE) == 0 && static_cast<const long long*>(P.E.loss_rows)[r] == c) P.E.target_logit[r] = z;
      const float top = fmaxf(m, z);
      if (top == -INFINITY) s += z == z ? 0.0f : z;        // nothing but -inf and NaN
      else s = (m == -INFINITY ? s : s * expf(m - top)) + expf(z - top);
      m = top;
    }
  }
  if constexpr (LOSS) {
    // lanes that differ in the bits of the exchanges' first log2(NF) steps hold other words of the same row
    int index = 0;
#pragma unroll
    for (int d = 16, n = NA / 2; n >= 1 && d > 0; d >>= 1, n >>= 1)
      if (lane & d) index += n;
#pragma unroll
    for (int d = 16, f = NF / 2; f >= 1; d >>= 1, f >>= 1) {
      const float m2 = __shfl_xor_sync(~0u, m, d), s2 = __shfl_xor_sync(~0u, s, d);
      join_stats(m, s, make_float2(m2, s2));
    }
    __shared__ float2 stat[kRowsThreads / 32][ROWS];
    if (index < ROWS && (lane & (NA >= 32 ? 0 : 32 / NA - 1)) == 0) stat[threadIdx.x >> 5][index] = make_float2(m, s);
    __syncthreads();
    const int r = threadIdx.x;
    if (r < ROWS && r < P.R) {
      m = -INFINITY;
      s = 0.0f;
      for (int w = 0; w < kRowsThreads / 32; ++w) join_stats(m, s, stat[w][r]);
      static_cast<float2*>(P.E.partial)[(long long)blockIdx.x * P.E.ld_partial + r] = make_float2(m, s);
    }
  }
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_ROWS_CUH
