// Matrix products on the fp32 units, for any strides.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_LINEAR_SIMT_CUH
#define GBMUF_CSRC_LINEAR_SIMT_CUH

namespace {

// C[r][c] = sum_k A(r, k) B(c, k), A(r, k) = a[r * sa_r + k * sa_k], B alike; 64 x 64 outputs per
// block of 256 threads, 4 x 4 per thread, 16 k per step through shared memory.
struct SimtParams {
  const void *a, *b;
  long long sa_r, sa_k, sb_c, sb_k;
  long long R, C, K;
  Epilogue E;
};

template <int KIND, typename T, typename TO>
__global__ void __launch_bounds__(256) linear_simt_kernel(const SimtParams P) {
  __shared__ float sa[16][65], sb[16][65];
  const T* const a = static_cast<const T*>(P.a);
  const T* const b = static_cast<const T*>(P.b);
  const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4;
  const long long tiles_c = (P.C + 63) / 64, tiles = tiles_c * ((P.R + 63) / 64);
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const long long r0 = tile / tiles_c * 64, c0 = tile % tiles_c * 64;
    float acc[4][4] = {};
    for (long long k0 = 0; k0 < P.K; k0 += 16) {
      for (int i = threadIdx.x; i < 1024; i += 256) {
        // consecutive threads along whichever index is contiguous in memory
        const int ka = P.sa_k == 1 ? i & 15 : i >> 6, ra = P.sa_k == 1 ? i >> 4 : i & 63;
        const int kb = P.sb_k == 1 ? i & 15 : i >> 6, cb = P.sb_k == 1 ? i >> 4 : i & 63;
        sa[ka][ra] = r0 + ra < P.R && k0 + ka < P.K ? to_f32(a[(r0 + ra) * P.sa_r + (k0 + ka) * P.sa_k]) : 0.0f;
        sb[kb][cb] = c0 + cb < P.C && k0 + kb < P.K ? to_f32(b[(c0 + cb) * P.sb_c + (k0 + kb) * P.sb_k]) : 0.0f;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        float x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = sa[k][tr + 16 * i]; y[i] = sb[k][tc + 16 * i]; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long r = r0 + tr + 16 * i, c = c0 + tc + 16 * j;
        if (r < P.R && c < P.C) finish_element<KIND, T, TO>(P.E, r, c, acc[i][j]);
      }
  }
}

// out[c] (+)= sum over the rows of a [R][C] matrix: one block per 32 columns, 8 row groups summed
// in a fixed order.
template <typename T, typename TO>
__global__ void __launch_bounds__(256) column_sum_kernel(const T* a, long long ld, long long R, long long C,
                                                         TO* out, int accumulate) {
  __shared__ float part[8][33];
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
  for (long long c0 = (long long)blockIdx.x * 32; c0 < C; c0 += (long long)gridDim.x * 32) {
    const long long c = c0 + lane;
    float s = 0.0f;
    if (c < C)
      for (long long r = g; r < R; r += 8) s += to_f32(a[r * ld + c]);
    part[g][lane] = s;
    __syncthreads();
    if (g == 0 && c < C) {
      float t = part[0][lane];
      for (int i = 1; i < 8; ++i) t += part[i][lane];
      out[c] = from_f32<TO>(accumulate ? t + to_f32(out[c]) : t);
    }
    __syncthreads();
  }
}

template <typename T>
__global__ void __launch_bounds__(256) activation_backward_kernel(const T* dy, long long ld_dy, const T* z,
                                                                  long long ld_z, T* dz, long long ld_dz,
                                                                  long long rows, long long cols, int act) {
  const long long n = rows * cols;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    const long long r = i / cols, c = i - r * cols;
    dz[r * ld_dz + c] = from_f32<T>(to_f32(dy[r * ld_dy + c]) * activate_slope(to_f32(z[r * ld_z + c]), act));
  }
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_SIMT_CUH
