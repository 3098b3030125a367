// Matrix products on the fp32 units, for any strides.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_LINEAR_SIMT_CUH
#define GBMUF_CSRC_LINEAR_SIMT_CUH

namespace {

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
    dz[r * ld_dz + c] = from_f32<T>(to_f32(dy[r * ld_dy + c]) * activate_slope<sizeof(T) == 2>(to_f32(z[r * ld_z + c]), act));
  }
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_SIMT_CUH
