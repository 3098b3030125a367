// Column sums, and the gradient of an activation by itself.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_COLUMN_SUM_CUH
#define GBMUF_CSRC_COLUMN_SUM_CUH

namespace {

// out[c] (+)= sum over the rows of a [R][C] matrix.  A cluster takes a strip of columns (VEC: 128
// bytes wide, 16 bytes per thread; else 32 columns) and shares its rows; sums are joined through
// shared memory and rank 0's shared memory, in a fixed order; every rank arrives at the cluster's barrier
// first thing and waits for it after its rows, so that rank 0 has started before anybody writes there.
// Bound by memory latency: 8,192 x 4,096 bf16 in 10 to 14 us (5 to 6.7 TB/s, part of it from L2 behind the
// product that reads the same matrix); one block per strip without a cluster took 366.
template <typename T, typename TO, bool VEC>
__global__ void __launch_bounds__(256) column_sum_kernel(const T* a, long long ld, long long R, long long C, TO* out,
                                                         int accumulate) {
  constexpr int W = VEC ? 16 / (int)sizeof(T) : 1, L = VEC ? 8 : 32, ROWS = 256 / L, COLS = L * W;
  __shared__ float part[ROWS][COLS + 1];
  __shared__ float ranks[8][COLS];
  cluster_arrive();
  grid_launch_dependents();
  grid_dependency_wait();
  uint32_t share, rank;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(share));
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const long long c0 = (long long)(blockIdx.x / share) * COLS;
  const int lane = threadIdx.x % L, row = threadIdx.x / L;
  const long long c = c0 + lane * W;
  float s[W] = {};
  if (c < C) {                                              // VEC: C is a multiple of W
    const T* p = a + c;
    const long long step = (long long)share * ROWS;
#pragma unroll 8
    for (long long r = (long long)rank * ROWS + row; r < R; r += step) {
      __align__(16) T v[W];
      if constexpr (VEC) *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(p + r * ld);
      else v[0] = p[r * ld];
#pragma unroll
      for (int i = 0; i < W; ++i) s[i] += to_f32(v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i) part[row][lane * W + i] = s[i];
  __syncthreads();
  cluster_wait();
  if (threadIdx.x < COLS) {
    float t = part[0][threadIdx.x];
    for (int i = 1; i < ROWS; ++i) t += part[i][threadIdx.x];
    st_remote(smem_u32(&ranks[rank][threadIdx.x]), 0, t);
  }
  cluster_sync();
  if (rank == 0 && threadIdx.x < COLS && c0 + threadIdx.x < C) {
    float t = ranks[0][threadIdx.x];
    for (uint32_t q = 1; q < share; ++q) t += ranks[q][threadIdx.x];
    TO* const o = out + c0 + threadIdx.x;
    *o = from_f32<TO>(accumulate ? t + to_f32(*o) : t);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) activation_backward_kernel(const T* dy, long long ld_dy, const T* z,
                                                                  long long ld_z, T* dz, long long ld_dz,
                                                                  long long rows, long long cols, int act) {
  grid_launch_dependents();
  grid_dependency_wait();
  const long long n = rows * cols;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    const long long r = i / cols, c = i - r * cols;
    float v[2] = {to_f32(dy[r * ld_dy + c]), 0.0f};
    const float y = to_f32(z[r * ld_z + c]), at[2] = {y, y};
    slope_all<sizeof(T) == 2>(v, at, act);
    dz[r * ld_dz + c] = from_f32<T>(v[0]);
  }
}

}  // namespace

#endif  // GBMUF_CSRC_COLUMN_SUM_CUH
