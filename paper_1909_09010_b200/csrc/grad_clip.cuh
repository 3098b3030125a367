// The norm over all gradients of a group (a worker) and the clipped copy.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_GRAD_CLIP_CUH
#define GBMUF_CSRC_GRAD_CLIP_CUH

namespace {

// A tensor of the handle's table, tensors sorted by group.  Its elements, row after row, are cut
// into chunks of kClipChunk; chunk0 is the number of chunks of the tensors before it.
constexpr int kClipChunk = 8192;
struct ClipTensor {
  const void* grad;
  void* out;
  long long n, cols, ld_grad, ld_out, chunk0;
  int32_t dtype, out_dtype, group;
  int32_t run;         // groups before this one that have a tensor
};
// Block b of the norm kernel takes chunks [b C / G, (b + 1) C / G).  Its sum over the chunks of run
// r goes to slot b + r: blocks and runs both ascend along the chunks, so no two pairs share a slot
// and the slots of a run are consecutive.
struct ClipParams {
  const ClipTensor* tensors;
  double* partial;
  float* norms;
  long long chunks;
  const int* slots;    // [groups][2]: first slot of the group and their number
  int count, groups, blocks;
  float max_norm;
};

__device__ __forceinline__ long long clip_chunk_of(const ClipParams& P, int b) { return P.chunks * b / P.blocks; }

// The tensor that chunk c belongs to: the last one with chunk0 <= c (an empty one has the chunk0 of
// the next).
__device__ __forceinline__ int clip_find(const ClipParams& P, long long c) {
  int lo = 0, hi = P.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (P.tensors[mid].chunk0 <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* scratch) {
  for (int d = 16; d > 0; d >>= 1) v += __shfl_down_sync(~0u, v, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = scratch[0];
  for (int w = 1; w < (int)(blockDim.x >> 5); ++w) s += scratch[w];
  return s;
}

__device__ __forceinline__ float clip_load(const ClipTensor& t, long long e) {
  const long long at = t.cols == t.ld_grad ? e : e / t.cols * t.ld_grad + e % t.cols;
  return t.dtype == GBMUF_F32 ? static_cast<const float*>(t.grad)[at]
                              : __bfloat162float(static_cast<const __nv_bfloat16*>(t.grad)[at]);
}

__global__ void __launch_bounds__(256) clip_norm_kernel(const ClipParams P) {
  __shared__ double scratch[8];
  const long long first = clip_chunk_of(P, blockIdx.x), end = clip_chunk_of(P, blockIdx.x + 1);
  if (first == end) return;
  int i = clip_find(P, first);
  double acc = 0.0;
  int run = P.tensors[i].run;
  for (long long c = first; c < end; ++c) {
    while (i + 1 < P.count && P.tensors[i + 1].chunk0 <= c) ++i;
    const ClipTensor& t = P.tensors[i];
    if (t.run != run) {
      const double s = block_sum(acc, scratch);
      if (threadIdx.x == 0) P.partial[blockIdx.x + run] = s;
      run = t.run;
      acc = 0.0;
    }
    const long long e0 = (c - t.chunk0) * kClipChunk, e1 = e0 + kClipChunk < t.n ? e0 + kClipChunk : t.n;
    for (long long e = e0 + threadIdx.x; e < e1; e += 256) {
      const double g = clip_load(t, e);
      acc += g * g;
    }
  }
  const double s = block_sum(acc, scratch);
  if (threadIdx.x == 0) P.partial[blockIdx.x + run] = s;
}

// Norm of group g from its slots, the same bits in every block.
__device__ __forceinline__ float clip_group_norm(const ClipParams& P, int g, double* scratch) {
  double v = 0.0;
  const int first = P.slots[2 * g], n = P.slots[2 * g + 1];
  for (int i = threadIdx.x; i < n; i += blockDim.x) v += P.partial[first + i];
  return (float)sqrt(block_sum(v, scratch));
}

__global__ void __launch_bounds__(256) clip_finish_kernel(const ClipParams P) {
  __shared__ double scratch[8];
  for (int g = blockIdx.x; g < P.groups; g += gridDim.x) {
    const float norm = clip_group_norm(P, g, scratch);
    if (threadIdx.x == 0) P.norms[g] = norm;
  }
}

__global__ void __launch_bounds__(256) clip_scale_kernel(const ClipParams P) {
  __shared__ double scratch[8];
  for (int g = blockIdx.x; g < P.groups; g += gridDim.x) {
    const float norm = clip_group_norm(P, g, scratch);
    if (threadIdx.x == 0) P.norms[g] = norm;
  }
  const long long first = clip_chunk_of(P, blockIdx.x), end = clip_chunk_of(P, blockIdx.x + 1);
  if (first == end) return;
  int i = clip_find(P, first), group = -1;
  float scale = 1.0f;
  bool zero = false;
  for (long long c = first; c < end; ++c) {
    while (i + 1 < P.count && P.tensors[i + 1].chunk0 <= c) ++i;
    const ClipTensor& t = P.tensors[i];
    if (t.group != group) {
      group = t.group;
      const float norm = clip_group_norm(P, group, scratch);
      zero = !(norm <= 3.402823466e38f);
      scale = P.max_norm > 0.0f ? __fdiv_rn(P.max_norm, norm > P.max_norm ? norm : P.max_norm) : 1.0f;
    }
    if (!t.out) continue;
    const long long e0 = (c - t.chunk0) * kClipChunk, e1 = e0 + kClipChunk < t.n ? e0 + kClipChunk : t.n;
    for (long long e = e0 + threadIdx.x; e < e1; e += 256) {
      const float v = zero ? 0.0f : __fmul_rn(clip_load(t, e), scale);
      const long long at = t.cols == t.ld_out ? e : e / t.cols * t.ld_out + e % t.cols;
      if (t.out_dtype == GBMUF_F32) static_cast<float*>(t.out)[at] = v;
      else static_cast<__nv_bfloat16*>(t.out)[at] = __float2bfloat16_rn(v);
    }
  }
}

}  // namespace

#endif  // GBMUF_CSRC_GRAD_CLIP_CUH
