// The norm over all gradients of a group (a worker) and the clipped copy.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_GRAD_CLIP_CUH
#define GBMUF_CSRC_GRAD_CLIP_CUH

namespace {

// norm_g = sqrt(sum x^2) over the tensors of group g, and out = x * (c / max(norm_g, c)): both bound
// by memory (2 or 4 bytes read per element for the norm; the copy reads them again, unless they are
// still in the L2 cache, and writes 2 or 4).  Two kernels of the same build: a block's producer warp
// has the copy engine fetch its chunks into a ring of shared-memory slots, 256 threads sum or scale
// them from there.  The gradients' loads so never wait for arithmetic, nor for the stores (loads
// into registers, 64 KB of them in flight per SM, reached 3.6 TB/s in the norm pass).
//
// Measured, 954 M bf16 elements to fp32: norms 290 to 318 us (6.0 to 6.6 TB/s), copy 990 to 1,000 us (5.7 to
// 5.8 TB/s).
//
// The handle's table: one entry per run of elements that follow one another in memory, sorted by
// group, cut into chunks of kClipSlot bytes at multiples of 16 bytes.  A tensor of short strided
// rows is one entry that is read element by element ("direct").
constexpr int kClipSlot = 32768;                 // (six of 16 KB: norm pass 352 us, three of 32 KB: 318)
constexpr int kClipRing = 3;
constexpr int kClipKeep = 6;                     // chunks per block that L2 keeps for the copy: 58 MB in all (10 MB of gradients: 23 us with all of them passing, 16 with these kept)
constexpr int kClipWorkers = 256;                // threads that sum or scale
constexpr int kClipThreads = kClipWorkers + 32;
constexpr int kClipBlocksPerSm = 2;
constexpr uint32_t kClipSmem = 128 + kClipRing * kClipSlot;

struct ClipEntry {
  const void* grad;
  void* out;
  long long n, cols, ld_grad, ld_out;            // cols, ld: of a direct entry
  long long chunk0;                              // chunks of the entries before this one
  int32_t dtype, out_dtype, group;
  int32_t run;                                   // groups before this one that have an entry
  int32_t direct;
  int32_t shift;                                 // elements by which grad is past a multiple of 16 bytes
};
// Block b takes chunks [b C / G, (b + 1) C / G).  Its sum over the chunks of run r goes to slot b + r:
// blocks and runs both ascend along the chunks, so no two pairs share a slot and the slots of a run
// are consecutive.
struct ClipParams {
  const ClipEntry* entries;
  double* partial;
  float* norms;
  int32_t* status;
  long long chunks;
  const int* slots;    // [groups][2]: first slot of the group and their number
  int count, groups, blocks;
  float max_norm;
};

__device__ __forceinline__ long long clip_chunk_of(const ClipParams& P, int b) { return P.chunks * b / P.blocks; }

// The entry that chunk c belongs to: the last one with chunk0 <= c.
__device__ __forceinline__ int clip_find(const ClipParams& P, long long c) {
  int lo = 0, hi = P.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (P.entries[mid].chunk0 <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int clip_chunk_elems(int dtype) { return dtype == GBMUF_F32 ? kClipSlot / 4 : kClipSlot / 2; }
// Chunk j of an entry: elements [e0, e1), of which [a0, a1) are whole 16-byte pieces of memory.
struct ClipSpan { long long e0, e1, a0, a1; };
__device__ __forceinline__ ClipSpan clip_span(const ClipEntry& t, long long j) {
  const int ch = clip_chunk_elems(t.dtype), v = t.dtype == GBMUF_F32 ? 4 : 8;
  ClipSpan s;
  s.e0 = j * ch - t.shift;
  s.e1 = s.e0 + ch < t.n ? s.e0 + ch : t.n;
  s.a1 = ((s.e1 + t.shift) & ~(long long)(v - 1)) - t.shift;
  s.a0 = s.e0;
  if (s.e0 < 0) { s.e0 = 0; s.a0 = v - t.shift; }
  if (t.direct || s.a1 <= s.a0) s.a0 = s.a1 = s.e1;
  return s;
}
// Where element e of a direct entry lies, in elements from its base.
__device__ __forceinline__ long long clip_at(const ClipEntry& t, long long e, long long ld) {
  return t.direct ? e / t.cols * ld + e % t.cols : e;
}

__device__ __forceinline__ void workers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kClipWorkers) : "memory"); }
// Sum over the worker threads, the same in all of them.
__device__ __forceinline__ double workers_sum(double v, double* scratch) {
  const int t = threadIdx.x;
  for (int d = 16; d > 0; d >>= 1) v += __shfl_down_sync(~0u, v, d);
  workers_sync();
  if ((t & 31) == 0) scratch[t >> 5] = v;
  workers_sync();
  double s = scratch[0];
  for (int w = 1; w < kClipWorkers / 32; ++w) s += scratch[w];
  return s;
}

// Sum of squares of up to four 16-byte pieces (raw words; zeros where there is none): in fp32, unless
// that leaves the range in which fp32 squares are exact to their last bits; then in double, as are the
// sums of these sums, so that every norm that fp32 can hold comes out right.  A sum has passed at most
// five fp32 roundings (fp32) or six (bf16, whose squares are exact), 6 x 2^-24; the square root halves that,
// and rounding the norm adds 2^-24: 2^-22 in all.  (Every square in double made the conversions the
// bound; one range test per four squares made each wait for the one before.)
template <bool F32> __device__ __forceinline__ float piece_value(uint4 u, int i) {
  const uint32_t w = i / (F32 ? 1 : 2) == 0 ? u.x : i / (F32 ? 1 : 2) == 1 ? u.y : i / (F32 ? 1 : 2) == 2 ? u.z : u.w;
  return __uint_as_float(F32 ? w : i & 1 ? w & 0xffff0000u : w << 16);
}
template <bool F32> __device__ __forceinline__ double square_sum(const uint4 (&u)[4]) {
  constexpr int E = F32 ? 4 : 8;
  float q[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const float x = piece_value<F32>(u[p], i), y = piece_value<F32>(u[p], i + 1);
      a = fmaf(x, x, a);
      b = fmaf(y, y, b);
    }
    q[p] = a + b;
  }
  const float t = (q[0] + q[1]) + (q[2] + q[3]);
  if (t > 1e-24f && t < 1e38f) return t;          // a square lost below 1e-38 is below 1e-14 of t
  double s = 0.0;
  for (int p = 0; p < 4; ++p) {
    if (((u[p].x | u[p].y | u[p].z | u[p].w) & 0x7fff7fffu) == 0 && !F32) continue;
    if (((u[p].x | u[p].y | u[p].z | u[p].w) & 0x7fffffffu) == 0) continue;
    for (int i = 0; i < E; ++i) { const double x = piece_value<F32>(u[p], i); s = fma(x, x, s); }
  }
  return s;
}

// Walks a block's chunks, upwards or downwards.
template <bool UP> struct ClipWalk {
  ClipEntry t;
  int i;
  long long c, left;
  __device__ __forceinline__ bool begin(const ClipParams& P) {
    const long long first = clip_chunk_of(P, blockIdx.x), end = clip_chunk_of(P, blockIdx.x + 1);
    left = end - first;
    if (left == 0) return false;
    c = UP ? first : end - 1;
    i = clip_find(P, c);
    t = P.entries[i];
    return true;
  }
  __device__ __forceinline__ bool next(const ClipParams& P) {
    if (--left == 0) return false;
    if (UP) {
      ++c;
      if (i + 1 < P.count && P.entries[i + 1].chunk0 <= c) t = P.entries[++i];
    } else {
      --c;
      if (t.chunk0 > c) t = P.entries[--i];
    }
    return true;
  }
};

// The producer warp: fetches the whole pieces of every chunk into the ring.
template <bool UP> __device__ __forceinline__ void clip_produce(const ClipParams& P, uint32_t bars, uint32_t ring) {
  if ((threadIdx.x & 31) != 0) return;
  ClipWalk<UP> w;
  int n = 0;
  bool ok = true;
  if (w.begin(P)) do {
      const ClipSpan s = clip_span(w.t, w.c - w.t.chunk0);
      if (s.a1 == s.a0 || (!UP && !w.t.out)) continue;
      const int slot = n % kClipRing;
      if (n >= kClipRing) ok = mbar_wait_bounded(bars + 64 + 8 * slot, (n / kClipRing - 1) & 1, P.status);
      if (!ok) break;
      const int size = w.t.dtype == GBMUF_F32 ? 4 : 2;
      const uint32_t bytes = (uint32_t)(s.a1 - s.a0) * size;
      mbar_arrive_expect_tx(bars + 8 * slot, bytes);
      // the norm pass ends with the chunks that the copy begins with
      bulk_load_hint(ring + slot * kClipSlot, static_cast<const char*>(w.t.grad) + s.a0 * size, bytes, bars + 8 * slot,
                     UP && w.left <= kClipKeep);
      ++n;
    } while (w.next(P));
  if (!ok)                                       // copies requested into this block's memory land first
    for (int j = n > kClipRing ? n - kClipRing : 0; j < n; ++j)
      mbar_wait_bounded(bars + 8 * (j % kClipRing), (j / kClipRing) & 1, P.status);
}

__device__ __forceinline__ void clip_prologue(unsigned char* smem) {
  if (threadIdx.x == 0) {
    const uint32_t bars = smem_u32(smem);
    for (int r = 0; r < kClipRing; ++r) { mbar_init(bars + 8 * r, 1); mbar_init(bars + 64 + 8 * r, kClipWorkers / 32); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
}

__device__ __forceinline__ float clip_single(const ClipEntry& t, long long e) {
  const long long at = clip_at(t, e, t.ld_grad);
  return t.dtype == GBMUF_F32 ? static_cast<const float*>(t.grad)[at] : to_f32(static_cast<const __nv_bfloat16*>(t.grad)[at]);
}
// Element number k of those of a chunk that are not in the ring.
__device__ __forceinline__ long long clip_outside(const ClipSpan& s, long long k) {
  const long long head = s.a0 - s.e0;
  return k < head ? s.e0 + k : s.a1 + (k - head);
}

__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm) clip_norm_kernel(const ClipParams P) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ double scratch[kClipWorkers / 32];
  const uint32_t bars = smem_u32(smem);
  clip_prologue(smem);
  grid_launch_dependents();
  grid_dependency_wait();
  if (threadIdx.x >= kClipWorkers) { clip_produce<true>(P, bars, bars + 128); return; }
  ClipWalk<true> w;
  w.begin(P);                                    // every block has a chunk
  double s0 = 0.0, s1 = 0.0;
  int run = w.t.run, n = 0;
  bool ok = true;
  do {
    if (w.t.run != run) {
      const double sum = workers_sum(s0 + s1, scratch);
      if (threadIdx.x == 0) P.partial[blockIdx.x + run] = sum;
      run = w.t.run;
      s0 = s1 = 0.0;
    }
    const ClipSpan s = clip_span(w.t, w.c - w.t.chunk0);
    if (s.a1 > s.a0) {
      const int slot = n % kClipRing;
      ok = ok && mbar_wait_bounded(bars + 8 * slot, (n / kClipRing) & 1, P.status);
      const uint4* const p = reinterpret_cast<const uint4*>(smem + 128 + slot * kClipSlot);
      const int pieces = (int)(s.a1 - s.a0) / (w.t.dtype == GBMUF_F32 ? 4 : 8);
      if (ok)
        for (int k = threadIdx.x; k < pieces; k += 4 * kClipWorkers) {
          uint4 u[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) u[j] = k + j * kClipWorkers < pieces ? p[k + j * kClipWorkers] : make_uint4(0, 0, 0, 0);
          s0 += w.t.dtype == GBMUF_F32 ? square_sum<true>(u) : square_sum<false>(u);
        }
      __syncwarp();                              // one arrival per warp: they are serialised
      if ((threadIdx.x & 31) == 0) mbar_arrive(bars + 64 + 8 * slot);
      ++n;
    }
    const long long rest = (s.e1 - s.e0) - (s.a1 - s.a0);
#pragma unroll 4
    for (long long k = threadIdx.x; k < rest; k += kClipWorkers) {
      const double g = clip_single(w.t, clip_outside(s, k));
      s1 = fma(g, g, s1);
    }
  } while (w.next(P));
  const double sum = workers_sum(s0 + s1, scratch);
  if (threadIdx.x == 0) P.partial[blockIdx.x + run] = sum;
}

// Norm of group g from its slots, the same bits in every block.
__device__ __forceinline__ float clip_group_norm(const ClipParams& P, int g, double* scratch) {
  double v = 0.0;
  const int first = P.slots[2 * g], n = P.slots[2 * g + 1];
  for (int i = threadIdx.x; i < n; i += kClipWorkers) v += P.partial[first + i];
  return (float)sqrt(workers_sum(v, scratch));
}
__device__ __forceinline__ void clip_write_norms(const ClipParams& P, double* scratch) {
  for (int g = blockIdx.x; g < P.groups; g += gridDim.x) {
    const float norm = clip_group_norm(P, g, scratch);
    if (threadIdx.x == 0) P.norms[g] = norm;
  }
}

__global__ void __launch_bounds__(kClipWorkers) clip_finish_kernel(const ClipParams P) {
  __shared__ double scratch[kClipWorkers / 32];
  grid_dependency_wait();
  clip_write_norms(P, scratch);
}

__device__ __forceinline__ float clip_scaled(float v, float factor, bool zero) { return zero ? 0.0f : __fmul_rn(v, factor); }
__device__ __forceinline__ void clip_put(const ClipEntry& t, long long at, float v) {
  if (t.out_dtype == GBMUF_F32) __stcs(static_cast<float*>(t.out) + at, v);
  else static_cast<__nv_bfloat16*>(t.out)[at] = __float2bfloat16_rn(v);
}

// The norms from the partial sums, and the clipped copies.  A block goes through the chunks it read
// for the norm from the last to the first: the last ones are still in the L2 cache.  Four elements
// per thread and store (16 bytes of fp32: whole 128-byte lines per warp).
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm) clip_scale_kernel(const ClipParams P) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ double scratch[kClipWorkers / 32];
  const uint32_t bars = smem_u32(smem);
  clip_prologue(smem);
  if (threadIdx.x >= kClipWorkers) { grid_dependency_wait(); clip_produce<false>(P, bars, bars + 128); return; }
  grid_dependency_wait();
  clip_write_norms(P, scratch);
  ClipWalk<false> w;
  if (!w.begin(P)) return;                       // a handle without elements
  int group = -1, n = 0;
  float factor = 1.0f;
  bool zero = false, ok = true;
  do {
    if (w.t.group != group) {
      group = w.t.group;
      const float norm = clip_group_norm(P, group, scratch);
      zero = !(norm <= 3.402823466e38f);
      factor = P.max_norm > 0.0f && norm > P.max_norm ? __fdiv_rn(P.max_norm, norm) : 1.0f;
    }
    if (!w.t.out) continue;
    const ClipSpan s = clip_span(w.t, w.c - w.t.chunk0);
    if (s.a1 > s.a0) {
      const int slot = n % kClipRing;
      ok = ok && mbar_wait_bounded(bars + 8 * slot, (n / kClipRing) & 1, P.status);
      const unsigned char* const in = smem + 128 + slot * kClipSlot;
      const int elems = (int)(s.a1 - s.a0);
      const bool wide = (uintptr_t)(static_cast<char*>(w.t.out) + s.a0 * (w.t.out_dtype == GBMUF_F32 ? 4 : 2)) %
                            (w.t.out_dtype == GBMUF_F32 ? 16 : 8) == 0;
      auto each = [&](auto load4, auto load1) {
        if (wide) {
#pragma unroll 8
          for (int k = 4 * threadIdx.x; k < elems; k += 4 * kClipWorkers) {
            float v[4];
            load4(k, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = clip_scaled(v[j], factor, zero);
            if (w.t.out_dtype == GBMUF_F32) ThetaTraits<float>::stg_quad(static_cast<float*>(w.t.out) + s.a0 + k, v);
            else ThetaTraits<__nv_bfloat16>::stg_quad(static_cast<__nv_bfloat16*>(w.t.out) + s.a0 + k, v);
          }
        } else {
#pragma unroll 4
          for (int k = threadIdx.x; k < elems; k += kClipWorkers) clip_put(w.t, s.a0 + k, clip_scaled(load1(k), factor, zero));
        }
      };
      if (ok) {
        if (w.t.dtype == GBMUF_F32) {
          const float* const x = reinterpret_cast<const float*>(in);
          each([&](int k, float (&v)[4]) { ThetaTraits<float>::lds_quad(x + k, v); }, [&](int k) { return x[k]; });
        } else {
          const __nv_bfloat16* const x = reinterpret_cast<const __nv_bfloat16*>(in);
          each([&](int k, float (&v)[4]) { ThetaTraits<__nv_bfloat16>::lds_quad(x + k, v); }, [&](int k) { return to_f32(x[k]); });
        }
      }
      __syncwarp();                              // one arrival per warp: they are serialised
      if ((threadIdx.x & 31) == 0) mbar_arrive(bars + 64 + 8 * slot);
      ++n;
    }
    const long long rest = (s.e1 - s.e0) - (s.a1 - s.a0);
#pragma unroll 4
    for (long long k = threadIdx.x; k < rest; k += kClipWorkers) {
      const long long e = clip_outside(s, k);
      clip_put(w.t, clip_at(w.t, e, w.t.ld_out), clip_scaled(clip_single(w.t, e), factor, zero));
    }
  } while (w.next(P));
}

// A wait for a barrier that nothing signals: it expires, sets the status word and returns.
__global__ void clip_expired_wait_kernel(int32_t* status) {
  __shared__ __align__(8) unsigned long long barrier;
  const uint32_t bar = smem_u32(&barrier);
  if (threadIdx.x == 0) {
    mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  mbar_wait_bounded(bar, 0, status);
}

}  // namespace

#endif  // GBMUF_CSRC_GRAD_CLIP_CUH
