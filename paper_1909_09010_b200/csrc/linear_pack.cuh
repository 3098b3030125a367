// Operands of the tensor-core products that cannot be read in place.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_LINEAR_PACK_CUH
#define GBMUF_CSRC_LINEAR_PACK_CUH

namespace {

// x as hi + mid + lo, each bf16: hi = RN(x), mid = RN(x - hi), lo = RN(x - hi - mid); the differences
// are exact, and three times 8 bits hold all 24 of x (down to the smallest bf16).  Two values at a time, the
// parts of both in a word.
__device__ __forceinline__ uint32_t pair_bf16(Two t) {
  float x, y;
  apart(t, x, y);
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ Two pair_f32(uint32_t u) { return two(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
__device__ __forceinline__ void split3(Two x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  hi = pair_bf16(x);
  x = x - pair_f32(hi);
  mid = pair_bf16(x);
  lo = pair_bf16(x - pair_f32(mid));
}
// The same for n elements among which there are magnitudes that round to a bf16 that is not finite.  The hi
// of a finite one is the largest bf16.  A NaN is in hi alone.  An infinity is in lo, with 1 of its sign in hi:
// lo meets hi of the other operand only, whose sign is the operand's and which is not 0 unless that is, so
// the sum of the six products is what the plain product gives (in hi it would meet mid and lo of the other
// operand as well, which can be 0 or of the other sign: NaN).  Not in line: the loop it is called from stays
// short (tests of every element in that loop cost 2.6 us of 9 at 5 M elements).
__device__ __noinline__ void split3_edges(const float* s, __nv_bfloat16* d, long long part, int n) {
  for (int j = 0; j < n; ++j) {
    const float x = s[j];
    const uint32_t bits = __float_as_uint(x), size = bits & 0x7fffffffu;
    const uint16_t sign = (uint16_t)(bits >> 16 & 0x8000u);
    uint16_t hi = __bfloat16_as_ushort(__float2bfloat16_rn(x)), mid = 0, lo = 0;
    if (size == 0x7f800000u) {
      lo = hi;
      hi = sign | 0x3f80u;
    } else if (size < 0x7f800000u) {
      if ((hi & 0x7f80u) == 0x7f80u) hi = sign | 0x7f7fu;
      const float r1 = x - __uint_as_float((uint32_t)hi << 16);
      mid = __bfloat16_as_ushort(__float2bfloat16_rn(r1));
      lo = __bfloat16_as_ushort(__float2bfloat16_rn(r1 - __uint_as_float((uint32_t)mid << 16)));
    }
    d[j] = __ushort_as_bfloat16(hi);
    d[part + j] = __ushort_as_bfloat16(mid);
    d[2 * part + j] = __ushort_as_bfloat16(lo);
  }
}

// src [outer][inner] with any stride and alignment -> bf16 parts [1 or 3][outer][ld_dst], ld_dst a
// multiple of 8; columns inner .. ld_dst-1 are never read as data and get zeros.  One thread per
// eight columns; vec: src rows are 16-byte aligned.
struct PackJob {
  const void* src;
  __nv_bfloat16* dst;
  long long ld, outer, inner, ld_dst;
  int vec, blocks;             // blocks: of the grid, 0: nothing to do
};
template <typename T, bool VEC> __device__ __forceinline__ void pack_run(const PackJob& J, int block) {
  const long long per_row = J.ld_dst / 8, n = J.outer * per_row, part = J.outer * J.ld_dst;
  for (long long i = (long long)block * 256 + threadIdx.x; i < n; i += (long long)J.blocks * 256) {
    const long long r = i / per_row, c = (i - r * per_row) * 8;
    const T* const s = static_cast<const T*>(J.src) + r * J.ld + c;
    __align__(16) T v[8];
    if (VEC && c + 8 <= J.inner) {
#pragma unroll
      for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(v)[j] = reinterpret_cast<const uint4*>(s)[j];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = c + j < J.inner ? s[j] : from_f32<T>(0.0f);
    }
    __nv_bfloat16* const d = J.dst + r * J.ld_dst + c;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(d) = *reinterpret_cast<const uint4*>(v);
    } else {
      __align__(16) uint32_t p[3][4];
      uint32_t edge = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        split3(two(v[2 * j], v[2 * j + 1]), p[0][j], p[1][j], p[2][j]);
        edge |= (p[0][j] & 0x7f807f80u) + 0x00800080u;     // an exponent of ones carries into the sign's place
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(d + q * part) = *reinterpret_cast<const uint4*>(p[q]);
      if (edge & 0x80008000u) split3_edges(s, d, part, J.inner - c < 8 ? (int)(J.inner - c) : 8);
    }
  }
}
// Both operands of a product in one launch.  Bound by memory: 21 MB of fp32 to 31 MB of parts in 10 us from cold caches.
template <typename T> __global__ void __launch_bounds__(256) pack_kernel(const PackJob a, const PackJob b) {
  grid_launch_dependents();
  grid_dependency_wait();
  const bool first = (int)blockIdx.x < a.blocks;
  const PackJob& J = first ? a : b;
  const int block = first ? blockIdx.x : blockIdx.x - a.blocks;
  if (J.vec) pack_run<T, true>(J, block); else pack_run<T, false>(J, block);
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_PACK_CUH
