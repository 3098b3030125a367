// A row of logits in shared memory, by 16-byte pieces: what the kernels for long rows share.
// Part of libgbmuf (CUDA, sm_100a); included by the local-step operators' translation units.
#ifndef GBMUF_CSRC_ROW_PIECES_CUH
#define GBMUF_CSRC_ROW_PIECES_CUH

namespace {

constexpr int kLossWorkers = 256;
constexpr int kLossWarps = kLossWorkers / 32;
constexpr int kLossThreads = kLossWorkers + 32;
constexpr int kLossPieces = 4;                              // per thread and chunk
constexpr int kLossChunk = 16 * kLossPieces * kLossWorkers; // 16 KB
constexpr int kLossRing = 6;
constexpr int kLossKept = 5;
constexpr int kLossBlocksPerSm = 2;
constexpr uint32_t kLossHead = 512;
constexpr uint32_t kLossSmem = kLossHead + kLossRing * kLossChunk;

// The part of a row that a CTA of its cluster goes through.
struct RowSpan {
  int a0;                    // elements before the first whole piece
  int pieces;                // whole pieces of the row
  int p0, n;                 // this CTA's pieces
};
template <typename T, typename Params> __device__ __forceinline__ RowSpan row_span(const Params& P, long long row, int rank) {
  constexpr int E = 16 / (int)sizeof(T);
  RowSpan r;
  const int past = (int)((uintptr_t)(static_cast<const T*>(P.logits) + row * P.ld) % 16 / sizeof(T));
  r.a0 = past ? E - past : 0;                              // vocab > E
  r.pieces = ((int)P.vocab - r.a0) / E;
  r.p0 = (int)((unsigned)r.pieces * (unsigned)rank / (unsigned)P.split);       // pieces * 8 < 2^32
  r.n = (int)((unsigned)r.pieces * (unsigned)(rank + 1) / (unsigned)P.split) - r.p0;
  return r;
}
__device__ __forceinline__ void loss_workers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kLossWorkers) : "memory"); }
// Maximum of a piece's values (NaN does not count) and its values.
__device__ __forceinline__ float piece_max(uint4 u, const float (&)[4]) {
  return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
}
__device__ __forceinline__ float piece_max(uint4 u, const float (&)[8]) {
  auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
  const __nv_bfloat162 m = __hmax2(__hmax2(h(u.x), h(u.y)), __hmax2(h(u.z), h(u.w)));
  return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ void piece_values(uint4 u, float (&v)[4]) {
  v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void piece_values(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}

}  // namespace

#endif  // GBMUF_CSRC_ROW_PIECES_CUH
