// Matrix products of the linear layer on the tensor cores.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_LINEAR_TC_CUH
#define GBMUF_CSRC_LINEAR_TC_CUH

namespace {

// Result[r][c] = sum_k A(c, k) B(r, k), bf16 operands, fp32 sums.  Columns c of the result (they lie
// next to one another in memory) run along the 128 lanes of tensor memory, rows r along its columns:
//   forward       A = w, B = x,  k = n_in   (both with k contiguous)
//   input grad    A = w, B = dz, k = n_out  (A with c contiguous)
//   weight grad   A = x, B = dz, k = rows   (A with c contiguous, B with r contiguous)
// so a warp that holds 32 lanes of one accumulator column stores 32 neighbouring elements, and few
// rows (single tokens) make the tile narrow (BN), not half empty.
//
// fp32 operands come as three bf16 parts (hi, mid, lo: together all 24 bits; PARTS 3), and each step
// along k does six of the nine products of parts; mid lo, lo mid and lo lo, left out, come to at most
// 2^-23 of a product.
//
// A tile is 128 x BN, or 256 x BN for a pair of CTAs whose tensor cores work as one (PAIR 2): each
// holds half of the accumulator and loads half of B, a third less to fetch from L2 per product at
// BN = 256, which is what bounds a single CTA.  Warp 0 loads 64 k of both operands per step with the copy engine (128-byte
// swizzle), warp 1 issues the matrix instructions, the warps from 4 on finish the sums.  Two accumulators:
// one is finished while the next is summed.
//
// Measured: 2,048 x 1,024 x 100,000 bf16 292 to 307 us in short runs (up to 1,437 TFLOP/s, 89 % of a library
// product's rate; tensor pipe 92 % active; single CTAs 327 us), 358 to 370 back to back under the power cap
// (up to 1,170 TFLOP/s); 8,192 x 1,024 x 4,096 to fp32 58 us in short runs (1,185 TFLOP/s; its 128 tiles
// leave 20 of 148 SMs idle, on the others the tensor pipe is 74 % active, L2 47 % busy); 4,096 x 512 x 2,048 with
// gelu 17.4 to 18.7 us, of which the two epilogues of a CTA are 10: 16 finishing warps hide their own
// latencies better than 8 (24 us then), 32-row strips spill (20 us).
constexpr int kTcFinishers = 16;               // warps
constexpr int kTcThreads = 128 + 32 * kTcFinishers;
constexpr int kTcK = 64;                       // k per step
constexpr int kTcMaxStages = 12;

struct TcParams {
  Epilogue E;
  int32_t* status;
  int R, C;
  int ksteps;            // steps of 64 along k
  int tiles_r, tiles;    // row tiles; all tiles, row tiles running fastest
  int tile_step, step_c, step_r;   // from a CTA's tile to its next: tiles, and as column and row tiles
  int split;             // CTAs of a cluster that share a tile's steps (1: none)
  int stages;
};

// PAIR CTAs of a cluster work on one tile of PAIR * 128 x BN: each loads 128 of A's rows and BN / PAIR
// of B's.  A stage of the ring holds 64 k of one part of both.
__host__ __device__ constexpr uint32_t tc_stage_bytes(int bn, int pair) { return (128u + (uint32_t)(bn / pair)) * 128u; }
constexpr uint32_t kTcHead = 1024;             // barriers and the tensor-memory address
__host__ __device__ constexpr uint32_t tc_smem_bytes(int bn, int pair, int stages) {
  return 1024u + kTcHead + (uint32_t)stages * tc_stage_bytes(bn, pair);
}

// PAIR 2: the barrier may be the other CTA's.
template <int PAIR>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  if (PAIR == 1)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
        "[%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], "
        "[%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

// Shared-memory operand descriptor, 128-byte swizzle.  k contiguous: rows of 128 bytes (64 k), groups
// of 8 rows 1024 bytes apart.  k strided: blocks of 64 elements x 64 k, rows of 128 bytes along the
// operand's own dimension, 8 k 1024 bytes apart, the next 64 elements 8192 bytes on.  The upper word is
// a constant, the lower one the address / 16 (14 bits) and the block stride.
constexpr uint32_t kDescUpper = (1024u >> 4) | (1u << 14) | (2u << 29);
template <bool K_CONTIGUOUS> __device__ __forceinline__ uint32_t desc_lower(uint32_t addr) {
  return ((addr >> 4) & 0x3fffu) | ((K_CONTIGUOUS ? 1u : 8192u >> 4) << 16);
}
template <bool K_CONTIGUOUS> constexpr uint32_t kDescStep = (K_CONTIGUOUS ? 32u : 2048u) >> 4;     // 16 k
// Instruction descriptor: fp32 accumulator, bf16 operands, PAIR * 128 x BN.
template <bool A_K, bool B_K>
__device__ __forceinline__ constexpr uint32_t instr_desc(int bn, int pair) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (A_K ? 0u : 1u << 15) | (B_K ? 0u : 1u << 16) |
         ((uint32_t)(bn >> 3) << 17) | ((uint32_t)(pair * 128 >> 4) << 24);
}
template <int PAIR>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t keep) {
#define MMA(GROUP)                                                                                       \
  asm volatile(                                                                                          \
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"                                                    \
      "setp.ne.u32 p, %4, 0;\n\t"                                                                        \
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"                                              \
      "tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),                   \
      "r"(a), "r"(b), "r"(idesc), "r"(keep), "r"(kDescUpper)                                             \
      : "memory")
  if (PAIR == 1) MMA("1"); else MMA("2");
#undef MMA
}
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// Arrives on a barrier once the matrix instructions issued so far are done; PAIR 2: in both CTAs.
template <int PAIR> __device__ __forceinline__ void mma_commit(uint32_t bar) {
  if (PAIR == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}
// The address of rank 0's copy of a shared-memory location.
__device__ __forceinline__ uint32_t in_leader(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void arrive_remote(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ void st_remote(uint32_t addr, uint32_t rank, float v) {
  asm volatile("{\n\t.reg .b32 r;\n\tmapa.shared::cluster.u32 r, %0, %1;\n\tst.shared::cluster.f32 [r], %2;\n\t}" ::"r"(addr),
               "r"(rank), "f"(v)
               : "memory");
}
// N accumulator columns of this warp's 32 lanes.
template <int N> __device__ __forceinline__ void tmem_ld(uint32_t addr, float (&v)[N]) {
  static_assert(N == 8 || N == 16, "");
  uint32_t u[N];
  if constexpr (N == 16)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
          "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(addr));
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
                 : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    asm volatile("" : "+r"(u[i]));                                 // no use of the values moves before the wait
    v[i] = __uint_as_float(u[i]);
  }
}

// PROMOTE (results that stay fp32): the tensor cores' sum is moved into fp32 registers, and added there
// with rounding to nearest, after every 16 (24) instructions: in the accumulator every addition cuts
// towards zero, which over thousands of them would cost a few units of 2^-18.  Results that are rounded
// to bf16 stay in the accumulator: k / 16 cuts of at most 2^-23 of a sum that grows like a random walk are
// (2/3) k / 16 x 2^-23 of the result, 1.3e-3 at k = 267,735, about what the rounding to bf16 costs.
template <int KIND, typename T, typename TO, int PARTS, int BN, int PAIR>
__global__ void __launch_bounds__(kTcThreads, 1)
    linear_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const TcParams P) {
  constexpr bool A_K = KIND == kForward, B_K = KIND != kWeightGrad, PROMOTE = sizeof(TO) == 4;
  constexpr int TILE_C = 128 * PAIR, OWN_R = BN / PAIR;           // a tile's columns; rows of B that this CTA loads
  constexpr uint32_t STAGE = tc_stage_bytes(BN, PAIR), A_BYTES = 128 * 128;
  constexpr int ACC = BN;                      // tensor-memory columns of one accumulator
  constexpr int NCOL = BN / (kTcFinishers / 4);   // accumulator columns per finishing warp
  constexpr int N = NCOL < 16 ? NCOL : 16;        // of them at a time
  extern __shared__ __align__(128) unsigned char raw[];
  unsigned char* const smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const uint32_t bars = smem_u32(smem), ring = bars + kTcHead;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 128u + 8u * s; };
  auto acc_full = [&](int b) { return bars + 256u + 8u * b; };
  auto acc_empty = [&](int b) { return bars + 272u + 8u * b; };
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + 320);
  const int warp = __shfl_sync(~0u, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int S = P.stages;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), PAIR * kTcFinishers); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // Before the wait for the kernel before: a block of it that has yet to allocate (the fused round lets
  // its dependents start first thing) cannot be on this SM, whose registers or shared memory do not hold both.
  if (warp == 1) {
    if (PAIR == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2u * ACC) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2u * ACC) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (PAIR == 2) cluster_sync();                                   // both CTAs' barriers exist
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0);
  grid_launch_dependents();
  grid_dependency_wait();

  // this CTA's tiles and its share of each one's steps
  const int rank = P.split > 1 ? (int)(blockIdx.x % (unsigned)P.split) : 0;      // among the CTAs that share the steps
  const int side = PAIR == 2 ? (int)(blockIdx.x & 1) : 0;                        // of the pair that shares the tile
  const int step0 = P.split > 1 ? (int)((unsigned)P.ksteps * (unsigned)rank / (unsigned)P.split) : 0;
  const int step1 = P.split > 1 ? (int)((unsigned)P.ksteps * (unsigned)(rank + 1) / (unsigned)P.split) : P.ksteps;
  const int iters = step1 - step0;
  // without PROMOTE a tile is one chunk
  const int chunk = PROMOTE ? (PARTS == 1 ? 4 : 1) : (iters > 0 ? iters : 1);
  const int chunks = iters == 0 ? 0 : (iters + chunk - 1) / chunk;
  const int first_tile = P.split > 1 ? (int)(blockIdx.x / (unsigned)P.split) : (int)(blockIdx.x / PAIR);
  struct Walk {                                                    // tile number, column tile, row tile
    int tile, c, r;
  };
  auto first = [&] { return Walk{first_tile, first_tile / P.tiles_r, first_tile % P.tiles_r}; };
  auto next = [&](Walk& w) {
    w.tile += P.tile_step;
    w.c += P.step_c;
    w.r += P.step_r;
    if (w.r >= P.tiles_r) { w.r -= P.tiles_r; ++w.c; }
  };

  if (warp == 0) {
    // -------------------------------------------------------------------- loads
    // The whole warp goes through the loops of this and the next role, so that addresses, coordinates
    // and descriptors stay in uniform registers; an elected lane waits and issues.  Where a wait gives
    // up, the rest of the loop does nothing.
    constexpr int BOXES_A = A_K ? 1 : 2, BOXES_B = B_K ? 1 : OWN_R / 64;
    int s = 0, issued = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (Walk w = first(); w.tile < P.tiles; next(w)) {
      const int c0 = w.c * TILE_C + side * 128, r0 = w.r * BN + side * OWN_R;
      for (int it = 0; it < iters; ++it) {
        const int k0 = (step0 + it) * kTcK;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {                          // parts in the order of their use: hi, lo, mid
          const int part = q == 0 ? 0 : 3 - q;
          // the leader's barrier counts both CTAs' bytes
          const uint32_t bar = PAIR == 2 ? in_leader(full(s)) : full(s), a = ring + s * STAGE, b = a + A_BYTES;
          if (elect_one()) {
            if (issued >= S) ok = ok && wait_phase(empty(s), ph ^ 1, P.status);
            if (ok) {
              if (side == 0) mbar_arrive_expect_tx(full(s), PAIR * STAGE);
#pragma unroll
              for (int i = 0; i < BOXES_A; ++i)
                tma_load_3d<PAIR>(a + i * 8192, &map_a, A_K ? k0 : c0 + 64 * i, A_K ? c0 : k0, part, bar);
#pragma unroll
              for (int i = 0; i < BOXES_B; ++i)
                tma_load_3d<PAIR>(b + i * 8192, &map_b, B_K ? k0 : r0 + 64 * i, B_K ? r0 : k0, part, bar);
            }
          }
          ++issued;
          if (++s == S) { s = 0; ph ^= 1; }
        }
      }
    }
    // the copies requested so far land before the CTAs end; the leader's barriers count both CTAs'
    if (!ok && side == 0)
      for (int j = 0; j < S; ++j) { mbar_wait_bounded(full(j), 0, P.status); mbar_wait_bounded(full(j), 1, P.status); }
    __syncwarp();
  } else if (warp == 1 && side == 0) {
    // -------------------------------------------------------------------- matrix instructions
    int s = 0, n = 0;                                              // n: chunks started
    uint32_t ph = 0;
    bool ok = true;
    const uint32_t a0 = desc_lower<A_K>(ring), b0 = desc_lower<B_K>(ring + A_BYTES);
    // 64 k of A in one stage against B in another
    auto multiply = [&](uint32_t d, int sa, int sb, uint32_t keep) {
      const uint32_t a = a0 + sa * (STAGE >> 4), b = b0 + sb * (STAGE >> 4);
#pragma unroll
      for (int k = 0; k < kTcK / 16; ++k)
        mma_bf16<PAIR>(d, a + k * kDescStep<A_K>, b + k * kDescStep<B_K>, instr_desc<A_K, B_K>(BN, PAIR), k > 0 ? 1u : keep);
    };
    for (int tile = first_tile; tile < P.tiles; tile += P.tile_step) {
      int in_chunk = 0;
      for (int it = 0; it < iters; ++it) {
        const uint32_t d = tmem + (uint32_t)(n & 1) * ACC;
        const bool last = in_chunk + 1 == chunk || it == iters - 1;
        // with three parts: hi in stage s, lo in s1, mid in s2
        int s1 = s + 1, s2 = s + 2;
        uint32_t ph1 = ph, ph2 = ph;
        if (PARTS == 3) {
          if (s1 >= S) { s1 -= S; ph1 ^= 1; }
          if (s2 >= S) { s2 -= S; ph2 ^= 1; }
        }
        if (elect_one()) {
          if (in_chunk == 0) {
            if (n >= 2) ok = ok && wait_phase(acc_empty(n & 1), ((n >> 1) & 1) ^ 1, P.status);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          }
          ok = ok && wait_phase(full(s), ph, P.status);
          if constexpr (PARTS == 1) {
            if (ok) multiply(d, s, s, (uint32_t)in_chunk);
          } else {
            // smallest products first: an accumulator that is still small loses less to each addition
            ok = ok && wait_phase(full(s1), ph1, P.status);
            if (ok) {
              multiply(d, s, s1, (uint32_t)in_chunk);
              multiply(d, s1, s, 1);
              mma_commit<PAIR>(empty(s1));
            }
            ok = ok && wait_phase(full(s2), ph2, P.status);
            if (ok) {
              multiply(d, s2, s2, 1);
              multiply(d, s, s2, 1);
              multiply(d, s2, s, 1);
              mma_commit<PAIR>(empty(s2));
              multiply(d, s, s, 1);
            }
          }
          if (ok) {
            mma_commit<PAIR>(empty(s));
            if (last) mma_commit<PAIR>(acc_full(n & 1));
          }
        }
        ++in_chunk;
        if (last) { ++n; in_chunk = 0; }
        s += PARTS;
        if (s >= S) { s -= S; ph ^= 1; }
      }
    }
    __syncwarp();
  }

  // ---------------------------------------------------------------------- finishing warps
  const int quad = warp & 3, part = (warp - 4) >> 2;
  const uint32_t my_tmem = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(part * NCOL);
  auto release = [&](int b) {                                      // one arrival per warp, at the leader's barrier
    if (lane == 0) {
      if (PAIR == 2) arrive_remote(in_leader(acc_empty(b)));
      else mbar_arrive(acc_empty(b));
    }
  };
  // Asked for before the wait for the sums and converted after it: a conversion here would wait for it.
  auto bias_of = [&](int c) { return KIND == kForward && P.E.bias && c < P.C ? static_cast<const T*>(P.E.bias)[c] : from_f32<T>(0.0f); };
  if (warp >= 4 && P.split == 1) {
    int n = 0;
    bool ok = true;
    for (Walk w = first(); w.tile < P.tiles && ok; next(w)) {
      const int c = w.c * TILE_C + side * 128 + quad * 32 + lane, r0 = w.r * BN + part * NCOL;
      const T bias = bias_of(c);
      if (PROMOTE) {
        float acc[NCOL];
#pragma unroll
        for (int i = 0; i < NCOL; ++i) acc[i] = 0.0f;
        for (int ch = 0; ch < chunks; ++ch, ++n) {
          ok = mbar_wait_bounded(acc_full(n & 1), (n >> 1) & 1, P.status);
          ok = __all_sync(~0u, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int j = 0; j < NCOL; j += N) {
            float v[N];
            tmem_ld<N>(my_tmem + (uint32_t)(n & 1) * ACC + j, v);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[j + i] += v[i];
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          release(n & 1);
        }
        if (!ok) break;
#pragma unroll
        for (int j = 0; j < NCOL; j += N) {
          Finisher<KIND, T, TO, N> F;
          float v[N];
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] = acc[j + i];
          F.ask(P.E, r0 + j, c, P.R, P.C, lane);
          F.finish(P.E, r0 + j, c, P.R, P.C, lane, to_f32(bias), v);
        }
      } else {
        // what the epilogue reads is requested one strip ahead, the first one during the sums
        Finisher<KIND, T, TO, N> F;
        F.ask(P.E, r0, c, P.R, P.C, lane);
        if (chunks > 0) {
          ok = mbar_wait_bounded(acc_full(n & 1), (n >> 1) & 1, P.status);
          ok = __all_sync(~0u, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        }
#pragma unroll 1
        for (int j = 0; j < NCOL; j += N) {
          float v[N] = {};
          if (chunks > 0) tmem_ld<N>(my_tmem + (uint32_t)(n & 1) * ACC + j, v);
          Finisher<KIND, T, TO, N> now = F;
          if (j + N < NCOL) F.ask(P.E, r0 + j + N, c, P.R, P.C, lane);
          now.finish(P.E, r0 + j, c, P.R, P.C, lane, to_f32(bias), v);
        }
        if (chunks > 0) {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          release(n & 1);
          ++n;
        }
      }
    }
  }
  if (PAIR == 1 && P.split > 1) {
    // The cluster's CTAs hold partial sums of one tile.  CTA j finishes accumulator columns
    // [j, j + 1) BN / split: everybody writes its sums of those columns into CTA j's shared memory
    // (the operand ring, idle by then) and CTA j adds them in the order of the ranks.
    const int cols = BN / P.split;
    float acc[PROMOTE ? NCOL : 1];
    if (warp >= 4) {
      bool ok = true;
      if (PROMOTE)
#pragma unroll
        for (int i = 0; i < NCOL; ++i) acc[i] = 0.0f;
      for (int n = 0; n < chunks && ok; ++n) {
        ok = mbar_wait_bounded(acc_full(n & 1), (n >> 1) & 1, P.status);
        ok = __all_sync(~0u, ok);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (PROMOTE && ok) {
#pragma unroll
          for (int j = 0; j < NCOL; j += N) {
            float v[N];
            tmem_ld<N>(my_tmem + (uint32_t)(n & 1) * ACC + j, v);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[j + i] += v[i];
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          release(n & 1);
        }
      }
    }
    cluster_sync();                                                // every ring is idle
    if (warp >= 4) {
      const uint32_t mine = ring + 4u * (uint32_t)(rank * cols * 128 + quad * 32 + lane);
#pragma unroll
      for (int j = 0; j < NCOL; j += N) {
        float v[N];
        if (!PROMOTE) tmem_ld<N>(my_tmem + j, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int col = part * NCOL + j + i, owner = col / cols;
          st_remote(mine + 512u * (uint32_t)(col - owner * cols), (uint32_t)owner, PROMOTE ? acc[PROMOTE ? j + i : 0] : v[i]);
        }
      }
    }
    cluster_sync();                                                // everybody's sums have arrived
    if (warp >= 4) {
      // strips of 4 rows (BN / split is a multiple of 4)
      const float* const sums = reinterpret_cast<const float*>(smem + kTcHead) + quad * 32 + lane;
      const Walk w = first();
      const int c = w.c * 128 + quad * 32 + lane;
      const T bias = bias_of(c);
      for (int i = 4 * part; i < cols; i += kTcFinishers) {
        const int r = w.r * BN + rank * cols + i;
        Finisher<KIND, T, TO, 4> F;
        F.ask(P.E, r, c, P.R, P.C, lane);
        float v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          v[x] = sums[(i + x) * 128];
          for (int q = 1; q < P.split; ++q) v[x] += sums[(q * cols + i + x) * 128];
        }
        F.finish(P.E, r, c, P.R, P.C, lane, to_f32(bias), v);
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (PAIR == 2) cluster_sync();                                   // nothing of this CTA is used any more
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (PAIR == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2u * ACC) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2u * ACC) : "memory");
  }
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_TC_CUH
