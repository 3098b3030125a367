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
  int tiles_fast, tiles; // row tiles (kLossStats: column tiles), which run fastest; all tiles
  int tile_step, step_slow, step_fast;   // from a CTA's tile to its next: tiles, and as tiles of either kind
  int split;             // CTAs of a cluster that share a tile's steps (1: none)
  int tiles_c;           // kLossTerm: column tiles; the tiles of a slice of the steps follow those of the one before
  int slices;
  int stages;
};

// PAIR CTAs of a cluster work on one tile of PAIR * 128 x BN: each loads 128 of A's rows and BN / PAIR
// of B's.  A stage of the ring holds 64 k of one part of both.
__host__ __device__ constexpr uint32_t tc_stage_bytes(int bn, int pair) { return (128u + (uint32_t)(bn / pair)) * 128u; }
constexpr uint32_t kTcHead = 1024;             // barriers and the tensor-memory address
// Behind the ring: where the finishing warps lay results out for the copy engine (linear_loss.cuh), 4 or 2 KB each.
// (Tiles too narrow for strips of 32 rows store by themselves.)
template <int KIND, int PARTS, int BN> constexpr uint32_t kTcOut = KIND == kLossGrad && BN >= 128 ? (PARTS == 1 ? 4096u : 2048u) * kTcFinishers : 0u;
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
// N accumulator columns of this warp's 32 lanes.
template <int N> __device__ __forceinline__ void tmem_ld(uint32_t addr, float (&v)[N]) {
  static_assert(N == 8 || N == 16 || N == 32, "");
  uint32_t u[N];
  if constexpr (N == 32)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
          "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]),
          "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]),
          "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
  else if constexpr (N == 16)
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
// towards zero, which over thousands of them would cost a few units of 2^-18.  (Terms of dx of bf16 operands, which are
// rounded to bf16 once they are added up: every 128, at most 1.5e-5 of the result.)  Results that are rounded
// to bf16 stay in the accumulator: k / 16 cuts of at most 2^-23 of a sum that grows like a random walk are
// (2/3) k / 16 x 2^-23 of the result, 1.3e-3 at k = 267,735, about what the rounding to bf16 costs.
template <int KIND, typename T, typename TO, int PARTS, int BN, int PAIR>
__global__ void __launch_bounds__(kTcThreads, 1)
    linear_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
                     const TcParams P) {
  constexpr bool A_K = KIND == kForward || KIND == kLossStats || KIND == kLossGrad, B_K = KIND != kWeightGrad && KIND != kLossTerm;
  constexpr bool PROMOTE = sizeof(TO) == 4;
  constexpr int TILE_C = 128 * PAIR, OWN_R = BN / PAIR;           // a tile's columns; rows of B that this CTA loads
  constexpr uint32_t STAGE = tc_stage_bytes(BN, PAIR), A_BYTES = 128 * 128;
  constexpr int ACC = BN;                      // tensor-memory columns of one accumulator
  // Accumulators in turn.  Where sums leave them as they go, the finishing warps' work at a tile's end (exponentials and
  // stores of the loss) holds the chunks up: narrow tiles have room for four.
  constexpr int NACC = PROMOTE && KIND >= kLossStats && BN <= 128 ? 4 : 2, LOG_ACC = NACC / 2;
  constexpr int NCOL = BN / (kTcFinishers / 4);   // accumulator columns per finishing warp
  constexpr int MOST = (KIND == kLossStats && !PROMOTE) || KIND == kLossGrad ? 32 : 16;
  constexpr int N = NCOL < MOST ? NCOL : MOST;    // of them at a time
  // fp32 weight gradients are stored 8 rows at a time: with 16, registers ran out in the loop of the sums (8,192 x 1,024 x
  // 4,096: 60.4 -> 58.6 us)
  constexpr int LAST = PROMOTE && (KIND == kWeightGrad || KIND == kLossWeight) && N > 8 ? 8 : N;
  extern __shared__ __align__(128) unsigned char raw[];
  unsigned char* const smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const uint32_t bars = smem_u32(smem), ring = bars + kTcHead;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 128u + 8u * s; };
  auto acc_full = [&](int b) { return bars + 256u + 8u * b; };
  auto acc_empty = [&](int b) { return bars + 288u + 8u * b; };
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + 320);
  const int warp = __shfl_sync(~0u, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int S = P.stages;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < NACC; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), PAIR * kTcFinishers); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // Before the wait for the kernel before: a block of it that has yet to allocate (the fused round lets
  // its dependents start first thing) cannot be on this SM, whose registers or shared memory do not hold both.
  if (warp == 1) {
    if (PAIR == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)NACC * ACC) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)NACC * ACC) : "memory");
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
  // what of a tile there is to do: its column tile, its steps, and these in chunks (without PROMOTE a tile is one)
  struct Share {
    int c, slice, step0, iters, chunks;
  };
  constexpr int chunk = !PROMOTE ? 0x7fffffff : PARTS == 3 ? 1 : KIND == kLossTerm ? 32 : 4;
  auto chunks_of = [](int iters) { return PROMOTE ? (iters + chunk - 1) / chunk : iters > 0 ? 1 : 0; };
  const Share whole{0, 0, step0, step1 - step0, chunks_of(step1 - step0)};
  auto share = [&](int c) {
    Share s = whole;
    s.c = c;
    if (KIND == kLossTerm) {
      s.slice = c / P.tiles_c;
      s.c = c - s.slice * P.tiles_c;
      s.step0 = (int)((long long)P.ksteps * s.slice / P.slices);
      s.iters = (int)((long long)P.ksteps * (s.slice + 1) / P.slices) - s.step0;
      s.chunks = chunks_of(s.iters);
    }
    return s;
  };
  const int first_tile = P.split > 1 ? (int)(blockIdx.x / (unsigned)P.split) : (int)(blockIdx.x / PAIR);
  struct Walk {                                                    // tile number, column tile, row tile
    int tile, c, r;
    __device__ __forceinline__ int& fast() { return KIND == kLossStats ? c : r; }
    __device__ __forceinline__ int& slow() { return KIND == kLossStats ? r : c; }
  };
  auto first = [&] {
    Walk w;
    w.tile = first_tile;
    w.slow() = first_tile / P.tiles_fast;
    w.fast() = first_tile % P.tiles_fast;
    return w;
  };
  auto next = [&](Walk& w) {
    w.tile += P.tile_step;
    w.slow() += P.step_slow;
    w.fast() += P.step_fast;
    if (w.fast() >= P.tiles_fast) { w.fast() -= P.tiles_fast; ++w.slow(); }
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
      const Share mine = share(w.c);
      const int c0 = mine.c * TILE_C + side * 128, r0 = w.r * BN + side * OWN_R;
      for (int it = 0; it < mine.iters; ++it) {
        const int k0 = (mine.step0 + it) * kTcK;
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
      const int iters = KIND == kLossTerm ? share(tile / P.tiles_fast).iters : whole.iters;
      for (int it = 0; it < iters; ++it) {
        const uint32_t d = tmem + (uint32_t)(n & (NACC - 1)) * ACC;
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
            if (n >= NACC) ok = ok && wait_phase(acc_empty(n & (NACC - 1)), ((n >> LOG_ACC) & 1) ^ 1, P.status);
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
            if (last) mma_commit<PAIR>(acc_full(n & (NACC - 1)));
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
  auto bias_of = [&](int c) { return (KIND == kForward || KIND == kLossGrad) && P.E.bias && c < (KIND == kLossGrad ? P.E.words : P.C) ? static_cast<const T*>(P.E.bias)[c] : from_f32<T>(0.0f); };
  if constexpr (KIND == kLossStats) {
    if (warp >= 4) {
      int n = 0;
      bool ok = true;
      RowStats<T> S;
      const int chunks = whole.chunks;
      for (Walk w = first(); w.tile < P.tiles && ok; next(w)) {
        S.open(P.E, w.c * TILE_C + side * 128 + quad * 32 + lane, P.C, w.r * (kTcFinishers / 4) + part);
        const int r0 = w.r * BN + part * NCOL;
        if (PROMOTE) {
          float acc[NCOL];
#pragma unroll
          for (int i = 0; i < NCOL; ++i) acc[i] = 0.0f;
          for (int ch = 0; ch < chunks; ++ch, ++n) {
            ok = mbar_wait_bounded(acc_full(n & (NACC - 1)), (n >> LOG_ACC) & 1, P.status);
            ok = __all_sync(~0u, ok);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int j = 0; j < NCOL; j += N) {
              float v[N];
              tmem_ld<N>(my_tmem + (uint32_t)(n & (NACC - 1)) * ACC + j, v);
#pragma unroll
              for (int i = 0; i < N; ++i) acc[j + i] += v[i];
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            release(n & (NACC - 1));
          }
          if (!ok) break;
#pragma unroll
          for (int j = 0; j < NCOL; j += N) {
            float v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = acc[j + i];
            S.add(P.E, v, r0 + j, P.R);
          }
        } else {
          if (chunks > 0) {
            ok = mbar_wait_bounded(acc_full(n & (NACC - 1)), (n >> LOG_ACC) & 1, P.status);
            ok = __all_sync(~0u, ok);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          }
#pragma unroll 1
          for (int j = 0; j < NCOL; j += N) {
            float v[N] = {};
            if (chunks > 0) tmem_ld<N>(my_tmem + (uint32_t)(n & (NACC - 1)) * ACC + j, v);
            S.add(P.E, v, r0 + j, P.R);
          }
          if (chunks > 0) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            release(n & (NACC - 1));
            ++n;
          }
        }
      }
      S.close(P.E);
    }
  }
  if (KIND != kLossStats && warp >= 4 && P.split == 1) {
    int n = 0;
    bool ok = true;
    // two halves in turn: from one address to the other and back
    const uint32_t out_base = ring + (uint32_t)S * STAGE + kTcOut<KIND, PARTS, BN> / kTcFinishers * (uint32_t)(warp - 4);
    const uint32_t out_flip = PARTS == 1 ? out_base ^ (out_base + 2048u) : 0u;
    uint32_t out_room = out_base;
    const float factor = KIND == kLossWeight && PARTS == 1 && P.E.factor ? *P.E.factor : 1.0f;
    for (Walk w = first(); w.tile < P.tiles && ok; next(w)) {
      const Share mine = share(w.c);
      const int c = mine.c * TILE_C + side * 128 + quad * 32 + lane, r0 = w.r * BN + part * NCOL, chunks = mine.chunks;
      const T bias = bias_of(c);
      float column = 0.0f;                                         // kLossGrad: of the gradients of column c
      if (PROMOTE) {
        float acc[NCOL];
#pragma unroll
        for (int i = 0; i < NCOL; ++i) acc[i] = 0.0f;
        if constexpr (KIND == kLossTerm)
          if (P.E.accumulate) {
#pragma unroll
            for (int j = 0; j < NCOL; j += N) {
              Finisher<KIND, T, TO, N> F;
              F.slice = mine.slice;
              float v[N];
              F.begin(P.E, r0 + j, c, P.R, P.C, lane, v);
#pragma unroll
              for (int i = 0; i < N; ++i) acc[j + i] = v[i];
            }
          }
        for (int ch = 0; ch < chunks; ++ch, ++n) {
          ok = mbar_wait_bounded(acc_full(n & (NACC - 1)), (n >> LOG_ACC) & 1, P.status);
          ok = __all_sync(~0u, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int j = 0; j < NCOL; j += N) {
            float v[N];
            tmem_ld<N>(my_tmem + (uint32_t)(n & (NACC - 1)) * ACC + j, v);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[j + i] += v[i];
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          release(n & (NACC - 1));
        }
        if (!ok) break;
#pragma unroll
        for (int j = 0; j < NCOL; j += LAST) {
          Finisher<KIND, T, TO, LAST> F;
          if constexpr (KIND == kLossTerm) F.slice = mine.slice;
          if constexpr (KIND == kLossWeight) F.factor = factor;
          if constexpr (kTcOut<KIND, PARTS, BN> > 0) { F.map = &map_out; F.room = out_room; F.half = out_flip; }
          float v[LAST];
#pragma unroll
          for (int i = 0; i < LAST; ++i) v[i] = acc[j + i];
          F.ask(P.E, r0 + j, c, P.R, P.C, lane);
          F.finish(P.E, r0 + j, c, P.R, P.C, lane, to_f32(bias), v);
          if constexpr (KIND == kLossGrad) column += F.column;
          if constexpr (kTcOut<KIND, PARTS, BN> > 0) out_room = F.room;
        }
      } else {
        // what the epilogue reads is requested one strip ahead, the first one during the sums
        Finisher<KIND, T, TO, N> F;
        if constexpr (KIND == kLossWeight) F.factor = factor;
        if constexpr (kTcOut<KIND, PARTS, BN> > 0) { F.map = &map_out; F.room = out_room; F.half = out_flip; }
        F.ask(P.E, r0, c, P.R, P.C, lane);
        if (chunks > 0) {
          ok = mbar_wait_bounded(acc_full(n & (NACC - 1)), (n >> LOG_ACC) & 1, P.status);
          ok = __all_sync(~0u, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        }
#pragma unroll 1
        for (int j = 0; j < NCOL; j += N) {
          float v[N] = {};
          if (chunks > 0) tmem_ld<N>(my_tmem + (uint32_t)(n & (NACC - 1)) * ACC + j, v);
          Finisher<KIND, T, TO, N> now = F;
          if (j + N < NCOL) F.ask(P.E, r0 + j + N, c, P.R, P.C, lane);
          now.finish(P.E, r0 + j, c, P.R, P.C, lane, to_f32(bias), v);
          if constexpr (KIND == kLossGrad) column += now.column;
          if constexpr (kTcOut<KIND, PARTS, BN> > 0) out_room = F.room = now.room;
        }
        if (chunks > 0) {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          release(n & (NACC - 1));
          ++n;
        }
      }
      if (KIND == kLossGrad && P.E.partial && c < P.E.words)
        static_cast<float*>(P.E.partial)[(w.r * (kTcFinishers / 4) + part) * P.E.ld_partial + c] = column;
    }
    if (kTcOut<KIND, PARTS, BN> > 0 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if constexpr (KIND < kLossStats && PAIR == 1) if (P.split > 1) {
    const int chunks = whole.chunks;
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
        ok = mbar_wait_bounded(acc_full(n & (NACC - 1)), (n >> LOG_ACC) & 1, P.status);
        ok = __all_sync(~0u, ok);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (PROMOTE && ok) {
#pragma unroll
          for (int j = 0; j < NCOL; j += N) {
            float v[N];
            tmem_ld<N>(my_tmem + (uint32_t)(n & (NACC - 1)) * ACC + j, v);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[j + i] += v[i];
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          release(n & (NACC - 1));
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
    if (PAIR == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)NACC * ACC) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)NACC * ACC) : "memory");
  }
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_TC_CUH
