// Cross-entropy of a softmax over a vocabulary, with its gradient.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_CROSS_ENTROPY_CUH
#define GBMUF_CSRC_CROSS_ENTROPY_CUH

namespace {

// Per row: m = max x, s = sum exp(x - m), then d = s_i (exp(x - m) / s - [target]).  Every logit is
// needed twice with the whole row between, so the row stays on the chip from its one read to its
// one write: in the registers of a warp (short rows), or in shared memory and the L2 cache.
// Measured: 2,048 x 267,735 bf16 417 to 458 us (4.8 to 5.3 TB/s of the bytes that have to move, 73 to 80 % of the
// copy rate; 69 % of the logits are fetched twice and 27 % of that misses L2; exponentials keep their unit 62 %
// busy); a row held by four CTAs' shared memory alone, one row at a time, 602:
// the exchange and the refill of the slots were exposed; one block per row that reads it twice 2,231.
// 512 x 10,000 fp32 12 us.  A cluster of eight per row leaves SMs idle (575 us).
struct LossParams {
  const void* logits;
  const int64_t* targets;
  const float* row_weight;
  float *loss, *lse;
  void* dlogits;
  long long rows, vocab, ld, ld_d;
  long long ignore_index;
  float scale;
  int32_t* status;
  int split;           // CTAs per row (ring kernel)
};

// exp(x - m) for a fixed m, two at a time; m = -inf counts as 0.  2^y with y = (x - m) log2 e from the
// special-function unit.  The difference comes first (and not x log2 e - m log2 e in one operation)
// so that x = m gives 1 exactly and no finite logit overflows.  bf16 logits (FAST): the rounding of y,
// 2^-24 of at most a few tens, is far below bf16.  fp32: what y lost (its rounding, and that of log2 e)
// is computed exactly as f and put back as the factor 1 + f ln 2.
template <bool FAST> struct Shift {
  float m;
  __device__ __forceinline__ void set(float top) { m = top == -INFINITY ? 0.0f : top; }
  __device__ __forceinline__ Two operator()(float x0, float x1) const {
    constexpr float kHi = 1.44269502f, kLo = 1.925963033e-8f, kLn2 = 0.693147181f;     // log2 e = kHi + kLo
    Two t = two(x0, x1) + two(-m, -m);
    float y0, y1;
    if (FAST) {
      apart(t * two(kHi, kHi), y0, y1);
      return two(exp2_unit(y0), exp2_unit(y1));
    }
    apart(t, y0, y1);                                      // -inf would give inf - inf below; NaN stays
    t = two(max_nan(y0, -200.0f), max_nan(y1, -200.0f));
    const Two y = t * two(kHi, kHi);
    const Two f = fma_two(t, two(kLo, kLo), fma_two(t, two(kHi, kHi), y * two(-1.0f, -1.0f)));
    apart(y, y0, y1);
    const Two r = two(exp2_unit(y0), exp2_unit(y1));
    return fma_two(r, f * two(kLn2, kLn2), r);
  }
  __device__ __forceinline__ float operator()(float x) const {
    float a, b;
    apart((*this)(x, x), a, b);
    return a;
  }
};

// What the statistics of a row say: its loss and whether its gradient is zero.
struct RowOutcome { float lse, loss; bool zero; };
__device__ __forceinline__ bool target_ignored(const LossParams& P, long long t, float w) { return t == P.ignore_index || w == 0.0f; }
__device__ __forceinline__ bool target_inside(const LossParams& P, long long t) { return t >= 0 && t < P.vocab; }
__device__ __forceinline__ RowOutcome row_outcome(const LossParams& P, float m, float sum, float x_target, long long t, float w) {
  RowOutcome o;
  const bool empty = m == -INFINITY && sum == 0.0f;
  const float l = logf(sum);
  o.lse = empty ? -INFINITY : m + l;
  const bool ignored = target_ignored(P, t, w), outside = !ignored && !target_inside(P, t);
  o.zero = ignored || outside || empty;
  // not lse - x_target: what the logits have in common would take digits from the logarithm
  o.loss = ignored ? 0.0f : outside ? NAN : empty ? INFINITY : w * ((m - x_target) + l);
  return o;
}
__device__ __forceinline__ void report_target(const LossParams& P, long long t, float w) {
  if (!target_ignored(P, t, w) && !target_inside(P, t)) atomicExch(P.status, (int32_t)GBMUF_ERR_INVALID_ARG);
}

// ---- short rows: one warp per row, 32 * kWarpRegs logits in its registers at most
constexpr int kWarpRegs = 64;
constexpr int kWarpVocab = 32 * kWarpRegs;

template <typename T, int REGS>
__global__ void __launch_bounds__(128) cross_entropy_warp_kernel(const LossParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  grid_launch_dependents();
  grid_dependency_wait();
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= P.rows) return;
  const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
  const long long t = P.targets[row];
  const float w = P.scale * (P.row_weight ? P.row_weight[row] : 1.0f);
  const int V = (int)P.vocab;
  float v[REGS];
#pragma unroll
  for (int i = 0; i < REGS; ++i) v[i] = lane + 32 * i < V ? to_f32(x[lane + 32 * i]) : -INFINITY;
  const float xt = target_inside(P, t) ? to_f32(x[t]) : 0.0f;
  float m = v[0];
#pragma unroll
  for (int i = 1; i < REGS; ++i) m = fmaxf(m, v[i]);
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
  m = m == m ? m : -INFINITY;                              // nothing but NaN
  Shift<FAST> e;
  e.set(m);
  Two s01 = two(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < REGS; i += 2) {
    const Two r = e(v[i], v[i + 1]);
    s01 = s01 + r;
    apart(r, v[i], v[i + 1]);
  }
  float s, s1;
  apart(s01, s, s1);
  s += s1;
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
  const RowOutcome o = row_outcome(P, m, s, xt, t, w);
  if (lane == 0) {
    report_target(P, t, w);
    if (P.loss) P.loss[row] = o.loss;
    if (P.lse) P.lse[row] = o.lse;
  }
  if (!P.dlogits) return;
  T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
  const float k = w / s;
#pragma unroll
  for (int i = 0; i < REGS; ++i) {
    const int c = lane + 32 * i;
    if (c < V) d[c] = from_f32<T>(o.zero ? 0.0f : v[i] * k - (c == (int)t ? w : 0.0f));
  }
}

// ---- longer rows.  A cluster of `split` CTAs takes a row; each goes through a slice of its 16-byte
// pieces in chunks that a producer warp fetches into a ring of slots by bulk copies.  256 threads sum
// the chunks as they land (four pieces per thread), the CTAs exchange their maxima and sums, and a
// second walk writes the gradient: first over the slice's last kLossKept chunks, which have stayed in
// their slots, then over the others, last to first, which the producer has fetched again -- from the
// L2 cache: what was read last is needed first, and the host splits rows so that all slices in flight
// fit it.  Two CTAs per SM: one sums while the other one writes or waits.
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

struct RowSpan {
  int a0;                    // elements before the first whole piece
  int pieces;                // whole pieces of the row
  int p0, n;                 // this CTA's pieces
};
__device__ __forceinline__ void loss_workers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kLossWorkers) : "memory"); }
template <typename T> __device__ __forceinline__ RowSpan row_span(const LossParams& P, long long row, int rank) {
  constexpr int E = 16 / (int)sizeof(T);
  RowSpan r;
  const int past = (int)((uintptr_t)(static_cast<const T*>(P.logits) + row * P.ld) % 16 / sizeof(T));
  r.a0 = past ? E - past : 0;                              // vocab > E
  r.pieces = ((int)P.vocab - r.a0) / E;
  r.p0 = (int)((unsigned)r.pieces * (unsigned)rank / (unsigned)P.split);       // pieces * 8 < 2^32
  r.n = (int)((unsigned)r.pieces * (unsigned)(rank + 1) / (unsigned)P.split) - r.p0;
  return r;
}
// What a thread needs of a row besides the ring, asked for a row ahead.  The elements before and after
// the whole pieces, at most 7 each, belong to one thread of rank 0 each.
template <typename T> struct RowAhead {
  long long t;
  float weight, own;
  int at;                    // index of the element in `own`, or -1
  __device__ __forceinline__ void ask(const LossParams& P, long long row, int rank, int thread) {
    constexpr int E = 16 / (int)sizeof(T);
    t = -1; weight = 1.0f; own = -INFINITY; at = -1;
    if (row >= P.rows) return;
    t = P.targets[row];
    if (P.row_weight) weight = P.row_weight[row];
    if (rank != 0 || thread >= 2 * E) return;
    const RowSpan r = row_span<T>(P, row, 0);
    const int e = thread < r.a0 ? thread : r.pieces * E + thread;             // tail: a0 + pieces E + (thread - a0)
    if (e >= (int)P.vocab) return;
    at = e;
    own = to_f32((static_cast<const T*>(P.logits) + row * P.ld)[e]);
  }
};
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

template <typename T>
__global__ void __launch_bounds__(kLossThreads, kLossBlocksPerSm) cross_entropy_ring_kernel(const LossParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  constexpr int E = 16 / (int)sizeof(T);
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t bars = smem_u32(smem), ring = bars + kLossHead;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 64u + 8u * s; };
  auto heard = [&](int b) { return bars + 128u + 8u * b; };
  float2* const told = reinterpret_cast<float2*>(smem + 144);          // [2][8]: statistics of the ranks
  float2* const warp_stat = reinterpret_cast<float2*>(smem + 288);     // [8]
  const int rank = P.split > 1 ? (int)(blockIdx.x % (unsigned)P.split) : 0;
  const long long first = blockIdx.x / (unsigned)P.split, step = gridDim.x / (unsigned)P.split;
  const int thread = threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (thread == 0) {
    for (int s = 0; s < kLossRing; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), kLossWarps); }
    for (int b = 0; b < 2; ++b) mbar_init(heard(b), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (P.split > 1) cluster_sync();                         // barriers exist before a peer uses them
  grid_launch_dependents();
  grid_dependency_wait();

  int slot = 0;                                            // next slot of the ring and its phase
  uint32_t phase = 0;
  auto advance = [&] { if (++slot == kLossRing) { slot = 0; phase ^= 1; } };
  if (thread >= kLossWorkers) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      int filled = 0;
      bool ok = true;
      for (long long row = first; row < P.rows && ok; row += step) {
        const RowSpan r = row_span<T>(P, row, rank);
        const char* const src = reinterpret_cast<const char*>(static_cast<const T*>(P.logits) + row * P.ld + r.a0) + 16ll * r.p0;
        const int chunks = (16 * r.n + kLossChunk - 1) / kLossChunk, again = P.dlogits ? chunks - kLossKept : 0;
        for (int i = 0; i < chunks + (again > 0 ? again : 0) && ok; ++i) {
          const int c = i < chunks ? i : again - 1 - (i - chunks);
          if (filled == kLossRing) ok = mbar_wait_bounded(empty(slot), phase ^ 1, P.status);
          else ++filled;
          if (!ok) break;
          const int left = 16 * r.n - c * kLossChunk;
          const uint32_t bytes = left < kLossChunk ? left : kLossChunk;
          mbar_arrive_expect_tx(full(slot), bytes);
          bulk_load_hint(ring + slot * kLossChunk, src + (long long)c * kLossChunk, bytes, full(slot), c < again && i < chunks);
          advance();
        }
      }
      if (!ok)                                             // copies requested into this CTA's memory land first
        for (int j = 0; j < kLossRing; ++j) { mbar_wait_bounded(full(slot), phase ^ 1, P.status); advance(); }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ 8 worker warps
    bool ok = true;
    RowAhead<T> ahead;
    ahead.ask(P, first, rank, thread);
    int turn = 0;
    for (long long row = first; row < P.rows; row += step, ++turn) {
      const RowSpan r = row_span<T>(P, row, rank);
      const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
      const int chunks = (r.n + kLossPieces * kLossWorkers - 1) / (kLossPieces * kLossWorkers);
      const int again = P.dlogits && chunks > kLossKept ? chunks - kLossKept : 0;      // chunks that are fetched twice
      const RowAhead<T> now = ahead;
      const long long t = now.t;
      const float w = P.scale * now.weight;
      // of the pieces of a slice, this thread's part in chunk c, and the slot's values
      auto left_in = [&](int c) { return r.n - c * kLossPieces * kLossWorkers - thread; };
      auto pieces_in = [&](int s) { return reinterpret_cast<const uint4*>(smem + kLossHead + s * kLossChunk) + thread; };
      auto release = [&](int s) {
        __syncwarp();                                      // one arrival per warp: they are serialised
        if (lane == 0) mbar_arrive(empty(s));
      };

      Shift<FAST> e;
      float m = now.own == now.own ? now.own : -INFINITY;
      e.set(m);
      Two s01 = two(now.at >= 0 && now.own != -INFINITY ? 1.0f + (now.own - now.own) : 0.0f, 0.0f), s23 = two(0.0f, 0.0f);
      // the target's place: chunk and element of the slice, if it is in a whole piece of this CTA's
      const int ti = target_inside(P, t) ? (int)t - r.a0 - r.p0 * E : -1;
      const bool mine = ti >= 0 && ti < r.n * E;
      float xt = 0.0f;                                     // of thread 0
      if (thread == 0 && rank == 0 && target_inside(P, t) && ((int)t < r.a0 || (int)t >= r.a0 + r.pieces * E)) xt = to_f32(x[t]);
      const bool owns = rank == 0 ? (mine || !target_inside(P, t) || (int)t < r.a0 || (int)t >= r.a0 + r.pieces * E) : mine;
      int kept_slot = 0;                                   // slot of the first chunk that stays
      for (int c = 0; c < chunks; ++c) {
        ok = ok && mbar_wait_bounded(full(slot), phase, P.status);
        const int left = left_in(c);
        const uint4* const p = pieces_in(slot);
        if (ok && left > 0) {
          uint4 u[kLossPieces];
#pragma unroll
          for (int h = 0; h < kLossPieces; ++h) u[h] = p[h * kLossWorkers < left ? h * kLossWorkers : 0];
          float v[E];
          float top = piece_max(u[0], v);
#pragma unroll
          for (int h = 1; h < kLossPieces; ++h) top = fmaxf(top, piece_max(u[h], v));
          if (top > m) {
            const float before = m;
            m = top;
            e.set(m);
            if (before != -INFINITY) {                     // else the sums are 0 or NaN
              const float k = e(before);
              s01 = s01 * two(k, k);
              s23 = s23 * two(k, k);
            }
          }
          // whole chunks without a branch between the pieces: their latencies overlap
          auto add = [&](uint4 piece) {
            piece_values(piece, v);
#pragma unroll
            for (int i = 0; i < E; i += 4) {
              s01 = s01 + e(v[i], v[i + 1]);
              s23 = s23 + e(v[i + 2], v[i + 3]);
            }
          };
          if ((kLossPieces - 1) * kLossWorkers < left) {
#pragma unroll
            for (int h = 0; h < kLossPieces; ++h) add(u[h]);
          } else {
#pragma unroll
            for (int h = 0; h < kLossPieces; ++h)
              if (h * kLossWorkers < left) add(u[h]);
          }
        }
        if (thread == 0 && mine && ti / (kLossChunk / (int)sizeof(T)) == c)
          xt = to_f32(reinterpret_cast<const T*>(smem + kLossHead + slot * kLossChunk)[ti % (kLossChunk / (int)sizeof(T))]);
        if (c == again) kept_slot = slot;
        if (c < again || !P.dlogits) release(slot);
        advance();
      }
      float s, s1;
      apart(s01 + s23, s, s1);
      s += s1;
      ahead.ask(P, row + step, rank, thread);
      // statistics of the warp, the CTA, the row: every thread ends with the same bits
      float wm = m;
      for (int d = 16; d > 0; d >>= 1) wm = fmaxf(wm, __shfl_xor_sync(~0u, wm, d));
      if (wm != -INFINITY && m != -INFINITY) s *= expf(m - wm);
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
      if (lane == 0) warp_stat[warp] = make_float2(wm, s);
      loss_workers_sync();
      auto join = [&](float2 st, float& top, float& sum) { // over eight lanes
        top = st.x;
        for (int d = 4; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        sum = st.x == -INFINITY ? st.y : st.y * expf(st.x - top);
        for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
      };
      float top, sum;
      join(warp_stat[lane & 7], top, sum);
      if (P.split > 1) {
        // to every rank; two sets: a peer is one row ahead at most
        const int b = turn & 1;
        if (thread == 0) mbar_arrive_expect_tx(heard(b), 8u * P.split);
        if (thread < P.split)
          asm volatile(
              "{\n\t.reg .b32 ra, rb;\n\t"
              "mapa.shared::cluster.u32 ra, %0, %2;\n\tmapa.shared::cluster.u32 rb, %1, %2;\n\t"
              "st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [ra], {%3, %4}, [rb];\n\t}" ::"r"(
                  smem_u32(&told[b * 8 + rank])),
              "r"(heard(b)), "r"(thread), "f"(top), "f"(sum)
              : "memory");
        ok = mbar_wait_bounded(heard(b), (turn >> 1) & 1, P.status) && ok;
        join((lane & 7) < P.split ? told[b * 8 + (lane & 7)] : make_float2(-INFINITY, 0.0f), top, sum);
      }
      const RowOutcome o = row_outcome(P, top, sum, xt, t, w);
      if (thread == 0) {
        if (rank == 0) { report_target(P, t, w); if (P.lse) P.lse[row] = o.lse; }
        if (owns && P.loss) P.loss[row] = o.loss;
      }
      if (P.dlogits) {
        e.set(top);
        const float k = w / sum;
        T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
        const bool wide = (uintptr_t)(d + r.a0) % 16 == 0;
        if (now.at >= 0) d[now.at] = from_f32<T>(o.zero ? 0.0f : e(now.own) * k - (now.at == t ? w : 0.0f));
        for (int i = 0; i < chunks; ++i) {
          // kept chunks, oldest first, then those that come again
          const bool kept = i < chunks - again;
          const int c = kept ? again + i : chunks - 1 - i, sl = kept ? kept_slot : slot;
          if (!kept) ok = ok && mbar_wait_bounded(full(slot), phase, P.status);
          const int left = left_in(c);
          const uint4* const p = pieces_in(sl);
          if (left > 0 && ok) {
            const int c0 = r.a0 + (r.p0 + c * kLossPieces * kLossWorkers + thread) * E;
            T* const dc = d + c0;
            auto gradient = [&](uint4 piece, float (&v)[E]) {
              piece_values(piece, v);
#pragma unroll
              for (int j = 0; j < E; j += 2) apart(e(v[j], v[j + 1]) * two(k, k), v[j], v[j + 1]);
            };
            if (wide && !o.zero && (kLossPieces - 1) * kLossWorkers < left) {
              uint4 u[kLossPieces];
#pragma unroll
              for (int h = 0; h < kLossPieces; ++h) u[h] = p[h * kLossWorkers];
#pragma unroll
              for (int h = 0; h < kLossPieces; ++h) {
                float v[E];
                gradient(u[h], v);
                ThetaTraits<T>::stg(dc + h * kLossWorkers * E, v);
              }
            } else {
              for (int h = 0; h * kLossWorkers < left && h < kLossPieces; ++h) {
                float v[E] = {};
                if (!o.zero) gradient(p[h * kLossWorkers], v);
                if (wide) ThetaTraits<T>::stg(dc + h * kLossWorkers * E, v);
                else {
#pragma unroll
                  for (int j = 0; j < E; ++j) dc[h * kLossWorkers * E + j] = from_f32<T>(v[j]);
                }
              }
            }
            // the target: the thread that has just stored its piece stores it once more
            const int off = mine ? ti - c * (kLossChunk / (int)sizeof(T)) : -1;
            if (off >= 0 && off < kLossChunk / (int)sizeof(T) && off / E % kLossWorkers == thread && !o.zero) {
              const float y = to_f32(reinterpret_cast<const T*>(smem + kLossHead + sl * kLossChunk)[off]);
              d[t] = from_f32<T>(e(y) * k - w);
            }
          }
          release(sl);
          if (kept) { if (++kept_slot == kLossRing) kept_slot = 0; }
          else advance();
        }
      }
      loss_workers_sync();                                 // warp_stat may be written again
    }
  }
  __syncwarp();
  if (P.split > 1) cluster_sync();                         // no peer writes to a CTA that has ended
}

}  // namespace

#endif  // GBMUF_CSRC_CROSS_ENTROPY_CUH
