// Cross-entropy of a softmax over a vocabulary, with its gradient.
// Part of libgbmuf (CUDA, sm_100a); included by local_ops.cu.
#ifndef GBMUF_CSRC_CROSS_ENTROPY_CUH
#define GBMUF_CSRC_CROSS_ENTROPY_CUH

namespace {

// Per row: m = max x, s = sum exp(x - m), then d = s_i (exp(x - m) / s - [target]).  Every logit is
// needed twice with the whole row between, so the row stays on the chip from its one read to its
// one write: in the registers of a warp (short rows), or in the shared memory of 1 to 8 CTAs of a
// cluster (16 KB to 1.1 MB of it).  Only longer rows are read twice.
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

// Two fp32 operations per instruction.
struct Two { unsigned long long u; };
__device__ __forceinline__ Two two(float x, float y) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.u) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void apart(Two t, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(t.u)); }
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
  return r;
}
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
  return r;
}

// exp(x - m) for a fixed m, two at a time; m = -inf counts as 0.  2^y with y = (x - m) log2 e from the
// special-function unit.  The difference comes first (and not x log2 e - m log2 e in one operation)
// so that x = m gives 1 exactly and no finite logit overflows.  bf16 logits (FAST): the rounding of y,
// 2^-24 of at most a few tens, is far below bf16.  fp32: what y lost (its rounding, and that of log2 e)
// is computed exactly as f and put back as the factor 1 + f ln 2.
template <bool FAST> struct Shift {
  float m;
  __device__ __forceinline__ void set(float top) { m = top == -INFINITY ? 0.0f : top; }
  __device__ __forceinline__ static float exp2_unit(float y) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    return r;
  }
  __device__ __forceinline__ Two operator()(float x0, float x1) const {
    constexpr float kHi = 1.44269502f, kLo = 1.925963033e-8f, kLn2 = 0.693147181f;     // log2 e = kHi + kLo
    Two t = two(x0, x1) + two(-m, -m);
    float y0, y1;
    if (FAST) {
      apart(t * two(kHi, kHi), y0, y1);
      return two(exp2_unit(y0), exp2_unit(y1));
    }
    apart(t, y0, y1);                                      // -inf would give inf - inf below; NaN stays
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(y0) : "f"(-200.0f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(y1) : "f"(-200.0f));
    t = two(y0, y1);
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

// (m, s): s = sum of exp(x - m) over some logits.  m = -inf: nothing but -inf (s = 0), or NaN (s).
__device__ __forceinline__ void softmax_merge(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  if (top == -INFINITY) { s += s2; return; }
  s = s * expf(m - top) + s2 * expf(m2 - top);
  m = top;
}

// What the statistics of a row say: its loss and whether its gradient is zero.
struct RowOutcome { float lse, loss; bool zero; };
__device__ __forceinline__ bool target_ignored(const LossParams& P, long long t, float w) { return t == P.ignore_index || w == 0.0f; }
__device__ __forceinline__ bool target_inside(const LossParams& P, long long t) { return t >= 0 && t < P.vocab; }
__device__ __forceinline__ RowOutcome row_outcome(const LossParams& P, float m, float sum, float x_target, long long t, float w) {
  RowOutcome o;
  const bool empty = m == -INFINITY && sum == 0.0f;
  o.lse = empty ? -INFINITY : m + logf(sum);
  const bool ignored = target_ignored(P, t, w), outside = !ignored && !target_inside(P, t);
  o.zero = ignored || outside || empty;
  o.loss = ignored ? 0.0f : outside ? NAN : empty ? INFINITY : w * (o.lse - x_target);
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

// ---- rows in shared memory.  A cluster of `split` CTAs takes a row; each holds a slice of its
// 16-byte pieces as chunks in a ring of slots that a producer warp keeps filled by bulk copies.  A
// group of 8 warps goes through the chunks as they land (two pieces per thread and chunk) and keeps a
// running maximum and sum, the CTAs exchange theirs, and a second walk over the same slots writes the
// gradient and frees the slots one by one.  Two groups take alternate rows: while one waits for the
// other CTAs, or writes, the other one's chunks arrive and are summed.
constexpr int kLossGroups = 2;
constexpr int kLossWorkers = 256;                          // threads of a group
constexpr int kLossThreads = kLossGroups * kLossWorkers + 32;
constexpr int kLossChunk = 32 * kLossWorkers;              // bytes: two pieces per thread
constexpr int kLossRing = 26;
constexpr int kLossMostChunks = 18;                        // of one row in one CTA: the rest is ahead
constexpr uint32_t kLossHead = 1280;
constexpr uint32_t kLossSmem = kLossHead + kLossRing * kLossChunk;

struct RowSpan {
  int a0;                    // elements before the first whole piece
  int pieces;                // whole pieces of the row
  int p0, n;                 // this CTA's pieces
};
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
__global__ void __launch_bounds__(kLossThreads, 1) cross_entropy_ring_kernel(const LossParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  constexpr int E = 16 / (int)sizeof(T);
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t bars = smem_u32(smem), ring = bars + kLossHead;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 256u + 8u * s; };
  auto heard = [&](int b) { return bars + 512u + 8u * b; };            // [group][2]
  float2* const told = reinterpret_cast<float2*>(smem + 576);          // [group][2][8]: statistics of the ranks
  float2* const warp_stat = reinterpret_cast<float2*>(smem + 896);     // [group][8]
  const int rank = P.split > 1 ? (int)(blockIdx.x % (unsigned)P.split) : 0;
  const long long first = blockIdx.x / (unsigned)P.split, step = gridDim.x / (unsigned)P.split;
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kLossRing; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), kLossWorkers); }
    for (int b = 0; b < 2 * kLossGroups; ++b) mbar_init(heard(b), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (P.split > 1) cluster_sync();                         // barriers exist before a peer uses them

  if (threadIdx.x >= kLossGroups * kLossWorkers) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      int n = 0, slot = 0;
      uint32_t round = 0;
      bool ok = true;
      for (long long row = first; row < P.rows && ok; row += step) {
        const RowSpan r = row_span<T>(P, row, rank);
        const char* src = reinterpret_cast<const char*>(static_cast<const T*>(P.logits) + row * P.ld + r.a0) + 16ll * r.p0;
        for (int left = 16 * r.n; left > 0; left -= kLossChunk, src += kLossChunk) {
          if (n >= kLossRing) ok = mbar_wait_bounded(empty(slot), round ^ 1, P.status);
          if (!ok) break;
          const uint32_t bytes = left < kLossChunk ? left : kLossChunk;
          mbar_arrive_expect_tx(full(slot), bytes);
          bulk_load_row(ring + slot * kLossChunk, src, bytes, full(slot));
          if (n < kLossRing) ++n;
          if (++slot == kLossRing) { slot = 0; round ^= 1; }
        }
      }
      if (!ok)                                             // copies requested into this CTA's memory land first
        for (int j = 0; j < kLossRing; ++j) {
          const int s = (slot + j) % kLossRing;
          mbar_wait_bounded(full(s), s >= slot ? round ^ 1 : round, P.status);
        }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ two groups of 8 warps
    const int group = threadIdx.x / kLossWorkers, thread = threadIdx.x % kLossWorkers, warp = thread >> 5;
    auto group_sync = [&] { asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(kLossWorkers) : "memory"); };
    int slot = 0, turn = 0;
    uint32_t round = 0;
    auto advance = [&](int& s, uint32_t& rd, int by) {
      s += by;
      while (s >= kLossRing) { s -= kLossRing; rd ^= 1; }
    };
    auto chunks_of = [&](const RowSpan& r) { return (r.n + 2 * kLossWorkers - 1) / (2 * kLossWorkers); };
    bool ok = true;
    long long row = first + group * step;
    if (group == 1 && first < P.rows) advance(slot, round, chunks_of(row_span<T>(P, first, rank)));
    RowAhead<T> ahead;
    ahead.ask(P, row, rank, thread);
    for (; row < P.rows; row += kLossGroups * step, ++turn) {
      const RowSpan r = row_span<T>(P, row, rank);
      const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
      const int chunks = chunks_of(r);
      const RowAhead<T> now = ahead;
      const long long t = now.t;
      const float w = P.scale * now.weight;

      Shift<FAST> e;
      float m = now.own == now.own ? now.own : -INFINITY;
      e.set(m);
      Two s01 = two(now.at >= 0 && now.own != -INFINITY ? 1.0f + (now.own - now.own) : 0.0f, 0.0f);
      int sl = slot;
      uint32_t rd = round;
      for (int c = 0; c < chunks; ++c) {
        ok = ok && mbar_wait_bounded(full(sl), rd, P.status);
        const int piece = c * 2 * kLossWorkers + thread;
        const uint4* const p = reinterpret_cast<const uint4*>(smem + kLossHead + sl * kLossChunk) + thread;
        if (ok && piece < r.n) {
          const bool both = piece + kLossWorkers < r.n;
          const uint4 u = p[0], u2 = both ? p[kLossWorkers] : u;
          float v[E], v2[E];
          const float top = fmaxf(piece_max(u, v), piece_max(u2, v2));
          if (top > m) {
            const float before = m;
            m = top;
            e.set(m);
            if (before != -INFINITY) { const float k = e(before); s01 = s01 * two(k, k); }   // else s is 0 or NaN
          }
          piece_values(u, v);
#pragma unroll
          for (int i = 0; i < E; i += 2) s01 = s01 + e(v[i], v[i + 1]);
          if (both) {
            piece_values(u2, v2);
#pragma unroll
            for (int i = 0; i < E; i += 2) s01 = s01 + e(v2[i], v2[i + 1]);
          }
        }
        advance(sl, rd, 1);
      }
      float s, s1;
      apart(s01, s, s1);
      s += s1;
      // the target's logit, before anything of the row may be overwritten, and whether this CTA has it
      bool owns = rank == 0;
      float xt = 0.0f;
      if (thread == 0 && target_inside(P, t)) {
        const int i = (int)t - r.a0;
        if (i < 0 || i >= r.pieces * E) {
          if (owns) xt = to_f32(x[t]);
        } else {
          const int piece = i / E - r.p0;
          owns = piece >= 0 && piece < r.n;
          if (owns) {
            int at = slot;
            uint32_t unused = 0;
            advance(at, unused, piece / (2 * kLossWorkers));
            xt = to_f32(reinterpret_cast<const T*>(smem + kLossHead + at * kLossChunk)[piece % (2 * kLossWorkers) * E + i % E]);
          }
        }
      }
      ahead.ask(P, row + kLossGroups * step, rank, thread);
      // statistics of the warp, the CTA, the row: every thread ends with the same bits
      float wm = m;
      for (int d = 16; d > 0; d >>= 1) wm = fmaxf(wm, __shfl_xor_sync(~0u, wm, d));
      if (wm != -INFINITY && m != -INFINITY) s *= expf(m - wm);
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
      if (lane == 0) warp_stat[group * 8 + warp] = make_float2(wm, s);
      group_sync();
      const float2 st = warp_stat[group * 8 + (lane & 7)];
      float top = st.x;
      for (int d = 4; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
      float sum = st.x == -INFINITY ? st.y : st.y * expf(st.x - top);
      for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
      if (P.split > 1) {
        // to every rank; two sets per group: a peer's group is one of its rows ahead at most
        const int b = 2 * group + (turn & 1);
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
        const float2 all = (lane & 7) < P.split ? told[b * 8 + (lane & 7)] : make_float2(-INFINITY, 0.0f);
        top = all.x;
        for (int d = 4; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        sum = all.x == -INFINITY ? all.y : all.y * expf(all.x - top);
        for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
      }
      const RowOutcome o = row_outcome(P, top, sum, xt, t, w);
      if (thread == 0) {
        if (rank == 0) { report_target(P, t, w); if (P.lse) P.lse[row] = o.lse; }
        if (owns && P.loss) P.loss[row] = o.loss;
      }
      e.set(top);
      const float k = w / sum;
      T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
      const bool wide = (uintptr_t)(d + r.a0) % 16 == 0;
      if (P.dlogits && now.at >= 0) d[now.at] = from_f32<T>(o.zero ? 0.0f : e(now.own) * k - (now.at == t ? w : 0.0f));
      for (int c = 0; c < chunks; ++c) {
        const uint4* const p = reinterpret_cast<const uint4*>(smem + kLossHead + slot * kLossChunk) + thread;
        const int piece = c * 2 * kLossWorkers + thread;
        if (P.dlogits) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (piece + h * kLossWorkers >= r.n) break;
            float v[E];
            piece_values(p[h * kLossWorkers], v);
            const int c0 = r.a0 + (r.p0 + piece + h * kLossWorkers) * E;
            const unsigned hit = (unsigned)((int)t - c0);  // t is inside the vocabulary, or o.zero
            if (o.zero) {
#pragma unroll
              for (int i = 0; i < E; ++i) v[i] = 0.0f;
            } else {
#pragma unroll
              for (int i = 0; i < E; i += 2) apart(e(v[i], v[i + 1]) * two(k, k), v[i], v[i + 1]);
              if (hit < E) {
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] -= (int)hit == i ? w : 0.0f;
              }
            }
            if (wide) ThetaTraits<T>::stg(d + c0, v);
            else {
#pragma unroll
              for (int i = 0; i < E; ++i) d[c0 + i] = from_f32<T>(v[i]);
            }
          }
        }
        mbar_arrive(empty(slot));
        advance(slot, round, 1);
      }
      // past the other group's next row
      if (row + step < P.rows) advance(slot, round, chunks_of(row_span<T>(P, row + step, rank)));
      group_sync();                                        // warp_stat may be written again
    }
  }
  __syncwarp();
  if (P.split > 1) cluster_sync();                         // no peer writes to a CTA that has ended
}

// ---- rows longer than that: read twice, one block per row
template <typename T>
__global__ void __launch_bounds__(512) cross_entropy_twice_kernel(const LossParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  __shared__ float2 stat[16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
    float m = -INFINITY, s = 0.0f;
    Shift<FAST> e;
    e.set(m);
#pragma unroll 4
    for (long long v = threadIdx.x; v < P.vocab; v += 512) {
      const float y = to_f32(x[v]);
      if (y > m) {
        s *= m == -INFINITY ? 1.0f : expf(m - y);
        m = y;
        e.set(m);
      }
      s += e(y);
    }
    for (int d = 16; d > 0; d >>= 1) {
      const float m2 = __shfl_xor_sync(~0u, m, d), s2 = __shfl_xor_sync(~0u, s, d);
      softmax_merge(m, s, m2, s2);
    }
    if (lane == 0) stat[warp] = make_float2(m, s);
    __syncthreads();
    m = stat[0].x; s = stat[0].y;
    for (int i = 1; i < 16; ++i) softmax_merge(m, s, stat[i].x, stat[i].y);
    const long long t = P.targets[row];
    const float w = P.scale * (P.row_weight ? P.row_weight[row] : 1.0f);
    const float xt = target_inside(P, t) ? to_f32(x[t]) : 0.0f;
    __syncthreads();                                       // dlogits may be the logits
    const RowOutcome o = row_outcome(P, m, s, xt, t, w);
    if (threadIdx.x == 0) {
      report_target(P, t, w);
      if (P.loss) P.loss[row] = o.loss;
      if (P.lse) P.lse[row] = o.lse;
    }
    if (!P.dlogits) continue;
    T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
    e.set(m);
    const float k = w / s;
#pragma unroll 4
    for (long long v = threadIdx.x; v < P.vocab; v += 512)
      d[v] = from_f32<T>(o.zero ? 0.0f : e(to_f32(x[v])) * k - (v == t ? w : 0.0f));
  }
}

}  // namespace

#endif  // GBMUF_CSRC_CROSS_ENTROPY_CUH
