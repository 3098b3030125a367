// The largest logits of each row, with their indices and the row's log-sum-exp.
// Part of libgbmuf (CUDA, sm_100a); included by vocab_ops.cu.
#ifndef GBMUF_CSRC_TOP_LOGITS_CUH
#define GBMUF_CSRC_TOP_LOGITS_CUH

namespace {

// One pass over the row.  A logit and its index make one whole number (key) that is larger where the logit
// is, and among equal logits where the index is smaller; keys are all different, so "the k largest" has one
// answer.  The pass keeps only the maximum of each group of 32 or more logits (what a thread sees of a chunk or
// a few).  The k-th largest maximum is a bound that at least k logits reach, and only the groups whose
// maximum reaches it, k of them but for equal ones, hold any of the k largest: they are read again (a few
// KB), and what reaches the bound is ranked.  Both selections go the same way: 256 threads' largest keys
// give a first bound (their k-th largest), what reaches it is put in a buffer, the buffer's k largest are
// kept and sorted.
//
// Rows with so many equal or so unevenly placed logits that lists or buffer overflow are gone through once
// more, chunk by chunk, with a bound that rises: at most k threads have keys above the k-th largest of the
// threads' largest keys, so piece by piece (a thread's 16 bytes) the buffer cannot overflow.
//
// Measured: 2,048 x 267,735 bf16, k 64: 259 to 266 us (4.1 to 4.2 TB/s), of which the log-sum-exp costs 55 (exponentials keep
// their unit 47 % busy) and the selection 28; k 1 without log-sum-exp 178 (6.2 TB/s, 94 % of the copy rate).  Bounds that rise as the
// row goes by, with a look at every piece, took 741.  A row's selection is 9 us, most of it waiting for memory that the
// other block of the SM keeps busy; three blocks per SM, with a ring of two slots, were no faster (279).
struct TopParams {
  const void* logits;
  void* values;
  long long* index;
  float* lse;
  long long rows, vocab, ld, ld_values, ld_index;
  int k, split;
  Temperature temperature;
  int32_t* status;
};
constexpr int kTopMost = 256;                  // k
constexpr int kTopBuffer = kTopMost * 10;      // keys: k kept ones and k pieces of 8, and room
constexpr int kTopGroupBytes = 20480;          // maxima of groups: 40 chunks of bf16 are a group each
constexpr int kTopHot = 1024;                  // groups that are read again
constexpr int kTopShort = 2048;                // vocabulary of the kernel without a ring
typedef unsigned long long Key;

__device__ __forceinline__ Key top_key(float x, int index) {
  const uint32_t b = __float_as_uint(x + 0.0f);                     // -0 counts as 0
  const uint32_t o = x == x ? b ^ ((uint32_t)((int)b >> 31) | 0x80000000u) : 0xffffffffu;
  return (Key)o << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);   // all ones: a NaN
}
__device__ __forceinline__ int key_index(Key k) { return (int)~(uint32_t)k; }
// Maximum of a piece's values, NaN if one of them is.
__device__ __forceinline__ float piece_max_nan(uint4 u, const float (&)[4]) {
  return max_nan(max_nan(__uint_as_float(u.x), __uint_as_float(u.y)), max_nan(__uint_as_float(u.z), __uint_as_float(u.w)));
}
__device__ __forceinline__ float piece_max_nan(uint4 u, const float (&)[8]) {
  auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h(u.x), h(u.y)), __hmax2_nan(h(u.z), h(u.w)));
  return max_nan(__low2float(m), __high2float(m));
}
__device__ __forceinline__ bool any_worker(bool mine) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(any)
               : "r"((uint32_t)mine), "n"(kLossWorkers)
               : "memory");
  return any != 0;
}

__device__ __forceinline__ int count_workers(bool mine) {
  int n;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.popc.u32 %0, 1, %2, p;\n\t}"
               : "=r"(n)
               : "r"((uint32_t)mine), "n"(kLossWorkers)
               : "memory");
  return n;
}

struct TopShared {
  Key buffer[kTopBuffer];
  unsigned char groups[kTopGroupBytes];
  unsigned short hot[kTopHot];
  int counts[64];
  Key threshold;
  uint32_t bounds[8];          // of the ranks
  int count, hot_count;
  float2 stat[kLossWarps];
  float4 told[8];
};

// What the 256 workers of a block keep of a row.  All of them call all functions.
struct TopState {
  TopShared& S;
  int k, thread;
  Key threshold;             // keys at or above it are wanted; the same in all threads

  __device__ __forceinline__ void start() {
    set(0);
    if (thread == 0) S.count = 0;
    loss_workers_sync();
  }
  __device__ __forceinline__ void set(Key t) { threshold = t; }
  // true where the buffer has got long
  __device__ __forceinline__ bool append(Key key) {
    const int at = atomicAdd(&S.count, 1);
    if (at < kTopBuffer) S.buffer[at] = key;
    return at >= k + max(k / 2, 32);
  }
  // A threshold from the threads' largest wanted keys (0: none).  The buffer past `used` is free.
  __device__ __forceinline__ void raise(Key mine, int used) {
    Key* const all = S.buffer + (used + 1) / 2 * 2;
    all[thread] = mine;
    if (thread == 0) S.threshold = threshold;
    loss_workers_sync();
    if (mine != 0) {
      int above = 0;
#pragma unroll 8
      for (int i = 0; i < kLossWorkers; i += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(all + i);
        above += (o.x > mine) + (o.y > mine);
      }
      if (above == k - 1) S.threshold = mine;
    }
    loss_workers_sync();
    set(S.threshold);
    loss_workers_sync();
  }
  // A number that at least k (and not many more) of the threads' numbers reach, or 0 where fewer than k are not 0: bit
  // by bit, from how many threads reach a number.
  // Where few threads reach it, an eighth too many is near enough.
  __device__ __forceinline__ uint32_t bound_of(uint32_t mine, int last_bit) {
    uint32_t bound = 0;
    for (int bit = 31; bit >= last_bit; --bit) {
      const uint32_t next = bound | 1u << bit;
      const int reach = count_workers(mine >= next);
      if (reach >= k) bound = next;
      if (reach >= k && reach <= k + k / 8 && k <= kLossWorkers / 2) break;
    }
    return bound;
  }
  // Sorts the buffer, keeps its k largest keys.  Returns how many keys there had been.
  __device__ __noinline__ int compact() {
    loss_workers_sync();
    const int found = S.count;
    int n = min(found, kTopBuffer);
    constexpr int MOST = kTopBuffer / kLossWorkers;
    if (n > 2 * kLossWorkers && n > k) {
      // Many: the k-th largest bit by bit, from how many keys reach a number; then those that reach it.
      Key mine[MOST], bound = 0;
#pragma unroll
      for (int q = 0; q < MOST; ++q) mine[q] = q * kLossWorkers + thread < n ? S.buffer[q * kLossWorkers + thread] : 0;
      if (thread < 64) S.counts[thread] = 0;
      loss_workers_sync();
      if (thread == 0) S.count = 0;                        // everybody has read it
      for (int bit = 63; bit >= 0; --bit) {
        const Key next = bound | (Key)1 << bit;
        int reach = 0;
#pragma unroll
        for (int q = 0; q < MOST; ++q) reach += mine[q] >= next;
        reach = __reduce_add_sync(~0u, reach);
        if ((thread & 31) == 0) atomicAdd(&S.counts[bit], reach);
        loss_workers_sync();
        reach = S.counts[bit];
        if (reach >= k) bound = next;
        if (reach == k) break;
      }
#pragma unroll
      for (int q = 0; q < MOST; ++q)
        if (mine[q] != 0 && mine[q] >= bound) S.buffer[atomicAdd(&S.count, 1)] = mine[q];
      loss_workers_sync();
      n = S.count;                                         // k: keys are all different
    }
    if (thread == 0 && (n & 1)) S.buffer[n] = 0;           // pairs are read; the buffer's size is even
    loss_workers_sync();
    Key mine[2];
    int rank[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      rank[q] = k;
      if (q * kLossWorkers + (thread & ~31) >= n) continue;    // the same for a warp
      const int i = q * kLossWorkers + thread;
      mine[q] = i < n ? S.buffer[i] : 0;
      int above = 0;
#pragma unroll 4
      for (int j = 0; j < n; j += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(S.buffer + j);
        above += (o.x > mine[q]) + (o.y > mine[q]);
      }
      if (i < n) rank[q] = above;
    }
    loss_workers_sync();
#pragma unroll
    for (int q = 0; q < 2; ++q)
      if (rank[q] < k) S.buffer[rank[q]] = mine[q];
    if (thread == 0) S.count = min(n, k);
    loss_workers_sync();
    if (n >= k) {
      const Key last = S.buffer[k - 1];
      set(last + (last != ~(Key)0));                       // itself is there already
    }
    return found;
  }
  // Whether a key is among the `n` sorted ones at the buffer's start.
  __device__ __forceinline__ bool kept(Key key, int n) const {
    int low = 0, high = n;
    while (low < high) {
      const int mid = (low + high) / 2;
      if (S.buffer[mid] > key) low = mid + 1; else high = mid;
    }
    return low < n && S.buffer[low] == key;
  }
};

// Maxima and sums of the warps, the block: every thread ends with the row's.
template <bool FAST>
__device__ __forceinline__ float2 join_workers(const Temperature& t, float m, float s, float2* stat, int lane, int warp) {
  TemperedShift<FAST> e;
  e.at(t);
  float top = m;
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  e.set(top);
  if (top != -INFINITY && m != -INFINITY) s *= e(m);
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
  if (lane == 0) stat[warp] = make_float2(top, s);
  loss_workers_sync();
  const float2 o = stat[lane & 7];
  top = o.x;
  for (int d = 4; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  e.set(top);
  s = o.x == -INFINITY ? o.y : o.y * e(o.x);
  for (int d = 4; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
  loss_workers_sync();                                     // stat may be written again
  return make_float2(top, s);
}
__device__ __forceinline__ float tempered_lse(const Temperature& t, float m, float s) {
  if (m == -INFINITY && s == 0.0f) return -INFINITY;
  return (float)((double)m * t.inverse + log_of(s));
}
template <typename T> __device__ __forceinline__ void top_write(const TopParams& P, long long row, int at, Key key) {
  const int i = key_index(key);
  const float v = key_value(key);                          // which zero and which NaN it is stands in the row
  static_cast<T*>(P.values)[row * P.ld_values + at] =
      v != 0.0f && v == v ? from_f32<T>(v) : (static_cast<const T*>(P.logits) + row * P.ld)[i];
  P.index[row * P.ld_index + at] = i;
}

// ---- short rows: a block per row, up to eight logits per thread
template <typename T>
__global__ void __launch_bounds__(kLossWorkers) top_short_kernel(const TopParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  constexpr int N = kTopShort / kLossWorkers;
  __shared__ __align__(16) TopShared S;
  grid_launch_dependents();
  grid_dependency_wait();
  const int thread = threadIdx.x, lane = thread & 31, warp = thread >> 5, V = (int)P.vocab;
  for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
    const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
    float v[N];
    Key largest = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = thread + i * kLossWorkers;
      v[i] = c < V ? to_f32(x[c]) : -INFINITY;
      if (c < V) largest = max(largest, top_key(v[i], c));
    }
    TopState top{S, P.k, thread};
    top.start();
    top.raise(largest, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = thread + i * kLossWorkers;
      const Key key = top_key(v[i], c);
      if (c < V && key >= top.threshold) top.append(key);
    }
    top.compact();
    if (thread < P.k) top_write<T>(P, row, thread, S.buffer[thread]);
    if (P.lse) {
      TemperedShift<FAST> e;
      e.at(P.temperature);
      float m = v[0];
#pragma unroll
      for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
      m = m == m ? m : -INFINITY;
      e.set(m);
      Two s = two(0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < N; i += 2) s = s + e(v[i], v[i + 1]);
      float a, b;
      apart(s, a, b);
      const float2 r = join_workers<FAST>(P.temperature, m, a + b, S.stat, lane, warp);
      if (thread == 0) P.lse[row] = tempered_lse(P.temperature, r.x, r.y);
    }
    loss_workers_sync();                                   // the buffer may be written again
  }
}

// ---- longer rows: chunks of a row through a ring of slots, which a producer warp fills.  Few rows: a cluster
// of `split` blocks shares one row, each keeps the k largest of its slice, and rank 0 joins the lists (one
// row per cluster).
constexpr int kTopRing = 4;
constexpr int kTopBlocksPerSm = 2;
constexpr uint32_t kTopHead = (256u + (uint32_t)sizeof(TopShared) + 127u) / 128u * 128u;
constexpr uint32_t kTopSmem = kTopHead + kTopRing * kLossChunk;

// A slice of a row, chunk by chunk, with a rising bound; `at_least`: a bound to begin with.
template <typename T>
__device__ __noinline__ void top_scan(TopState& top, const T* x, const RowSpan r, int chunks, float own, int own_at, Key at_least) {
  constexpr int E = 16 / (int)sizeof(T);
  TopShared& S = top.S;
  const int thread = top.thread;
  top.start();
  top.set(at_least);
  for (int c = 0; c < (chunks > 0 ? chunks : 1); ++c) {
    const int left = c < chunks ? r.n - c * kLossPieces * kLossWorkers - thread : 0;
    const int c0 = r.a0 + (r.p0 + c * kLossPieces * kLossWorkers + thread) * E;
    float v[E];
    // a thread's keys of one piece; h = -1: the element that it holds outside the whole pieces
    auto keys_of = [&](int h, Key (&mine)[E]) {
      const bool there = h >= 0 ? h * kLossWorkers < left : c == 0 && own_at >= 0;
      uint4 piece = make_uint4(0, 0, 0, 0);
      if (there && h >= 0) piece = *reinterpret_cast<const uint4*>(x + c0 + h * kLossWorkers * E);
      piece_values(piece, v);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        mine[i] = !there ? 0 : h >= 0 ? top_key(v[i], c0 + h * kLossWorkers * E + i) : i == 0 ? top_key(own, own_at) : 0;
        if (mine[i] < top.threshold) mine[i] = 0;
      }
    };
    bool lengthy = false;
#pragma unroll 1
    for (int h = -1; h < kLossPieces; ++h) {
      Key mine[E];
      keys_of(h, mine);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (mine[i] != 0) lengthy |= top.append(mine[i]);
    }
    if (!any_worker(lengthy)) continue;
    if (top.compact() <= kTopBuffer) continue;
    // what did not fit: piece by piece; keys that are there already are passed over
#pragma unroll 1
    for (int h = -1; h < kLossPieces; ++h) {
      const int have = S.count;
      Key mine[E], largest = 0;
      keys_of(h, mine);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (mine[i] != 0 && top.kept(mine[i], have)) mine[i] = 0;
        largest = max(largest, mine[i]);
      }
      loss_workers_sync();                                 // the count has been read
      top.raise(largest, have);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (mine[i] != 0 && mine[i] >= top.threshold) top.append(mine[i]);
      top.compact();
    }
  }
  top.compact();
}

template <typename T>
__global__ void __launch_bounds__(kLossThreads, kTopBlocksPerSm) top_ring_kernel(const TopParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  constexpr int E = 16 / (int)sizeof(T);
  typedef std::conditional_t<FAST, unsigned short, unsigned> Order;    // a maximum, as a whole number in its order
  constexpr int GROUPS = kTopGroupBytes / (int)sizeof(Order) / kLossWorkers;       // per thread
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t bars = smem_u32(smem), ring = bars + kTopHead;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 64u + 8u * s; };
  TopShared& S = *reinterpret_cast<TopShared*>(smem + 256);
  const int rank = P.split > 1 ? (int)(blockIdx.x % (unsigned)P.split) : 0;
  const long long first = blockIdx.x / (unsigned)P.split, step = gridDim.x / (unsigned)P.split;
  const int thread = threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (thread == 0) {
    for (int s = 0; s < kTopRing; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), kLossWarps); }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (P.split > 1) cluster_sync();                         // every block has started before a peer writes to it
  grid_launch_dependents();
  grid_dependency_wait();
  int slot = 0;
  uint32_t phase = 0;
  auto advance = [&] { if (++slot == kTopRing) { slot = 0; phase ^= 1; } };
  if (thread >= kLossWorkers) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      int filled = 0;
      bool ok = true;
      for (long long row = first; row < P.rows && ok; row += step) {
        const RowSpan r = row_span<T>(P, row, rank);
        const char* const src = reinterpret_cast<const char*>(static_cast<const T*>(P.logits) + row * P.ld + r.a0) + 16ll * r.p0;
        const int chunks = (int)((16ll * r.n + kLossChunk - 1) / kLossChunk);
        for (int c = 0; c < chunks; ++c) {
          if (filled == kTopRing) ok = mbar_wait_bounded(empty(slot), phase ^ 1, P.status);
          else ++filled;
          if (!ok) break;
          const long long left = 16ll * r.n - (long long)c * kLossChunk;
          const uint32_t bytes = left < kLossChunk ? (uint32_t)left : (uint32_t)kLossChunk;
          mbar_arrive_expect_tx(full(slot), bytes);
          bulk_load_row(ring + slot * kLossChunk, src + (long long)c * kLossChunk, bytes, full(slot));
          advance();
        }
      }
      if (!ok)                                             // copies requested into this block's memory land first
        for (int j = 0; j < kTopRing; ++j) { mbar_wait_bounded(full(slot), phase ^ 1, P.status); advance(); }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ 8 worker warps
    bool ok = true;
    Order* const groups = reinterpret_cast<Order*>(S.groups);
    for (long long row = first; row < P.rows; row += step) {
      const RowSpan r = row_span<T>(P, row, rank);
      const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
      const int chunks = (r.n + kLossPieces * kLossWorkers - 1) / (kLossPieces * kLossWorkers);
      const int run = (chunks + GROUPS - 1) / GROUPS;      // chunks of a group
      // the elements before and after the whole pieces: one thread of rank 0 each
      float own = -INFINITY;
      int own_at = -1;
      if (rank == 0 && thread < 2 * E) {
        const int at = thread < r.a0 ? thread : r.pieces * E + thread;
        if (at < (int)P.vocab) { own_at = at; own = to_f32(x[at]); }
      }
      TemperedShift<FAST> e;
      e.at(P.temperature);
      float m = own == own ? own : -INFINITY;
      e.set(m);
      Two s01 = two(own_at >= 0 && own != -INFINITY ? 1.0f + (own - own) : 0.0f, 0.0f), s23 = two(0.0f, 0.0f);
      uint32_t largest = 0;                                // order of this thread's largest maximum
      float group = -INFINITY;
      int in_run = 0, mine = 0;                            // chunks of the group so far, groups so far
      for (int c = 0; c < chunks; ++c) {
        ok = ok && mbar_wait_bounded(full(slot), phase, P.status);
        const int left = r.n - c * kLossPieces * kLossWorkers - thread;
        const uint4* const p = reinterpret_cast<const uint4*>(smem + kTopHead + slot * kLossChunk) + thread;
        uint4 u[kLossPieces];
        float v[E];
        const bool whole = (kLossPieces - 1) * kLossWorkers < left;
#pragma unroll
        for (int h = 0; h < kLossPieces; ++h) u[h] = p[h * kLossWorkers < left ? h * kLossWorkers : 0];
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(slot));
        advance();
        if (left > 0 && ok) {
          float top = piece_max_nan(u[0], v);              // what is missing counts as the first piece again
#pragma unroll
          for (int h = 1; h < kLossPieces; ++h) top = max_nan(top, piece_max_nan(u[h], v));
          group = max_nan(group, top);
          if (P.lse) {
            if (top > m || top != top) {
              const float before = m;
              if (top != top) s01 = s01 + two(top, top);   // a NaN among them: the sum is one
              else m = top;
              e.set(m);
              if (before != -INFINITY) {
                const float f = e(before);
                s01 = s01 * two(f, f);
                s23 = s23 * two(f, f);
              }
            }
            auto add = [&](uint4 piece) {
              piece_values(piece, v);
#pragma unroll
              for (int i = 0; i < E; i += 4) {
                s01 = s01 + e(v[i], v[i + 1]);
                s23 = s23 + e(v[i + 2], v[i + 3]);
              }
            };
            if (whole) {
#pragma unroll
              for (int h = 0; h < kLossPieces; ++h) add(u[h]);
            } else {
#pragma unroll
              for (int h = 0; h < kLossPieces; ++h)
                if (h * kLossWorkers < left) add(u[h]);
            }
          }
        }
        if (++in_run == run || c == chunks - 1) {
          const bool any = r.n - (c + 1 - in_run) * kLossPieces * kLossWorkers - thread > 0;
          const uint32_t order = any ? (uint32_t)(top_key(group, 0) >> 32) >> (FAST ? 16 : 0) : 0u;
          groups[mine * kLossWorkers + thread] = (Order)order;
          largest = max(largest, order << (FAST ? 16 : 0));
          group = -INFINITY;
          in_run = 0;
          ++mine;
        }
      }
      TopState top{S, P.k, thread};
      auto group_order = [&](int g) { return (uint32_t)groups[g * kLossWorkers + thread] << (FAST ? 16 : 0); };
      // (bf16: the lower half of an order is left out on both sides)
      if (thread == 0) S.hot_count = 0;
      top.start();
      uint32_t least = top.bound_of(largest, FAST ? 16 : 0);
      if (P.split > 1) {                                   // the best of all ranks' bounds
        if (thread < P.split) {
          uint32_t there;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(&S.bounds[rank])), "r"(thread));
          asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(there), "r"(least) : "memory");
        }
        cluster_sync();
        for (int o = 0; o < P.split; ++o) least = max(least, S.bounds[o]);
      }
      auto list_groups = [&] {
        if (largest >= least) {
          unsigned long long wanted = 0;
          for (int g0 = 0; g0 < mine; g0 += 8)
#pragma unroll
            for (int g = g0; g < g0 + 8; ++g) {
              const uint32_t o = g < mine ? group_order(g) : 0u;
              if (o != 0 && o >= least) wanted |= 1ull << g;
            }
          int at = wanted ? atomicAdd(&S.hot_count, __popcll(wanted)) : 0;
          for (; wanted; wanted &= wanted - 1, ++at)
            if (at < kTopHot) S.hot[at] = (unsigned short)((__ffsll(wanted) - 1) * kLossWorkers + thread);
        }
        loss_workers_sync();
        return S.hot_count;
      };
      int hot = list_groups();
      if (hot > 2 * P.k + 64) {
        // k near the number of threads, or many equal maxima: the k-th largest of all groups' maxima
        loss_workers_sync();
        if (thread == 0) S.hot_count = 0;
        for (int g = 0; g < mine; ++g) {
          const uint32_t o = group_order(g);
          if (o != 0 && o >= least) top.append((Key)o << 32 | (uint32_t)~(g * kLossWorkers + thread));
        }
        if (top.compact() <= kTopBuffer && S.count >= P.k) least = (uint32_t)(S.buffer[P.k - 1] >> 32);
        loss_workers_sync();                               // buffer and count have been read
        if (thread == 0) S.count = 0;
        hot = list_groups();
      }
      const Key bound = (Key)least << 32;
      top.set(bound);
      if (own_at >= 0 && top_key(own, own_at) >= bound) top.append(top_key(own, own_at));
      bool again = hot > kTopHot;
      if (!again) {
        // a warp takes the pieces of several groups at a time, a lane an element of a piece of one chunk of the run
        constexpr int LANES = E * kLossPieces, AT_ONCE = 32 / LANES, BATCH = 12;
        const int part = lane / LANES, h = lane % LANES / E, i = lane % E, items = hot * run;
        for (int j0 = warp * AT_ONCE + part; j0 - part < items; j0 += kLossWarps * AT_ONCE * BATCH) {
          int at[BATCH];
          T y[BATCH];
#pragma unroll
          for (int b = 0; b < BATCH; ++b) {
            const int j = j0 + b * kLossWarps * AT_ONCE;
            at[b] = -1;
            if (j >= items) continue;
            const int id = S.hot[run == 1 ? j : j / run], c = id / kLossWorkers * run + (run == 1 ? 0 : j % run);
            const int piece = (c * kLossPieces + h) * kLossWorkers + id % kLossWorkers;
            if (c >= chunks || piece >= r.n) continue;
            at[b] = r.a0 + (r.p0 + piece) * E + i;
            y[b] = x[at[b]];
          }
          // one place in the buffer for all that a lane has found
          unsigned found = 0;
#pragma unroll
          for (int b = 0; b < BATCH; ++b)
            if (at[b] >= 0 && top_key(to_f32(y[b]), at[b]) >= bound) found |= 1u << b;
          if (found) {
            int to = atomicAdd(&S.count, __popc(found));
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
              if (found >> b & 1) {
                if (to < kTopBuffer) S.buffer[to] = top_key(to_f32(y[b]), at[b]);
                ++to;
              }
          }
        }
        again = top.compact() > kTopBuffer;
      }
      if (again) top_scan<T>(top, x, r, chunks, own, own_at, bound);
      float2 stat = make_float2(0.0f, 0.0f);
      if (P.lse) {
        float a, b;
        apart(s01 + s23, a, b);
        stat = join_workers<FAST>(P.temperature, m, a + b, S.stat, lane, warp);
      }
      if (P.split == 1) {
        if (thread < P.k) top_write<T>(P, row, thread, S.buffer[thread]);
        if (P.lse && thread == 0) P.lse[row] = tempered_lse(P.temperature, stat.x, stat.y);
        loss_workers_sync();                               // the buffer may be written again
      } else {
        // this block's list for rank 0
        const int n = min(S.count, P.k);
        const Key key = thread < n ? S.buffer[thread] : 0;
        cluster_sync();                                    // nobody uses rank 0's buffer any more
        uint32_t list, told;
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(list) : "r"(smem_u32(&S.buffer[rank * kTopMost + thread])));
        asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(told) : "r"(smem_u32(&S.told[rank])));
        if (thread < n) asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(list), "l"(key) : "memory");
        if (thread == 0)
          asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %3};" ::"r"(told), "f"(stat.x), "f"(stat.y), "f"(__int_as_float(n))
                       : "memory");
        cluster_sync();
        if (rank == 0) {
          // the lists behind one another, and the k largest of them
          Key keys[8];
          int place[8], total = 0;
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int n_q = q < P.split ? __float_as_int(S.told[q].z) : 0;
            keys[q] = thread < n_q ? S.buffer[q * kTopMost + thread] : 0;
            place[q] = total + thread;
            total += n_q;
          }
          loss_workers_sync();
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (keys[q] != 0) S.buffer[place[q]] = keys[q];
          if (thread == 0) S.count = total;
          top.compact();
          if (thread < P.k) top_write<T>(P, row, thread, S.buffer[thread]);
          if (P.lse && thread == 0) {
            float hi = -INFINITY, sum = 0.0f;
            for (int o = 0; o < P.split; ++o) hi = fmaxf(hi, S.told[o].x);
            e.set(hi);
            for (int o = 0; o < P.split; ++o) sum += S.told[o].x == -INFINITY ? S.told[o].y : S.told[o].y * e(S.told[o].x);
            P.lse[row] = tempered_lse(P.temperature, hi, sum);
          }
        }
      }
    }
  }
  if (P.split > 1 && thread >= kLossWorkers) {             // the producer's part in the exchanges above
    cluster_sync();
    cluster_sync();
    cluster_sync();
  }
}

}  // namespace

#endif  // GBMUF_CSRC_TOP_LOGITS_CUH
