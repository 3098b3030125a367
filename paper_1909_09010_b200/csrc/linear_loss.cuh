// The softmax layer with its cross-entropy: what happens to a tile of logits while it is in tensor memory.
// Part of libgbmuf (CUDA, sm_100a); included before linear_tc.cuh.
#ifndef GBMUF_CSRC_LINEAR_LOSS_CUH
#define GBMUF_CSRC_LINEAR_LOSS_CUH

namespace {

// z = x w^T + bias is formed twice and never stored.  The first time (kLossStats) a thread of the finishing
// warps owns a row of the batch and goes through that row's logits of a tile with a running maximum and
// sum: rows of the batch lie along the lanes, words along the columns, so no two threads share a row's tile.
// The second time (kLossGrad) words lie along the lanes and d = w (exp(z - m) / s - [target]) of a piece of
// the vocabulary is stored, once, as the operand of the two products that follow: rounded to bf16, or for
// fp32 as its three parts.  bf16: that rounding is off by at most 2^-8 of an element, and the products'
// sums of many such elements by less.  What all rows have in common is a factor of the finished fp32 sums, the scale
// and the largest weight of a row that counts: within d it would be rounded the same way in every row, so that
// 1 / 300 (say) would take 0.2 % off every gradient, where a target's -1 is exact.  So w is the row's weight over that
// largest one: 1 where all are equal, or a mask.  Where they differ, each is rounded its own way, by 2^-8 at most, as
// any other element of d; up to kLossTwice weighted rows, which fill half a step of the sums and half a
// tile at most, come a second time, with what the rounding left: 16 bits of d (32 x 512 x 10,000: 47 -> 56 us).

// What kLossGrad needs of two rows of the batch, as two packed operands: minus their maxima, and weight / sum.
// Next to it stand per row the target (-1: no word of the vocabulary; -2: the row's gradient is zero) and the
// weight.
struct __align__(16) RowPair { float m[2], k[2]; };
constexpr int kLossRowPad = 256;   // rows of a tile, at most: the arrays cover all tiles
constexpr int kLossTwice = 32;

// Statistics of a row of the batch.  2,048 x 1,024 x 100,000 bf16: 263 us in short runs (1,595 TFLOP/s, tensor pipe 84 %
// active), bound by the products; 1,024 x 512 x 267,735: 217 to 232 us (1,210 to 1,290 TFLOP/s): eight steps a tile, whose
// epilogue takes as long.  Strips of 32 words: with 16 the loads' latencies and the tests cost 5 us more there.
template <typename T> struct RowStats {
  static constexpr bool FAST = sizeof(T) == 2;
  float m = -INFINITY;
  Two s = two(0.0f, 0.0f);
  int row = -1, slot = 0, target = -1;
  bool there = false;
  Shift<FAST> e;

  __device__ __forceinline__ void open(const Epilogue& E, int c, int rows, int at) {
    if (c == row) return;
    close(E);
    row = c;
    slot = at;
    m = -INFINITY;
    s = two(0.0f, 0.0f);
    e.set(m);
    there = c < rows;
    const long long t = there ? static_cast<const long long*>(E.loss_rows)[c] : -1;
    target = t >= 0 && t <= 0x7fffffff ? (int)t - E.first_word : -1;
    if (!FAST || !E.weight_max || slot != 0) return;       // one warp for each 32 rows
    const float w = there && t >= 0 && t < E.vocab && t != E.ignore_index ? fabsf(E.loss_weights[c]) : 0.0f;
    float top = E.scale * w != 0.0f && w < INFINITY ? w : 0.0f;
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    if (there && (c & 31) == 0) E.weight_max[c >> 5] = top;
  }
  // N words from r on
  template <int N> __device__ __forceinline__ void add(const Epilogue& E, float (&v)[N], int r, int words) {
    if (r + N > words) {                                   // the vocabulary's end
#pragma unroll
      for (int i = 0; i < N; ++i)
        v[i] = r + i >= words ? -INFINITY : E.bias ? v[i] + to_f32(static_cast<const T*>(E.bias)[r + i]) : v[i];
    } else if (E.bias) {
      const T* const bias = static_cast<const T*>(E.bias) + r;
      if (FAST && (uintptr_t)bias % 16 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
          const uint4 u = *reinterpret_cast<const uint4*>(bias + i);
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            apart(two(v[i + 2 * j], v[i + 2 * j + 1]) + two(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u)),
                  v[i + 2 * j], v[i + 2 * j + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += to_f32(bias[i]);
      }
    }
    const int at_target = target - r;
    if ((unsigned)at_target < (unsigned)N && target >= 0) {
      float x = v[0];
#pragma unroll
      for (int i = 1; i < N; ++i) x = at_target == i ? v[i] : x;
      E.target_logit[row] = x;
    }
    float top = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
    if (top > m) {
      const float before = m;
      m = top;
      e.set(m);
      if (before != -INFINITY) {                           // else the sum is 0 or NaN
        const float k = e(before);
        s = s * two(k, k);
      }
    }
#pragma unroll
    for (int i = 0; i < N; i += 2) s = s + e(v[i], v[i + 1]);
  }
  __device__ __forceinline__ void close(const Epilogue& E) {
    if (!there) return;
    float a, b;
    apart(s, a, b);
    static_cast<float2*>(E.partial)[(long long)slot * E.ld_partial + row] = make_float2(m, a + b);
  }
};

// 8 bf16 a register quad; a strip's rows follow one another in memory.
template <int N> __device__ __forceinline__ void store_rows(__nv_bfloat16* to, const float (&v)[N]) {
  uint32_t u[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) u[i] = pair_bf16(two(v[2 * i], v[2 * i + 1]));
#pragma unroll
  for (int i = 0; i < N / 2; i += 8) {
    if constexpr (N >= 16)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 2 * i), "r"(u[i]), "r"(u[i + 1]), "r"(u[i + 2]),
                   "r"(u[i + 3]), "r"(u[i + 4]), "r"(u[i + 5]), "r"(u[i + 6]), "r"(u[i + 7])
                   : "memory");
    else
      *reinterpret_cast<uint4*>(to) = make_uint4(u[0], u[1], u[2], u[3]);
  }
}

// d is stored with the rows of the batch along memory ([words][rows]): a lane holds a word and has a strip of its
// rows in one piece.  32 words of 32 rows (of each part) go through shared memory and leave by the copy engine: 32 stores
// to 32 lines each would keep the load-store unit longer than the tile's product takes (1,024 x 512 x 18,944 bf16: 24.9
// us, without any stores 19.8).  The 64-byte swizzle keeps a warp's 16-byte stores off the same banks.
template <typename T, typename TO, int N> struct Finisher<kLossGrad, T, TO, N> {
  float column;              // sum over the strip's rows
  // N 32: tensor map of d's parts, boxes of 32 rows x 32 words of one.  bf16: the half of 4 KB of shared memory that comes
  // next, and what turns it into the other one; what went out of a half two stores ago has been read.  fp32: 2 KB (and
  // half 0), which the store before has left: three parts of both operands need the room for stages of the ring (1,003 x
  // 515 x 10,007 on single CTAs: 85 -> 74 us).
  const CUtensorMap* map;
  uint32_t room, half;

  __device__ __forceinline__ void ask(const Epilogue&, int, int, int, int, int) {}
  __device__ __forceinline__ void finish(const Epilogue& E, int r, int c, int R, int, int lane, float bias, float (&v)[N]) {
    constexpr bool FAST = sizeof(T) == 2;
    const ulonglong2* const rows = static_cast<const ulonglong2*>(E.loss_rows) + r / 2;
    const int t = lane < N ? E.loss_targets[r + lane] : -1;
    Two sum = two(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const ulonglong2 pair = rows[i / 2];
      const Two z = two(v[i], v[i + 1]) + two(bias, bias), m{pair.x}, k{pair.y};
      const Two d = exp_of<FAST>(z + m) * k;
      sum = sum + d;
      apart(d, v[i], v[i + 1]);
    }
    float s0, s1;
    apart(sum, s0, s1);
    column = s0 + s1;
    // rows whose target is among the warp's words: few
    const unsigned hit = __ballot_sync(~0u, (unsigned)(t - E.first_word - (c - lane)) < 32u && t >= 0);
    if (hit) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (hit >> i & 1) {
          const float w = __shfl_sync(~0u, t, i) == c + E.first_word ? E.loss_weights[r + i] : 0.0f;
          v[i] -= w;
          column -= w;
        }
    }
    // rows without a gradient have k = 0: only what is not finite is left to be cleared
    if (!(fabsf(column) <= 3.4e38f)) {
      column = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (E.loss_targets[r + i] == -2) v[i] = 0.0f;
        column += v[i];
      }
    }
    if (FAST && r + N > E.rest_from) {
      column = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (r + i < E.rest_from) column += v[i];
        else v[i] -= __bfloat162float(__float2bfloat16_rn(v[i]));
      }
    }
    if constexpr (N == 32) {
      constexpr int PARTS = FAST ? 1 : 3;
      const bool there = r < R && c - lane < E.words;
      Two rest[N / 2];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) rest[i] = two(v[2 * i], v[2 * i + 1]);
#pragma unroll
      for (int q = 0; q < PARTS; ++q, room ^= half) {
        if (!there) {                                      // a group all the same, for the count of two
          if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          continue;
        }
        if (lane == 0) {
          if (FAST) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        }
        __syncwarp();
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          uint32_t u[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u[i] = pair_bf16(rest[4 * p + i]);
            if (q + 1 < PARTS) rest[4 * p + i] = rest[4 * p + i] - pair_f32(u[i]);
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(room + 64u * lane + 16u * (p ^ (lane >> 1 & 3))), "r"(u[0]), "r"(u[1]),
                       "r"(u[2]), "r"(u[3])
                       : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(reinterpret_cast<uint64_t>(map)),
                       "r"(r), "r"(c), "r"(q), "r"(room)
                       : "memory");
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      }
      return;
    }
    if (c >= E.words || r >= R) return;                    // a strip that holds a row at all is stored whole
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(E.out0) + (long long)c * E.ld_out0 + r;
    if constexpr (FAST) {
      store_rows(out, v);
    } else {
      float part[N];
#pragma unroll
      for (int q = 0; q < 3; ++q, out += E.part) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          part[i] = __bfloat162float(__float2bfloat16_rn(v[i]));
          v[i] -= part[i];
        }
        store_rows(out, part);
      }
    }
  }
};

// A term of dx: the sum over one piece's words, or over one of `slices` parts of them (each sums into an array of its
// own, so that a result of few tiles keeps all SMs busy; the arrays are added up at the end).  What an array holds of
// the pieces before is where the sums begin: its loads are under way while the first products are formed.
template <typename T, typename TO, int N> struct Finisher<kLossTerm, T, TO, N> {
  int slice;

  __device__ __forceinline__ TO* base(const Epilogue& E) const { return static_cast<TO*>(E.out0) + slice * E.part; }
  __device__ __forceinline__ void begin(const Epilogue& E, int r, int c, int R, int C, int lane, float (&v)[N]) {
    Strip<TO, N> old;
    if (r + N <= R && c - lane + 32 <= C) old.template load<true>(base(E), E.ld_out0, r, c, R, C, false, lane);
    else old.template load<false>(base(E), E.ld_out0, r, c, R, C, false, lane);
    old.unpack(v, false, lane);
  }
  __device__ __forceinline__ void ask(const Epilogue&, int, int, int, int, int) {}
  __device__ __forceinline__ void finish(const Epilogue& E, int r, int c, int R, int C, int lane, float, float (&v)[N]) {
    if (r + N <= R && c - lane + 32 <= C) store_strip<TO, true>(v, base(E), E.ld_out0, r, c, R, C, false, lane);
    else store_strip<TO, false>(v, base(E), E.ld_out0, r, c, R, C, false, lane);
  }
};
template <typename T>
__global__ void __launch_bounds__(256) loss_dx_kernel(const float* terms, long long ld, long long slice, int slices, T* dx, long long ld_dx,
                                                      long long rows, int cols, float scale, const float* factor, bool twice) {
  grid_launch_dependents();
  grid_dependency_wait();
  const float f = factor ? *factor : 1.0f;
  for (long long row = blockIdx.x; row < rows; row += gridDim.x)
    for (int c = threadIdx.x; c < cols; c += 256) {
      const float* p = terms + row * ld + c;
      float s = *p;
#pragma unroll 4
      for (int i = 1; i < slices; ++i) s += p[i * slice];
      if (twice)
        for (int i = 0; i < slices; ++i) s += p[i * slice + rows * ld];
      dx[row * ld_dx + c] = from_f32<T>(s * f * scale);
    }
}

// Joins the statistics of a row's slots, in their order: loss, lse, and what kLossGrad needs (rows past the
// last get a zero gradient).  32 rows by 16 shares of the slots per block.
constexpr int kJoinShares = 16;
struct JoinParams {
  LossParams L;
  const float2* slots;
  const float* target_logit;
  RowPair* pairs;            // or NULL
  int* targets;
  float* weights;
  const float* weight_max;   // or NULL: the largest weights of `groups` groups of rows, all of the batch
  float* factor;             // the largest of them
  long long ld, rows_padded, groups;
  int count, twice;          // twice: the gradients have the rows a second time
};
__device__ __forceinline__ void join_stats(float& m, float& s, float2 o) {
  const float top = fmaxf(m, o.x);
  if (top == -INFINITY) { s += o.y; return; }              // sums are 0 or NaN
  s = (m == -INFINITY ? s : s * expf(m - top)) + (o.x == -INFINITY ? o.y : o.y * expf(o.x - top));
  m = top;
}
__global__ void __launch_bounds__(32 * kJoinShares) loss_join_kernel(const JoinParams P) {
  __shared__ float2 part[kJoinShares][32];
  __shared__ float largest[kJoinShares];
  grid_launch_dependents();
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, share = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * 32 + lane;
  float m = -INFINITY, s = 0.0f;
  if (row < P.L.rows) {
    // the maximum first: neither loop's loads and exponentials wait for one another
#pragma unroll 8
    for (int i = share; i < P.count; i += kJoinShares) m = fmaxf(m, P.slots[i * P.ld + row].x);
#pragma unroll 8
    for (int i = share; i < P.count; i += kJoinShares) {
      const float2 o = P.slots[i * P.ld + row];
      s += o.x == -INFINITY ? o.y : o.y * expf(o.x - m);
    }
  }
  part[share][lane] = make_float2(m, s);
  float factor = 0.0f;
  if (P.weight_max) {
    for (long long i = threadIdx.x; i < P.groups; i += 32 * kJoinShares) factor = fmaxf(factor, P.weight_max[i]);
    for (int d = 16; d > 0; d >>= 1) factor = fmaxf(factor, __shfl_xor_sync(~0u, factor, d));
    if (lane == 0) largest[share] = factor;
  }
  __syncthreads();
  if (P.weight_max) {
    factor = largest[lane % kJoinShares];
    for (int d = kJoinShares / 2; d > 0; d >>= 1) factor = fmaxf(factor, __shfl_xor_sync(~0u, factor, d));
  }
  if (factor == 0.0f) factor = 1.0f;                       // no weights, or no row counts
  if (P.weight_max && blockIdx.x == 0 && threadIdx.x == 0) *P.factor = factor;
  if (share != 0 || row >= P.rows_padded) return;
  float offset = 0.0f, k = 0.0f, weight = 0.0f;
  int target = -2;
  if (row < P.L.rows) {
    for (int i = 1; i < kJoinShares; ++i) join_stats(m, s, part[i][lane]);
    const long long t = P.L.targets[row];
    const float own = P.L.row_weight ? P.L.row_weight[row] : 1.0f, w = P.L.scale * own;
    const float x = target_inside(P.L, t) ? P.target_logit[row] : 0.0f;
    const RowOutcome o = row_outcome(P.L, m, s, x, t, w);
    report_target(P.L, t, w);
    if (P.L.loss) P.L.loss[row] = o.loss;
    if (P.L.lse) P.L.lse[row] = o.lse;
    if (!o.zero) {
      offset = m == -INFINITY ? 0.0f : -m;
      weight = own / factor;
      k = weight / s;
      target = (int)t;
    }
  }
  if (!P.pairs) return;
  const bool again = P.twice && row < P.L.rows;
  if (P.twice && !again && row < 2 * P.L.rows) return;     // its first time's thread has it
  for (long long at = row; at <= row + (again ? P.L.rows : 0); at += P.L.rows) {
    P.pairs[at / 2].m[at & 1] = offset;
    P.pairs[at / 2].k[at & 1] = k;
    P.targets[at] = target;
    P.weights[at] = weight;
  }
}

// The largest of the rows' weights, where every block of the join would read more than kLossMostGroups of them: into the first.
constexpr long long kLossMostGroups = 4096;
__global__ void __launch_bounds__(1024) loss_max_kernel(float* weight_max, long long groups) {
  __shared__ float largest[32];
  grid_launch_dependents();
  grid_dependency_wait();
  float top = 0.0f;
#pragma unroll 8
  for (long long i = threadIdx.x; i < groups; i += 1024) top = fmaxf(top, weight_max[i]);
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  if ((threadIdx.x & 31) == 0) largest[threadIdx.x >> 5] = top;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  top = largest[threadIdx.x];
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  if (threadIdx.x == 0) weight_max[0] = top;
}

// dbias of a piece: the strips' sums in their order.
template <typename TO>
__global__ void __launch_bounds__(256) loss_bias_kernel(const float* partial, long long ld, int strips, long long words, TO* out,
                                                        int accumulate, float scale, const float* factor) {
  grid_launch_dependents();
  grid_dependency_wait();
  const long long c = (long long)blockIdx.x * 256 + threadIdx.x;
  if (c >= words) return;
  float t = 0.0f;
#pragma unroll 8
  for (int i = 0; i < strips; ++i) t += partial[i * ld + c];
  t = t * (factor ? *factor : 1.0f) * scale;
  out[c] = from_f32<TO>(accumulate ? t + to_f32(out[c]) : t);
}

}  // namespace

#endif  // GBMUF_CSRC_LINEAR_LOSS_CUH
