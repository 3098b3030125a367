// Distillation: the loss of a student's logits against a teacher's largest ones, with its gradient.
// Part of libgbmuf (CUDA, sm_100a); included by vocab_ops.cu.
#ifndef GBMUF_CSRC_DISTILL_CUH
#define GBMUF_CSRC_DISTILL_CUH

namespace {

// Per row, with p = softmax(x / T) and the teacher's probabilities q_j at words v_j (their sum at a word: Q_v):
//   soft = T^2 (sum_j q_j (log q_j - log p_vj) + q_r log (q_r / P_r)),  hard = log sum exp(x) - x_t
//   loss = w ((1 - h) soft + h hard)
// with q_r = 1 - sum q and P_r the student's probability of all words outside the list, or q_r = 0.  With
// M = sum q + q_r the gradient is T (M p_v - Q_v) at the list's words, T p_v (M - q_r / P_r) at the others.
// P_r and 1 - sum of the list's p differ by everything where the student is sure, so the list's words are left
// out of the running sum and counted by themselves: the statistics are those of "the rest" (maximum m_r,
// sum R relative to it) and of the list (m_s, S).
//
// A row's list is prepared by one warp, a row ahead of the others: probabilities, the student's logits at
// the words, sums; and for every worker thread a chain of the entries in the pieces that this thread goes
// through.  A thread looks at its next entry's place once per chunk.  The order within a chain depends on
// timing, the results do not: a word's Q is summed in the list's order.
//
// Measured: 2,048 x 267,735 bf16, lists of 64: 452 to 504 us (4.4 to 4.9 TB/s of the bytes that have to move, 67 to 74 % of
// the copy rate; the cross-entropy without lists 417 to 463), the loss alone 226 to 300; 480 to 510 with hard targets at
// T = 2 or 3, 680 at T = 1.5; 1,003 x 33,278 fp32 at T = 3 with hard targets 76 us (the cross-entropy 58): issue slots
// 58 % busy with the exact exponentials, whose latency 19 warps an SM do not cover.
struct DistillParams {
  const void* logits;
  const void* teacher;
  const long long* index;
  const float* teacher_lse;
  const long long* targets;
  const float* row_weight;
  float *loss, *lse;
  void* dlogits;
  long long rows, vocab, ld, ld_d, ld_teacher, ld_index, ignore_index;
  int k, split, teacher_bf16;
  float T, hard, scale;
  Temperature temperature;
  int32_t* status;
};
constexpr int kListMost = 256;                 // entries
constexpr int kListHeads = kLossWorkers;

struct RowList {
  int word[kListMost];       // -1: not there, or the word has an earlier entry
  float q[kListMost];        // Q of the word
  float x[kListMost];        // the student's logit
  short next[kListMost];     // of the chain, -1: end
  int head[kListHeads];
  // sums: q (log q - (x - m) / T); q; and of the student's exponentials, at T and at 1, relative to m
  double gap;
  float q_sum, m, s, s1, q_rest, target_logit, weight;
  int target;                // -1: none
  bool outside, ignored, target_listed;
};

__device__ __forceinline__ float warp_sum(float v) {
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
  for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, d));
  return v;
}

// What a lane needs of a row's list from memory (LANES entries of it): asked for two rows ahead, the student's
// logits at its words one row ahead.
template <typename T, int LANES> struct ListAhead {
  float t[LANES], x[LANES];
  long long word[LANES], target;
  float weight, lse, target_logit;

  __device__ __forceinline__ bool inside(const DistillParams& P, long long v) const { return v >= 0 && v < P.vocab; }
  __device__ __forceinline__ void ask(const DistillParams& P, long long row, int lane) {
    if (row >= P.rows) return;
#pragma unroll
    for (int i = 0; i < LANES; ++i) {
      const int j = lane + 32 * i;
      t[i] = -INFINITY;
      word[i] = -1;
      if (j >= P.k) continue;
      t[i] = P.teacher_bf16 ? to_f32(static_cast<const __nv_bfloat16*>(P.teacher)[row * P.ld_teacher + j])
                            : static_cast<const float*>(P.teacher)[row * P.ld_teacher + j];
      word[i] = P.index[row * P.ld_index + j];
    }
    target = P.targets ? P.targets[row] : -1;
    weight = P.row_weight ? P.row_weight[row] : 1.0f;
    lse = P.teacher_lse ? P.teacher_lse[row] : 0.0f;
  }
  __device__ __forceinline__ void ask_student(const DistillParams& P, long long row) {
    if (row >= P.rows) return;
    const T* const student = static_cast<const T*>(P.logits) + row * P.ld;
#pragma unroll
    for (int i = 0; i < LANES; ++i) x[i] = inside(P, word[i]) ? to_f32(student[word[i]]) : -INFINITY;
    target_logit = inside(P, target) ? to_f32(student[target]) : 0.0f;
  }
};

// Fills a row's list from what has been asked for; all lanes of one warp.  owner(word): the worker thread whose pieces
// hold a word.
template <typename T, int LANES, typename Owner>
__device__ __forceinline__ void prepare_list(const DistillParams& P, RowList& L, int lane, Owner owner, const ListAhead<T, LANES>& from) {
  constexpr bool FAST = false;
  for (int i = lane; i < kListHeads; i += 32) L.head[i] = -1;
  long long word[LANES];
  double a[LANES];
  float xs[LANES], largest = -INFINITY;
  bool outside = false, target_listed = false;
#pragma unroll
  for (int i = 0; i < LANES; ++i) {
    const float t = from.t[i];
    const long long v = from.word[i];
    word[i] = -1;
    a[i] = -INFINITY;
    xs[i] = -INFINITY;
    if (v == -1 || t == -INFINITY) continue;               // no entry
    if (v < 0 || v >= P.vocab) { outside = true; continue; }
    word[i] = v;
    target_listed |= v == from.target;
    xs[i] = from.x[i];
    a[i] = (double)t * P.temperature.inverse;
    largest = fmaxf(largest, (float)a[i]);
  }
  const long long target = from.target;
  const bool inside = from.inside(P, target);
  const float w = P.scale * from.weight, target_logit = from.target_logit, teacher_lse = from.lse;
  // log of the probabilities' common divisor
  double A;
  if (P.teacher_lse) {
    A = (double)teacher_lse;
  } else {
    largest = warp_max(largest);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < LANES; ++i)
      if (word[i] >= 0) s += expf((float)(a[i] - (double)largest));
    A = (double)largest + log_of(warp_sum(s));
  }
  float q[LANES], m = -INFINITY;
  double q_sum = 0.0;
#pragma unroll
  for (int i = 0; i < LANES; ++i) {
    a[i] -= A;                                             // log q
    q[i] = word[i] >= 0 ? expf((float)a[i]) : 0.0f;
    q_sum += (double)q[i];
    m = fmaxf(m, xs[i]);
  }
  for (int d = 16; d > 0; d >>= 1) q_sum += __shfl_xor_sync(~0u, q_sum, d);
  m = warp_max(m);
  __syncwarp();                                            // heads are clear
#pragma unroll
  for (int i = 0; i < LANES; ++i) {
    const int j = lane + 32 * i;
    if (j >= P.k) continue;
    L.word[j] = (int)word[i];
    L.q[j] = q[i];
    L.x[j] = xs[i];
    L.next[j] = word[i] >= 0 ? (short)atomicExch(&L.head[owner((int)word[i])], j) : (short)-1;
  }
  __syncwarp();
  // entries of the same word: the first one stands for all, with the sum of their q in the list's order
  bool first[LANES];
  float total[LANES];
#pragma unroll
  for (int i = 0; i < LANES; ++i) {
    const int j = lane + 32 * i;
    first[i] = word[i] >= 0;
    total[i] = q[i];
    if (word[i] < 0) continue;
    int after = kListMost;                                 // the next entry of this word
    for (int o = L.head[owner((int)word[i])]; o >= 0; o = L.next[o]) {
      if (o == j || L.word[o] != (int)word[i]) continue;
      if (o < j) first[i] = false; else after = min(after, o);
    }
    while (first[i] && after < kListMost) {
      total[i] += L.q[after];
      int further = kListMost;
      for (int o = L.head[owner((int)word[i])]; o >= 0; o = L.next[o])
        if (o > after && L.word[o] == (int)word[i]) further = min(further, o);
      after = further;
    }
  }
  __syncwarp();
  TemperedShift<FAST> e;
  Shift<FAST> e1;
  e.at(P.temperature);
  e.set(m);
  e1.set(m);
  float s = 0.0f, s1 = 0.0f;
  double gap = 0.0;
  int words = 0;
#pragma unroll
  for (int i = 0; i < LANES; ++i) {
    const int j = lane + 32 * i;
    if (word[i] >= 0) {
      if (q[i] != 0.0f) gap += (double)q[i] * (a[i] - (double)(xs[i] - e.m) * P.temperature.inverse);
      if (first[i]) {
        s += e(xs[i]);
        s1 += e1(xs[i]);
        ++words;
        L.q[j] = total[i];
      } else {
        L.word[j] = -1;
      }
    }
  }
  s = warp_sum(s);
  s1 = warp_sum(s1);
  for (int d = 16; d > 0; d >>= 1) gap += __shfl_xor_sync(~0u, gap, d);
  words = __reduce_add_sync(~0u, words);
  outside = __any_sync(~0u, outside);
  target_listed = __any_sync(~0u, target_listed);
  if (lane == 0) {
    const bool ignored = w == 0.0f || (P.targets && target == P.ignore_index);
    if (P.targets && !inside) outside = true;
    if (P.teacher_lse && teacher_lse != teacher_lse) q_sum = (double)teacher_lse;      // of a list without entries too
    L.gap = gap; L.m = m; L.s = s; L.s1 = s1;
    L.q_sum = (float)q_sum;
    const double rest = 1.0 - q_sum;
    L.q_rest = P.teacher_lse && words < P.vocab ? (rest < 0.0 ? 0.0f : (float)rest) : 0.0f;
    L.target = inside ? (int)target : -1;
    L.target_logit = target_logit;
    L.weight = w;
    L.outside = outside && !ignored;
    L.ignored = ignored;
    L.target_listed = target_listed;
  }
  __syncwarp();
}

// What a row's statistics and its list say.  (m, r, r1): maximum of the rest, its sums at T and at 1.
struct DistillRow {
  bool empty, zero;          // nothing but -inf; no gradient
  float k, k1;               // the gradient of a word of the rest is k exp((x - m) / T) + k1 exp(x - m)
  float top, per, per1;      // of a word of the list: per exp((x - top) / T) + per1 exp(x - top) - soft Q - hard [target]
  float soft, hard;
  float z, z1, share;        // sums of all words relative to top; P_r
};
__device__ __forceinline__ DistillRow distill_row(const DistillParams& P, const RowList& L, float m, float r, float r1) {
  DistillRow o;
  TemperedShift<false> e;
  Shift<false> e1;
  e.at(P.temperature);
  const float top = fmaxf(m, L.m);
  const bool one = P.T == 1.0f;
  e.set(top);
  e1.set(top);
  const float fr = m == -INFINITY ? 1.0f : e(m), fs = L.m == -INFINITY ? 1.0f : e(L.m);
  const float fr1 = m == -INFINITY ? 1.0f : e1(m), fs1 = L.m == -INFINITY ? 1.0f : e1(L.m);
  o.empty = top == -INFINITY && r + L.s == 0.0f;
  o.zero = L.ignored || L.outside || o.empty;
  o.z = r * fr + L.s * fs;
  o.z1 = one ? o.z : r1 * fr1 + L.s1 * fs1;
  o.share = r * fr / o.z;
  const float h = P.hard, mass = L.q_sum + L.q_rest, ws = L.weight * (1.0f - h) * P.T, wh = L.weight * h;
  o.per = ws * mass / o.z;
  o.k = r == 0.0f ? 0.0f * o.per : ws * (mass * o.share - L.q_rest) / r;      // NaN stays, where no word of the rest can occur
  o.k1 = h == 0.0f || (one ? r : r1) == 0.0f ? 0.0f : wh * fr1 / o.z1;
  o.per1 = h == 0.0f ? 0.0f : wh / o.z1;
  if (one) { o.k += o.k1; o.per += o.per1; o.k1 = o.per1 = 0.0f; }
  o.top = e.m;
  o.soft = ws;
  o.hard = wh;
  return o;
}
// (lse, loss).  In 64 bits past the sums: log z may be many times the loss.
__device__ __noinline__ float2 distill_loss(const DistillParams& P, const RowList& L, const DistillRow o, float m, float r) {
  const bool empty = o.empty, one = P.T == 1.0f;
  const double inverse = P.temperature.inverse, log_z = log_of(o.z);
  const float lse = empty ? -INFINITY : (float)((double)o.top * inverse + log_z);
  // sum q (log q - log p): log p = (x - m_s) / T + (m_s - top) / T - log z
  const double shift_s = L.m == -INFINITY ? 0.0 : (double)(L.m - o.top) * inverse;
  double soft = L.q_sum == 0.0f ? 0.0 : L.gap - (double)L.q_sum * (shift_s - log_z);
  if (L.q_rest != 0.0f)
    soft += (double)L.q_rest * (o.share > 1e-30f ? (double)logf(L.q_rest / o.share)
                                                 : (double)logf(L.q_rest) - (log_of(r) + (m == -INFINITY ? 0.0 : (double)(m - o.top) * inverse) - log_z));
  double loss = 0.0;
  if (P.hard != 1.0f) loss += (1.0 - (double)P.hard) * (double)(P.T * P.T) * soft;
  if (!(o.z == o.z && L.q_sum == L.q_sum)) loss = (double)(o.z + L.q_sum);     // NaN, where its factor is 0 too
  if (P.hard != 0.0f) loss += (double)P.hard * ((double)(o.top - L.target_logit) + (one ? log_z : log_of(o.z1)));
  return make_float2(lse, L.ignored ? 0.0f : L.outside ? NAN : empty ? INFINITY : (float)((double)L.weight * loss));
}
struct DistillEnd { DistillRow o; float m, r; };           // what the loss needs besides the list
__device__ __forceinline__ void store_loss(const DistillParams& P, const RowList& L, const DistillRow& o, float m, float r, long long row) {
  if (L.outside) atomicExch(P.status, (int32_t)GBMUF_ERR_INVALID_ARG);
  const float2 v = distill_loss(P, L, o, m, r);
  if (P.lse) P.lse[row] = v.x;
  if (P.loss) P.loss[row] = v.y;
}
__device__ __forceinline__ float listed_gradient(const DistillParams& P, const DistillRow& o, float x, float q, bool is_target) {
  TemperedShift<false> e;
  Shift<false> e1;
  e.at(P.temperature);
  e.m = e1.m = o.top;
  float g = o.per * e(x) - o.soft * q;
  if (o.per1 != 0.0f) g += o.per1 * e1(x);
  return is_target ? g - o.hard : g;
}

// ---- short rows: one warp per row, up to 32 * REGS logits in its registers
template <typename T, int REGS, int LANES>
__global__ void __launch_bounds__(128) distill_warp_kernel(const DistillParams P) {
  constexpr bool FAST = sizeof(T) == 2;
  __shared__ RowList lists[4];
  __shared__ uint32_t listed[4][REGS];
  grid_launch_dependents();
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * 4 + warp;
  if (row >= P.rows) return;
  RowList& L = lists[warp];
  const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
  const int V = (int)P.vocab;
  float v[REGS];
  ListAhead<T, LANES> ahead;
  ahead.ask(P, row, lane);
#pragma unroll
  for (int i = 0; i < REGS; ++i) v[i] = lane + 32 * i < V ? to_f32(x[lane + 32 * i]) : -INFINITY;
  for (int i = lane; i < REGS; i += 32) listed[warp][i] = 0;
  ahead.ask_student(P, row);
  prepare_list(P, L, lane, [](int word) { return word % kListHeads; }, ahead);
  for (int j = lane; j < P.k; j += 32)
    if (L.word[j] >= 0) atomicOr(&listed[warp][L.word[j] >> 5], 1u << (L.word[j] & 31));
  __syncwarp();
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < REGS; ++i) {
    const bool is = listed[warp][i] >> lane & 1;
    m = is ? m : fmaxf(m, v[i]);
  }
  m = warp_max(m);
  TemperedShift<FAST> e;
  Shift<FAST> e1;
  e.at(P.temperature);
  e.set(m);
  e1.set(m);
  const bool two_sums = P.hard != 0.0f && P.T != 1.0f;
  float r = 0.0f, r1 = 0.0f;
#pragma unroll
  for (int i = 0; i < REGS; ++i) {
    const bool is = listed[warp][i] >> lane & 1;
    if (!is) r += e(v[i]);
    if (two_sums && !is) r1 += e1(v[i]);
  }
  r = warp_sum(r);
  r1 = warp_sum(r1);
  const DistillRow o = distill_row(P, L, m, r, r1);
  if (!P.dlogits) {
    if (lane == 0) store_loss(P, L, o, m, r, row);
    return;
  }
  T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
#pragma unroll
  for (int i = 0; i < REGS; ++i) {
    const int c = lane + 32 * i;
    float g = e(v[i]) * o.k;
    if (two_sums) g += e1(v[i]) * o.k1;
    if (c == L.target && o.hard != 0.0f) g -= o.hard;
    if (c < V) d[c] = from_f32<T>(o.zero ? 0.0f : g);
  }
  __syncwarp();
  if (!o.zero)
    for (int j = lane; j < P.k; j += 32)
      if (L.word[j] >= 0) d[L.word[j]] = from_f32<T>(listed_gradient(P, o, L.x[j], L.q[j], L.word[j] == L.target));
  if (lane == 0) store_loss(P, L, o, m, r, row);
}

// ---- longer rows: as the cross-entropy's (a cluster per row, chunks through a ring of slots, the last ones kept
// and the others fetched again for the gradient), with the list's warp beside the producer.
constexpr int kDistillThreads = kLossWorkers + 64;
constexpr uint32_t kDistillLists = 768;
static_assert(576 + 2 * sizeof(DistillEnd) <= kDistillLists, "");
constexpr uint32_t kDistillHead = (kDistillLists + 2u * (uint32_t)sizeof(RowList) + 127u) / 128u * 128u;
constexpr uint32_t kDistillSmem = kDistillHead + kLossRing * kLossChunk;

// A piece with element `at` taken out (set to -inf).
template <typename T> __device__ __forceinline__ void take_out(uint4& u, int at) {
  uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) w[i] = at == i ? 0xff800000u : w[i];
    else w[i] = at >> 1 != i ? w[i] : at & 1 ? (w[i] & 0xffffu) | 0xff800000u : (w[i] & 0xffff0000u) | 0xff80u;
  }
  u = make_uint4(w[0], w[1], w[2], w[3]);
}

// MODE 0: one exponential per logit.  Else the hard targets' softmax is another one (T is not 1): 1, with exponentials of
// its own; 2, 3 and 4, where that is T: exp(x) = exp(x / T)^T, two multiplications at most (each 2^-24) in place of
// an exponential (1,003 x 33,278 fp32 at T = 3: 89 -> 77 us).
template <typename T, int MODE, int LANES>
__global__ void __launch_bounds__(kDistillThreads, kLossBlocksPerSm) distill_ring_kernel(const DistillParams P) {
  constexpr bool FAST = sizeof(T) == 2, TWO = MODE != 0;
  constexpr int E = 16 / (int)sizeof(T);
  constexpr int CHUNK = kLossChunk / (int)sizeof(T);               // elements
  extern __shared__ __align__(128) unsigned char smem[];
  const uint32_t bars = smem_u32(smem), ring = bars + kDistillHead;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 64u + 8u * s; };
  auto heard = [&](int b) { return bars + 128u + 8u * b; };
  auto list_full = [&](int b) { return bars + 144u + 8u * b; };
  auto list_empty = [&](int b) { return bars + 160u + 8u * b; };
  float4* const told = reinterpret_cast<float4*>(smem + 192);          // [2][8]: statistics of the ranks
  float4* const warp_stat = reinterpret_cast<float4*>(smem + 448);     // [8]
  DistillEnd* const outcome = reinterpret_cast<DistillEnd*>(smem + 576);       // [2]
  RowList* const lists = reinterpret_cast<RowList*>(smem + kDistillLists);
  const int rank = P.split > 1 ? (int)(blockIdx.x % (unsigned)P.split) : 0;
  const long long first = blockIdx.x / (unsigned)P.split, step = gridDim.x / (unsigned)P.split;
  const int thread = threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (thread == 0) {
    for (int s = 0; s < kLossRing; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), kLossWarps); }
    for (int b = 0; b < 2; ++b) { mbar_init(heard(b), 1); mbar_init(list_full(b), 1); mbar_init(list_empty(b), kLossWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (P.split > 1) cluster_sync();                         // barriers exist before a peer uses them
  grid_launch_dependents();
  grid_dependency_wait();

  // the worker thread that goes through an element's piece, or holds it as one outside the whole pieces
  auto owner_of = [](const RowSpan& r, int word) {
    const int at = word - r.a0;
    if (at < 0) return word;
    if (at >= r.pieces * E) return word - r.pieces * E;
    return (at / E - r.p0) & (kLossWorkers - 1);           // of another rank's: any, the same for a word
  };
  int slot = 0;                                            // next slot of the ring and its phase
  uint32_t phase = 0;
  auto advance = [&] { if (++slot == kLossRing) { slot = 0; phase ^= 1; } };
  if (warp == kLossWarps) {
    // ------------------------------------------------------------------ producer
    if (lane == 0) {
      int filled = 0;
      bool ok = true;
      for (long long row = first; row < P.rows && ok; row += step) {
        const RowSpan r = row_span<T>(P, row, rank);
        const char* const src = reinterpret_cast<const char*>(static_cast<const T*>(P.logits) + row * P.ld + r.a0) + 16ll * r.p0;
        const int chunks = (int)((16ll * r.n + kLossChunk - 1) / kLossChunk), again = P.dlogits ? chunks - kLossKept : 0;
        for (int i = 0; i < chunks + (again > 0 ? again : 0) && ok; ++i) {
          const int c = i < chunks ? i : again - 1 - (i - chunks);
          if (filled == kLossRing) ok = mbar_wait_bounded(empty(slot), phase ^ 1, P.status);
          else ++filled;
          if (!ok) break;
          const long long left = 16ll * r.n - (long long)c * kLossChunk;
          const uint32_t bytes = left < kLossChunk ? (uint32_t)left : (uint32_t)kLossChunk;
          mbar_arrive_expect_tx(full(slot), bytes);
          bulk_load_hint(ring + slot * kLossChunk, src + (long long)c * kLossChunk, bytes, full(slot), c < again && i < chunks);
          advance();
        }
      }
      if (!ok)                                             // copies requested into this CTA's memory land first
        for (int j = 0; j < kLossRing; ++j) { mbar_wait_bounded(full(slot), phase ^ 1, P.status); advance(); }
    }
    __syncwarp();
  } else if (warp > kLossWarps) {
    // ------------------------------------------------------------------ lists; what is left to do of rows behind the workers
    int turn = 0;
    bool ok = true;
    ListAhead<T, LANES> now, ahead;
    now.ask(P, first, lane);
    now.ask_student(P, first);
    ahead.ask(P, first + step, lane);
    // The row of turn t, once the workers have stored its gradient and left its list: the list's words and the
    // target are stored once more, and the loss is formed (its 64-bit logarithms would hold the workers up).
    auto finish = [&](long long row, int t) {
      ok = ok && mbar_wait_bounded(list_empty(t & 1), t >> 1 & 1, P.status);
      ok = __all_sync(~0u, ok);
      if (!ok) return;
      const RowList& L = lists[t & 1];
      const DistillEnd& end = outcome[t & 1];
      if (P.dlogits && !end.o.zero) {
        const RowSpan r = row_span<T>(P, row, rank);
        T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
        const int slice = r.a0 + r.p0 * E, length = r.n * E;
        auto mine = [&](int word) {
          const bool edge = word < r.a0 || word >= r.a0 + r.pieces * E;
          return edge ? rank == 0 : word >= slice && word - slice < length;
        };
        for (int j = lane; j < P.k; j += 32)
          if (L.word[j] >= 0 && mine(L.word[j]))
            d[L.word[j]] = from_f32<T>(listed_gradient(P, end.o, L.x[j], L.q[j], L.word[j] == L.target));
        if (lane == 0 && end.o.hard != 0.0f && L.target >= 0 && !L.target_listed && mine(L.target)) {
          TemperedShift<FAST> e;
          Shift<FAST> e1;
          e.at(P.temperature);
          e.set(end.m);
          e1.set(end.m);
          const float x = L.target_logit;
          d[L.target] = from_f32<T>((TWO ? e(x) * end.o.k + e1(x) * end.o.k1 : e(x) * end.o.k) - end.o.hard);
        }
      }
      if (lane == 0 && rank == 0) store_loss(P, L, end.o, end.m, end.r, row);
      __syncwarp();
    };
    for (long long row = first; row < P.rows; row += step, ++turn) {
      const int b = turn & 1;
      if (turn >= 2) finish(row - 2 * step, turn - 2);
      if (!ok) break;
      const RowSpan r = row_span<T>(P, row, rank);
      ahead.ask_student(P, row + step);
      prepare_list(P, lists[b], lane, [&](int word) { return owner_of(r, word); }, now);
      if (lane == 0) mbar_arrive(list_full(b));
      now = ahead;
      ahead.ask(P, row + 2 * step, lane);
    }
    for (int t = turn > 2 ? turn - 2 : 0; t < turn && ok; ++t) finish(first + t * step, t);
  } else {
    // ------------------------------------------------------------------ 8 worker warps
    bool ok = true;
    int turn = 0;
    for (long long row = first; row < P.rows; row += step, ++turn) {
      const RowSpan r = row_span<T>(P, row, rank);
      const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
      const int chunks = (r.n + kLossPieces * kLossWorkers - 1) / (kLossPieces * kLossWorkers);
      const int again = P.dlogits && chunks > kLossKept ? chunks - kLossKept : 0;      // chunks that are fetched twice
      auto left_in = [&](int c) { return r.n - c * kLossPieces * kLossWorkers - thread; };
      auto pieces_in = [&](int s) { return reinterpret_cast<const uint4*>(smem + kDistillHead + s * kLossChunk) + thread; };
      auto release = [&](int s) {
        __syncwarp();                                      // one arrival per warp: they are serialised
        if (lane == 0) mbar_arrive(empty(s));
      };
      // the elements before and after the whole pieces: one thread of rank 0 each
      float own = -INFINITY;
      int own_at = -1;
      if (rank == 0 && thread < 2 * E) {
        const int at = thread < r.a0 ? thread : r.pieces * E + thread;
        if (at < (int)P.vocab) { own_at = at; own = to_f32(x[at]); }
      }
      const int b = turn & 1;
      ok = ok && mbar_wait_bounded(list_full(b), turn >> 1 & 1, P.status);
      const RowList& L = lists[b];
      // this thread's next entry behind a place of the slice
      const int slice = r.a0 + r.p0 * E, length = r.n * E;
      auto next_entry = [&](int behind) {
        int best = 0x7fffffff;
        for (int j = L.head[thread]; j >= 0; j = L.next[j])
          if (L.word[j] >= slice && L.word[j] - slice < length && L.word[j] - slice > behind) best = min(best, L.word[j] - slice);
        return best;
      };
      bool own_listed = false;
      int entry = 0x7fffffff;
      if (ok) {
        if (own_at >= 0)
          for (int j = L.head[thread]; j >= 0; j = L.next[j]) own_listed |= L.word[j] == own_at;
        entry = next_entry(-1);
      }
      const float counted = own_listed ? -INFINITY : own;

      TemperedShift<FAST> e;
      Shift<FAST> e1;
      e.at(P.temperature);
      float m = counted == counted ? counted : -INFINITY;
      e.set(m);
      e1.set(m);
      // exp(x - m) beside r = exp((x - m) / T)
      auto at_one = [&](Two r, float x, float y) {
        return MODE <= 1 ? e1(x, y) : MODE == 2 ? r * r : MODE == 3 ? r * (r * r) : (r * r) * (r * r);
      };
      const float one = own_at >= 0 && counted != -INFINITY ? 1.0f + (counted - counted) : 0.0f;
      Two s01 = two(one, 0.0f), s23 = two(0.0f, 0.0f), t01 = s01, t23 = s23;
      int kept_slot = 0;                                   // slot of the first chunk that stays
      for (int c = 0; c < chunks; ++c) {
        ok = ok && mbar_wait_bounded(full(slot), phase, P.status);
        const int left = left_in(c);
        const uint4* const p = pieces_in(slot);
        if (ok && left > 0) {
          uint4 u[kLossPieces];
#pragma unroll
          for (int h = 0; h < kLossPieces; ++h) u[h] = p[h * kLossWorkers < left ? h * kLossWorkers : 0];
          while (entry < (c + 1) * CHUNK) {
            const int at = entry - c * CHUNK, mine = at / (E * kLossWorkers);
#pragma unroll
            for (int h = 0; h < kLossPieces; ++h)
              if (h == mine) take_out<T>(u[h], at % E);
            entry = next_entry(entry);
          }
          float v[E];
          float top = piece_max(u[0], v);
#pragma unroll
          for (int h = 1; h < kLossPieces; ++h)
            if (h * kLossWorkers < left) top = fmaxf(top, piece_max(u[h], v));
          if (top > m) {
            const float before = m;
            m = top;
            e.set(m);
            e1.set(m);
            if (before != -INFINITY) {                     // else the sums are 0 or NaN
              const float f = e(before);
              s01 = s01 * two(f, f);
              s23 = s23 * two(f, f);
              if (TWO) {
                const float f1 = e1(before);
                t01 = t01 * two(f1, f1);
                t23 = t23 * two(f1, f1);
              }
            }
          }
          auto add = [&](uint4 piece) {
            piece_values(piece, v);
#pragma unroll
            for (int i = 0; i < E; i += 4) {
              const Two a = e(v[i], v[i + 1]), b = e(v[i + 2], v[i + 3]);
              s01 = s01 + a;
              s23 = s23 + b;
              if (TWO) {
                t01 = t01 + at_one(a, v[i], v[i + 1]);
                t23 = t23 + at_one(b, v[i + 2], v[i + 3]);
              }
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
        if (c == again) kept_slot = slot;
        if (c < again || !P.dlogits) release(slot);
        advance();
      }
      // statistics of the warp, the CTA, the row: every thread ends with the same bits
      auto scaled = [&](float4 st, float top) {            // relative to another maximum
        e.set(top);
        e1.set(top);
        if (st.x != -INFINITY && top != -INFINITY) {
          st.y *= e(st.x);
          if (TWO) st.z *= e1(st.x);
        }
        return st;
      };
      auto join = [&](float4 st, int lanes) {
        float top = st.x;
        for (int d = lanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        st = scaled(st, top);
        for (int d = lanes / 2; d > 0; d >>= 1) {
          st.y += __shfl_xor_sync(~0u, st.y, d);
          if (TWO) st.z += __shfl_xor_sync(~0u, st.z, d);
        }
        st.x = top;
        return st;
      };
      float a0, a1, b0, b1;
      apart(s01 + s23, a0, a1);
      apart(t01 + t23, b0, b1);
      float4 st = join(make_float4(m, a0 + a1, TWO ? b0 + b1 : 0.0f, 0.0f), 32);
      if (lane == 0) warp_stat[warp] = st;
      loss_workers_sync();
      st = join(warp_stat[lane & 7], 8);
      if (P.split > 1) {
        // to every rank; two sets: a peer is one row ahead at most
        if (thread == 0) mbar_arrive_expect_tx(heard(b), 16u * P.split);
        if (thread < P.split)
          asm volatile(
              "{\n\t.reg .b32 ra, rb;\n\t"
              "mapa.shared::cluster.u32 ra, %0, %2;\n\tmapa.shared::cluster.u32 rb, %1, %2;\n\t"
              "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [ra], {%3, %4, %5, %6}, [rb];\n\t}" ::"r"(
                  smem_u32(&told[b * 8 + rank])),
              "r"(heard(b)), "r"(thread), "f"(st.x), "f"(st.y), "f"(st.z), "f"(st.w)
              : "memory");
        ok = mbar_wait_bounded(heard(b), turn >> 1 & 1, P.status) && ok;
        st = join((lane & 7) < P.split ? told[b * 8 + (lane & 7)] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f), 8);
      }
      const DistillRow o = distill_row(P, L, st.x, st.y, st.z);
      if (P.dlogits) {
        e.set(st.x);
        e1.set(st.x);
        T* const d = static_cast<T*>(P.dlogits) + row * P.ld_d;
        const bool wide = (uintptr_t)(d + r.a0) % 16 == 0;
        auto rest_gradient = [&](float y) { return TWO ? e(y) * o.k + e1(y) * o.k1 : e(y) * o.k; };
        if (own_at >= 0) d[own_at] = from_f32<T>(o.zero ? 0.0f : rest_gradient(own));
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
              for (int j = 0; j < E; j += 2) {
                const Two r = e(v[j], v[j + 1]);
                Two g = r * two(o.k, o.k);
                if (TWO) g = fma_two(at_one(r, v[j], v[j + 1]), two(o.k1, o.k1), g);
                apart(g, v[j], v[j + 1]);
              }
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
          }
          release(sl);
          if (kept) { if (++kept_slot == kLossRing) kept_slot = 0; }
          else advance();
        }
      }
      if (thread == 0) outcome[b] = DistillEnd{o, st.x, st.y};
      __syncwarp();
      if (lane == 0) mbar_arrive(list_empty(b));           // and the row's stores are done
      loss_workers_sync();                                 // warp_stat may be written again
    }
  }
  __syncwarp();
  if (P.split > 1) cluster_sync();                         // no peer writes to a CTA that has ended
}

}  // namespace

#endif  // GBMUF_CSRC_DISTILL_CUH
