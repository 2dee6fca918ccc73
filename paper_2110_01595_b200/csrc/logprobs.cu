// Log probabilities of given tokens under the softmax of a row of logits, with the row's entropy and its likeliest tokens, and
// the gradient with respect to the logits (solon_token_logprobs, solon_token_logprobs_backward):
//     M = max z, S = sum e^(z - M), logp = (z_t - M) - log S, H = log S - sum e^(z - M) (z - M) / S
//     dz_j = g_logp (1[j = t] - p_j) - g_H p_j (log p_j + H),   log p_j = (z_j - M) - log S
// M and log S are kept apart, never added up: of M + log S little would be left of log S under a large M, and nothing in a row
// masked with the type's lowest value (which is uniform: log p = -log cols).
// Statistics in float32, the maximum and both sums carried along in one sweep (a new maximum rescales the sums).
//
// Edge cases, the same in both directions: a logit of -infinity has p = 0 and adds nothing (0 log 0 = 0); a row of nothing
// but -infinity has M = logp = -infinity, log S = H = 0 and gradient 0; a negative target has logp 0 and passes no
// gradient; a target beyond the vocabulary is not read and has logp NaN; NaN and +infinity make the row's results NaN, but M is
// +infinity where that is the largest.  A probability below 2^-126 counts as 0.
#include <math.h>

#include "elements.cuh"
#include "solon_internal.h"
#include "token_args.h"

namespace solon {

// Measured: 8192 x 32768 bfloat16 91 to 100 us (5.4 to 5.9 TB/s), 4096 x 32768 float32 89 us (6.0 TB/s), 2047 x 50001 float32 72 us and
// with 20 likeliest tokens 88 to 93 us; the gradient on 8192 x 32768 bfloat16 182 to 193 us (5.6 to 5.9 TB/s).
//
// Bound by memory, with the exponentials (one a logit: at 16 a clock and SM 60 % of the time that bfloat16 logits take to
// arrive) and the instructions beside them close behind, so those are kept few: two values an instruction, one multiply-add
// from a logit to its exponent, and one comparison per 64 bytes for everything that is rare.
constexpr int kLpThreads = 256;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpWords = 4;                    // 16-byte words of a thread in an iteration
constexpr int kLpChunk = kLpThreads * kLpWords;
constexpr int kLpCtasPerSm = 4;
constexpr int kLpMaxCluster = 8;
constexpr int kLpCandidates = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Iterations' words in shared memory: three beside the 16 KB of candidates would leave room for three CTAs on an SM only.
template <bool TOP>
constexpr int lp_stages = TOP ? 2 : 3;

// Order of the likeliest tokens as one integer: value first (NaN above all, -0 = +0), of equal values the lower index.
__device__ __forceinline__ uint32_t order_bits(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return z != z ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : (b | 0x80000000u);      // > 0 for every value
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return o == 0xFFFFFFFFu ? NAN : __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ unsigned long long rank_key(float z, uint32_t index) {
  return ((unsigned long long)order_bits(z) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long key) { return 0xFFFFFFFFu - (uint32_t)key; }
__device__ __forceinline__ float key_value(unsigned long long key) { return order_value((uint32_t)(key >> 32)); }

struct LogprobArgs {
  const void* logits;
  const int64_t* targets;      // nullptr: none
  float* logp;                 // outputs (nullptr: not wanted)
  float* entropy;
  float* peak;
  float* log_sum;
  int64_t* top_ids;
  float* top_logp;
  int64_t rows, cols, pitch;
  int top_k;
};

// Softmax sums of a part of a row against its largest logit: s = sum 2^t, a = sum 2^t t, t = (z - peak) log2 e.
// Without a finite logit s = a = 0; s is NaN where the row has no softmax.
struct SoftmaxPart {
  float peak, s, a;
};

__device__ __forceinline__ SoftmaxPart join_parts(const SoftmaxPart& x, const SoftmaxPart& y) {
  SoftmaxPart r;
  r.peak = fmaxf(x.peak, y.peak);
  // (a part that holds nothing, or nothing that counts beside the other, adds nothing; its distance may be infinite)
  const float dx = (x.peak - r.peak) * kLog2e, fx = exp2_fast(dx), dy = (y.peak - r.peak) * kLog2e, fy = exp2_fast(dy);
  const bool has_x = x.s != 0.0f && !(fx == 0.0f && x.s == x.s), has_y = y.s != 0.0f && !(fy == 0.0f && y.s == y.s);
  r.s = (has_x ? x.s * fx : 0.0f) + (has_y ? y.s * fy : 0.0f);
  r.a = (has_x ? fx * fmaf(dx, x.s, x.a) : 0.0f) + (has_y ? fy * fmaf(dy, y.s, y.a) : 0.0f);
  return r;
}
// (the peak is NaN if one part's is; s is then NaN as well)
template <int LANES>
__device__ __forceinline__ SoftmaxPart join_lanes(SoftmaxPart p) {
  const bool nan = __any_sync(0xffffffffu, p.peak != p.peak);
#pragma unroll
  for (int off = LANES / 2; off > 0; off >>= 1) {
    SoftmaxPart o;
    o.peak = __shfl_xor_sync(0xffffffffu, p.peak, off);
    o.s = __shfl_xor_sync(0xffffffffu, p.s, off);
    o.a = __shfl_xor_sync(0xffffffffu, p.a, off);
    p = join_parts(p, o);
  }
  if (nan) p.peak = NAN;
  return p;
}

// The sums of a thread while its warp goes through a row.  The exponent of a logit is one multiply-add, t = z log2 e - ref, the
// product exact; the reference is the integer next to a logit's product, the same in the whole warp, and moves (rescaling the
// sums) only when a logit lies more than 8 above it in base 2: hardly ever after the first words.
// Logits below `floor`, 140 or more under the reference, are raised to it: their 2^t is 0 either way, but t 2^t is defined.
// That holds for references of logits up to 1e7.  From 2^24 / log2 e = 1.16e7 on the integers of float32 lie 2 and more apart (at 1e10
// 1024), so the largest logit's own t can be that far from 0, which costs digits and then overflows or leaves nothing; next to
// float16's lowest value there is no floor.  Such a row - masked with a large finite value, until something else turns up -
// takes differences from a logit, which are exact or their 2^t is 0; `limit` is NaN then, so that every iteration of such
// a row, and of no other, is told apart behind the comparison that all make (2047 x 50001 float32 72 us with every 50th row
// all -1e9 and without; a branch of its own in every iteration made 8192 x 32768 bfloat16 2 us longer).
template <typename T>
struct LogprobThread {
  static constexpr float kLowest = Word16<T>::kMinusInf == 0xFC00FC00u ? -64000.0f : -1e7f, kHighest = 1e7f;      // (float16 ends at 65504)
  float peak, ref, limit;
  uint32_t floor;
  Float2 s, a;
  bool nan;                            // one was seen (it has no part in peak)

  __device__ __forceinline__ bool differences() const { return limit != limit; }      // t = (z - ref) log2 e

  __device__ __forceinline__ void init() {
    peak = limit = -INFINITY;          // (no reference yet: every finite logit is above the limit)
    ref = 0.0f;
    floor = Word16<T>::twice(-140.0f);
    s = a = pack2(0.0f, 0.0f);
    nan = false;
  }
  // `big`: the thread's largest value of what comes next (NaN if there is one).  The whole warp calls it.
  __device__ __forceinline__ void move_reference(float big) {
    if (!(big < INFINITY)) {           // +infinity or NaN: the row has no softmax
      nan |= big != big;
      s = pack2(NAN, NAN);
      big = -INFINITY;
    }
    const float to = order_value(__reduce_max_sync(0xffffffffu, order_bits(big)));
    const bool was_far = differences(), far = to < kLowest || to > kHighest;
    if (!(to > (was_far ? ref + 8.0f / kLog2e : limit))) return;
    const float r = far ? to : rintf(to * kLog2e);
    if (was_far || limit > -INFINITY) {
      float d = was_far ? (far ? (ref - r) * kLog2e : fmaf(ref, kLog2e, -r)) : (far ? -fmaf(r, kLog2e, -ref) : ref - r);
      d = fmaxf(d, -1e4f);             // (finite)
      const float f = exp2_fast(d);
      s = mul2(s, pack2(f, f));
      a = fma2(s, pack2(d, d), mul2(a, pack2(f, f)));
    }
    ref = r;
    limit = far ? NAN : to + 8.0f / kLog2e;
    floor = Word16<T>::twice(to - fmaxf(140.0f, fabsf(to) * 0.015625f));
  }
  // Two elements: t = z log2 e - ref, none above the limit.
  __device__ __forceinline__ void add_pair(Float2 z) {
    const Float2 t = fma2(z, pack2(kLog2e, kLog2e), pack2(-ref, -ref));
    float t0, t1;
    unpack2(t, t0, t1);
    const Float2 e = pack2(exp2_fast(t0), exp2_fast(t1));
    s = add2(s, e);
    a = fma2(e, t, a);
  }
  __device__ __forceinline__ void add_word(const uint4& w) {
    uint4 q;
    q.x = Word16<T>::at_least(w.x, floor);
    q.y = Word16<T>::at_least(w.y, floor);
    q.z = Word16<T>::at_least(w.z, floor);
    q.w = Word16<T>::at_least(w.w, floor);
    float x[Word16<T>::kCount];
    Word16<T>::unpack(q, x);
#pragma unroll
    for (int j = 0; j < Word16<T>::kCount; j += 2) add_pair(pack2(x[j], x[j + 1]));
  }
  // The same by differences.
  __device__ __forceinline__ void add_pair_far(float z0, float z1) {
    const float t0 = max_nan((z0 - ref) * kLog2e, -200.0f), t1 = max_nan((z1 - ref) * kLog2e, -200.0f);
    const Float2 e = pack2(exp2_fast(t0), exp2_fast(t1));
    s = add2(s, e);
    a = fma2(e, pack2(t0, t1), a);
  }
  __device__ __forceinline__ void add_word_far(const uint4& w) {
    float x[Word16<T>::kCount];
    Word16<T>::unpack(w, x);
#pragma unroll
    for (int j = 0; j < Word16<T>::kCount; j += 2) add_pair_far(x[j], x[j + 1]);
  }
  // The warp's sums, against its largest logit (NaN if there is one).
  __device__ __forceinline__ SoftmaxPart warp_part() const {
    float s0, s1, a0, a1;
    unpack2(s, s0, s1);
    unpack2(a, a0, a1);
    SoftmaxPart p = {order_value(__reduce_max_sync(0xffffffffu, order_bits(peak))), s0 + s1, a0 + a1};
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      p.s += __shfl_xor_sync(0xffffffffu, p.s, off);
      p.a += __shfl_xor_sync(0xffffffffu, p.a, off);
    }
    if (p.peak > -INFINITY && p.s != 0.0f) {
      const float d = differences() ? (ref - p.peak) * kLog2e : fmaf(-p.peak, kLog2e, ref), f = exp2_fast(d);
      p.a = f * fmaf(d, p.s, p.a);
      p.s *= f;
    }
    if (__any_sync(0xffffffffu, nan)) p.peak = NAN;
    return p;
  }
};

// Largest element of a thread's words (NaN if there is one).
template <typename T, int N>
__device__ __forceinline__ float largest_of(const uint4 (&w)[N]) {
  using Word = Word16<T>;
  static_assert(N % 2 == 0 && N >= 4);
  if constexpr (sizeof(T) == 4) {                // three at a time: half as many instructions
    uint4 m = w[0];
#pragma unroll
    for (int u = 1; u < N - 1; u += 2) {
      m.x = Word::max3(m.x, w[u].x, w[u + 1].x);
      m.y = Word::max3(m.y, w[u].y, w[u + 1].y);
      m.z = Word::max3(m.z, w[u].z, w[u + 1].z);
      m.w = Word::max3(m.w, w[u].w, w[u + 1].w);
    }
    const uint4& last = w[N - 1];
    return Word::widest(Word::at_least(Word::max3(m.x, m.y, m.z), Word::max3(Word::max3(m.w, last.x, last.y), last.z, last.w)));
  } else {
    uint32_t m[N];
#pragma unroll
    for (int u = 0; u < N; ++u) m[u] = Word::at_least(Word::at_least(w[u].x, w[u].y), Word::at_least(w[u].z, w[u].w));
#pragma unroll
    for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
      for (int u = 0; u < n; ++u) m[u] = Word::at_least(m[u], m[u + n]);
    return Word::widest(m[0]);
  }
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ float peer_float(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long peer_key(uint32_t addr) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}

// Candidates for the likeliest tokens.  A value enters unless k values at least as large, of lower index, are known: the
// threshold is the k-th largest of the maxima of groups of eight threads, or of two from k = 9 on (of the eights' 32 maxima the
// 32nd is the smallest, with some 130 values above it, of the pairs' 128 it has 37), taken anew whenever the part of the row that
// has been seen has doubled, with all threads at the same place of the row.  The k largest are picked from the candidates at
// the end.  Should they overflow - ties by the thousand, as in a masked row, or a row that rises throughout -, they are
// collected once more with the final threshold, of the values equal to it only the row's first; failing that too, the k
// largest are found one by one.
struct LogprobTop {
  unsigned long long key[2][kLpCandidates];      // by the parity of the row: one warp picks while the others go on
  unsigned long long best[SOLON_MAX_TOP];        // this CTA's k largest, in falling order (0: fewer)
  unsigned long long scratch[kLpWarps];
  __align__(16) uint32_t pair_max[2][kLpThreads / 2];      // by the parity of the refresh
  uint32_t threshold;                            // order bits; 0: none yet
  int count[3];                                  // by the row modulo 3, see below
};

__device__ __forceinline__ void push_candidate(int* count, unsigned long long* keys, float z, uint32_t index) {
  const int at = atomicAdd(count, 1);
  if (at < kLpCandidates) keys[at] = rank_key(z, index);
}

// Which of a thread's elements are above the threshold (`ties`: not below it), as bits; words whose largest value is not are
// passed over.  Elements are fetched from the ring again by their bits: few are, and the code for them stays short.
template <typename T, int N>
__device__ __forceinline__ uint32_t candidate_bits(const uint4 (&w)[N], float threshold, bool ties) {
  uint32_t bits = 0;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const float big = Word16<T>::largest(w[u]);
    if (ties ? !(big < threshold) : !(big <= threshold)) {
      float x[Word16<T>::kCount];
      Word16<T>::unpack(w[u], x);
#pragma unroll
      for (int j = 0; j < Word16<T>::kCount; ++j)
        if (ties ? !(x[j] < threshold) : !(x[j] <= threshold)) bits |= 1u << (u * Word16<T>::kCount + j);
    }
  }
  return bits;
}

// A thread's largest value so far (order bits, 0: it has seen nothing) to its pair's.
__device__ __forceinline__ void write_pair_max(LogprobTop& top, int buffer, uint32_t seen) {
  seen = max(seen, __shfl_xor_sync(0xffffffffu, seen, 1));
  if ((threadIdx.x & 1) == 0) top.pair_max[buffer][threadIdx.x >> 1] = seen;
}
// The k-th largest of 32 values, one a lane, equal ones counted apart.
__device__ __forceinline__ uint32_t kth_largest(uint32_t mine, int k) {
  const int lane = threadIdx.x & 31;
  int rank = 0;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const uint32_t other = __shfl_sync(0xffffffffu, mine, j);
    rank += other > mine || (other == mine && j < lane);
  }
  return __shfl_sync(0xffffffffu, mine, __ffs(__ballot_sync(0xffffffffu, rank == k - 1)) - 1);
}
// The k-th largest of 128 values, four a lane, from the bits on in which they differ: until k lie above, or all bits are known.
__device__ __forceinline__ uint32_t kth_largest(const uint4& q, int k) {
  const uint32_t high = __reduce_max_sync(0xffffffffu, max(max(q.x, q.y), max(q.z, q.w)));
  const uint32_t low = __reduce_min_sync(0xffffffffu, min(min(q.x, q.y), min(q.z, q.w)));
  if (high == low) return high;
  const int top = 31 - __clz(high ^ low);
  uint32_t bound = high & ~((2u << top) - 1u);
  for (int bit = top; bit >= 0; --bit) {
    const uint32_t trial = bound | (1u << bit);
    const int above = (int)__reduce_add_sync(0xffffffffu, (uint32_t)((q.x >= trial) + (q.y >= trial) + (q.z >= trial) + (q.w >= trial)));
    if (above >= k) bound = trial;
    if (above == k) {
      const uint32_t least = min(min(q.x >= bound ? q.x : ~0u, q.y >= bound ? q.y : ~0u), min(q.z >= bound ? q.z : ~0u, q.w >= bound ? q.w : ~0u));
      return __reduce_min_sync(0xffffffffu, least);
    }
  }
  return bound;
}

// Of n > most keys in shared memory (all different, beside zeros) the k largest and some more, `most` at most, in their order; how
// many there are, and the order bits of the smallest.  One warp: bit by bit, from the first on in which the keys differ, the
// largest bound that k keys reach; up to 128 keys stay in registers, and hardly ever do values tie so that their indices count.
__device__ __noinline__ int trim_keys(unsigned long long* keys, int n, int k, int most, uint32_t* smallest) {
  constexpr int kHeld = 4;
  const int lane = threadIdx.x & 31;
  uint32_t order[kHeld], high = 0, low = ~0u;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    order[u] = u * 32 + lane < n ? (uint32_t)(keys[u * 32 + lane] >> 32) : 0u;
    if (u * 32 + lane < n) {
      high = max(high, order[u]);
      low = min(low, order[u]);
    }
  }
  for (int i = kHeld * 32 + lane; i < n; i += 32) {
    const uint32_t o = (uint32_t)(keys[i] >> 32);
    high = max(high, o);
    low = min(low, o);
  }
  high = __reduce_max_sync(0xffffffffu, high);
  low = __reduce_min_sync(0xffffffffu, low);
  const int top = high == low ? -1 : 31 - __clz(high ^ low);
  uint32_t bound = top < 0 ? high : high & ~((2u << top) - 1u);
  unsigned long long least = 0;                  // the smallest key that stays
  int left = n;
  for (int bit = top; bit >= 0 && left > most; --bit) {
    const uint32_t trial = bound | (1u << bit);
    uint32_t above = 0;
#pragma unroll
    for (int u = 0; u < kHeld; ++u) above += order[u] >= trial;
    for (int i = kHeld * 32 + lane; i < n; i += 32) above += (uint32_t)(keys[i] >> 32) >= trial;
    above = __reduce_add_sync(0xffffffffu, above);
    if ((int)above >= k) {
      bound = trial;
      left = (int)above;
    }
  }
  least = (unsigned long long)bound << 32;
  for (int bit = 31; bit >= 0 && left > most; --bit) {       // among equal values by the index
    const unsigned long long trial = least | (1ull << bit);
    uint32_t above = 0;
    for (int i = lane; i < n; i += 32) above += keys[i] >= trial;
    above = __reduce_add_sync(0xffffffffu, above);
    if ((int)above >= k) {
      least = trial;
      left = (int)above;
    }
  }
  int kept = 0;
  low = ~0u;
  for (int base = 0; base < n; base += 32) {
    const unsigned long long key = base + lane < n ? keys[base + lane] : 0;
    const bool keep = key >= least && key != 0;
    const uint32_t mask = __ballot_sync(0xffffffffu, keep);
    __syncwarp();
    if (keep) {
      keys[kept + __popc(mask & ((1u << lane) - 1u))] = key;
      low = min(low, (uint32_t)(key >> 32));
    }
    kept += __popc(mask);
    __syncwarp();
  }
  *smallest = __reduce_min_sync(0xffffffffu, low);
  return kept;
}

// The k largest of n keys (all different, beside zeros) into best, in falling order, zeros behind them; the keys are lost.  One
// warp: of more than 64 keys those that cannot be among them go first, then each counts the larger ones.
__device__ __forceinline__ void select_largest(unsigned long long* keys, int n, unsigned long long* best, int k) {
  const int lane = threadIdx.x & 31;
  uint32_t smallest;
  if (n > 64) n = trim_keys(keys, n, k, 64, &smallest);
  const unsigned long long mine = lane < n ? keys[lane] : 0, second = lane + 32 < n ? keys[lane + 32] : 0;
  int rank = 0, second_rank = 0;
  if (n <= 32) {
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += keys[j] > mine;
  } else {
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const unsigned long long other = keys[j];
      rank += other > mine;
      second_rank += other > second;
    }
  }
  if (lane < k) best[lane] = 0;
  __syncwarp();
  if (mine != 0 && rank < k) best[rank] = mine;
  if (second != 0 && second_rank < k) best[second_rank] = second;
  __syncwarp();
}

// The share of a row that a CTA reads: words [begin, end) of 16 bytes from the row's first 16-byte boundary on.  Elements before
// it (`head`) and behind the last whole word go one by one to the cluster's first and last CTA.
template <typename T>
struct RowShare {
  const T* z;
  int head, words, begin, end;

  __device__ __forceinline__ RowShare(const LogprobArgs& a, int64_t row, uint32_t rank, uint32_t size) {
    z = static_cast<const T*>(a.logits) + row * a.pitch;
    const int cols = (int)a.cols;
    const int to_boundary = (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T);
    head = to_boundary < cols ? to_boundary : cols;
    words = (cols - head) / Word16<T>::kCount;
    const int shift = __ffs(size) - 1;           // (a power of two)
    begin = (int)((uint32_t)words * rank >> shift);
    end = (int)((uint32_t)words * (rank + 1) >> shift);
  }
  __device__ __forceinline__ const uint4* body() const { return reinterpret_cast<const uint4*>(z + head); }
  // all its elements, those outside the words included
  __device__ __forceinline__ int first(uint32_t rank) const { return rank == 0 ? 0 : head + begin * Word16<T>::kCount; }
  __device__ __forceinline__ int behind(uint32_t rank, uint32_t size, int cols) const { return rank == size - 1 ? cols : head + end * Word16<T>::kCount; }
};

// The candidates of a CTA's share when they have overflowed.  All threads; true: they are in the list, false: top.best is done.
template <typename T>
__device__ __noinline__ bool collect_again(const T* z, int first, int behind, LogprobTop& top, int* count, unsigned long long* keys, int k) {
  const uint32_t threshold = top.threshold;
  __syncthreads();                               // (everybody has looked at the count)
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
  for (int c = first + threadIdx.x; c < behind; c += kLpThreads) {
    const float v = to_float(z[c]);
    const uint32_t o = order_bits(v);
    if (o > threshold || (o == threshold && c < first + kLpCandidates / 2)) push_candidate(count, keys, v, (uint32_t)c);
  }
  __syncthreads();
  const int found = *count;
  if (found >= k && found <= kLpCandidates) return true;
  unsigned long long last = ~0ull;
  for (int j = 0; j < k; ++j) {                  // the largest key below the one before
    unsigned long long best = 0;
    for (int c = first + threadIdx.x; c < behind; c += kLpThreads) {
      const unsigned long long key = rank_key(to_float(z[c]), (uint32_t)c);
      if (key < last && key > best) best = key;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, off));
    if ((threadIdx.x & 31) == 0) top.scratch[threadIdx.x >> 5] = best;
    __syncthreads();
    for (int i = 0; i < kLpWarps; ++i) best = max(best, top.scratch[i]);
    if (threadIdx.x == 0) top.best[j] = best;
    last = best;
    __syncthreads();
  }
  return false;
}

// A row is read by a cluster of 1 to 8 CTAs, each taking a stretch of it; clusters stay for many rows.  Every thread copies its
// words of the next iterations into shared memory ahead of time, across the rows' ends (cp.async: a thread waits for its own
// copies only), and one warp finishes a row - another one each row - while the others are at the next.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads, kLpCtasPerSm) logprob_kernel(LogprobArgs a) {
  constexpr int kVec = Word16<T>::kCount;
  constexpr int kStages = lp_stages<TOP>;
  extern __shared__ __align__(16) uint4 ring[];           // stages x kLpWords x threads
  __shared__ SoftmaxPart warp_part[2][kLpWarps];          // by the parity of the row
  __shared__ SoftmaxPart cta_part;
  __shared__ __align__(16) unsigned char top_bytes[TOP ? sizeof(LogprobTop) : 16];
  LogprobTop& top = *reinterpret_cast<LogprobTop*>(top_bytes);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const int cols = (int)a.cols;
  const int64_t stride = gridDim.x / size;

  int64_t ahead_row = blockIdx.x / size;                  // what is copied next
  RowShare<T> ahead(a, ahead_row < a.rows ? ahead_row : 0, rank, size);
  int ahead_base = ahead.begin;
  auto issue = [&](int stage) {
    while (ahead_row < a.rows && ahead_base >= ahead.end) {
      ahead_row += stride;
      if (ahead_row < a.rows) {
        ahead = RowShare<T>(a, ahead_row, rank, size);
        ahead_base = ahead.begin;
      }
    }
    if (ahead_row < a.rows) {
      const uint4* from = ahead.body() + ahead_base + threadIdx.x;
      uint4* to = ring + stage * kLpChunk + threadIdx.x;
      const int left = ahead.end - ahead_base - (int)threadIdx.x;
#pragma unroll
      for (int u = 0; u < kLpWords; ++u)
        if (u * kLpThreads < left) copy16_async(to + u * kLpThreads, from + u * kLpThreads);
      ahead_base += kLpChunk;
    }
    copies_commit();
  };
  if (TOP && threadIdx.x < 3) top.count[threadIdx.x] = 0;
#pragma unroll
  for (int s = 0; s < kStages; ++s) issue(s);
  __syncthreads();
  int stage = 0, parity = 0, third = 0, finisher = 0, refresh = 0;

  for (int64_t row = blockIdx.x / size; row < a.rows; row += stride) {
    const RowShare<T> share(a, row, rank, size);
    const T* z = share.z;
    int* const count = &top.count[TOP ? third : 0];
    unsigned long long* const keys = top.key[TOP ? parity : 0];
    // what the finishing warp will need from memory
    T edge = from_float<T>(-INFINITY);                    // the elements outside the words: head in lanes 0 .., tail in lanes 16 ..
    int edge_index = -1;
    int64_t target = -1;
    float target_logit = 0.0f;
    if (warp == finisher) {
      const int tail = share.head + share.words * kVec;
      if (rank == 0 && lane < share.head) edge_index = lane;
      if (rank == size - 1 && lane >= 16 && lane - 16 < cols - tail) edge_index = tail + lane - 16;
      if (edge_index >= 0) edge = z[edge_index];
      if (a.targets && a.logp && rank == 0) {
        target = a.targets[row];
        if (target >= 0 && target < a.cols) target_logit = to_float(z[target]);
      }
    }

    auto push_bits = [&](uint32_t bits, const uint4* words, int base) {
      while (bits) {
        const int e = __ffs(bits) - 1, u = e / kVec, j = e % kVec;
        bits &= bits - 1;
        const float v = to_float(reinterpret_cast<const T*>(words + u * kLpThreads)[j]);
        push_candidate(count, keys, v, (uint32_t)(share.head + (base + u * kLpThreads + (int)threadIdx.x) * kVec + j));
      }
    };

    LogprobThread<T> t;
    t.init();
    float threshold = -INFINITY;                          // candidates are above it
    int next_refresh = 2, iteration = 0;
    for (int base = share.begin; base < share.end; base += kLpChunk, ++iteration) {
      const uint4* words = ring + stage * kLpChunk + threadIdx.x;
      copies_wait<kStages - 1>();
      uint4 w[kLpWords];
#pragma unroll
      for (int u = 0; u < kLpWords; ++u) w[u] = words[u * kLpThreads];
      if (base + kLpChunk > share.end) {
        constexpr uint32_t kNone = Word16<T>::kMinusInf;
#pragma unroll
        for (int u = 0; u < kLpWords; ++u)
          if (base + u * kLpThreads + (int)threadIdx.x >= share.end) w[u] = make_uint4(kNone, kNone, kNone, kNone);
      }
      const float biggest = largest_of<T>(w);
      t.peak = fmaxf(t.peak, biggest);
      bool added = false;
      if (__any_sync(0xffffffffu, !(biggest <= t.limit))) {
        t.move_reference(biggest);
        if (t.differences()) {
#pragma unroll
          for (int u = 0; u < kLpWords; ++u) t.add_word_far(w[u]);
          added = true;
        }
      }
      if (!added) {
#pragma unroll
        for (int u = 0; u < kLpWords; ++u) t.add_word(w[u]);
      }

      if constexpr (TOP) {
        if (iteration > 0) {
          threshold = order_value(*(volatile uint32_t*)&top.threshold);
          if (!(biggest <= threshold)) push_bits(candidate_bits<T>(w, threshold, false), words, base);
        }
        if (iteration == 0 || (iteration + 1 == next_refresh && base + kLpChunk < share.end)) {
          // one warp works the threshold out; the others need not wait for it but in the first stretch, which is compared
          // with its own (so values equal to it count there)
          write_pair_max(top, refresh, share.begin + (int)threadIdx.x < share.end ? order_bits(t.peak) : 0u);
          __syncthreads();
          if (warp == kLpWarps - 1) {
            const uint4 q = reinterpret_cast<const uint4*>(top.pair_max[refresh])[lane];
            const uint32_t found = a.top_k <= 8 ? kth_largest(max(max(q.x, q.y), max(q.z, q.w)), a.top_k) : kth_largest(q, a.top_k);
            if (lane == 0) *(volatile uint32_t*)&top.threshold = found;
          }
          refresh ^= 1;
          if (iteration > 0) next_refresh *= 2;
          if (iteration == 0) {
            __syncthreads();
            const uint32_t at_least = top.threshold;
            uint32_t bits = candidate_bits<T>(w, at_least ? order_value(at_least) : -INFINITY, true);
#pragma unroll
            for (int u = 0; u < kLpWords; ++u)            // (not the -infinities behind the row's end)
              if (base + u * kLpThreads + (int)threadIdx.x >= share.end) bits &= ~(((1u << kVec) - 1u) << (u * kVec));
            push_bits(bits, words, base);
          }
        }
      }
      issue(stage);                                       // into the words just read
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }

    // the elements outside the words come last: the threshold takes what it has seen to be of lower index than what it is
    // compared with, so these have no part in it
    if (warp == finisher && __any_sync(0xffffffffu, edge_index >= 0)) {
      const float v = to_float(edge);
      t.peak = fmaxf(t.peak, v);
      if (__any_sync(0xffffffffu, !(v <= t.limit))) t.move_reference(v);
      constexpr uint32_t kNone = Word16<T>::kMinusInf;
      if (t.differences()) t.add_pair_far(v, -INFINITY);
      else t.add_word(make_uint4(Word16<T>::first(edge), kNone, kNone, kNone));
      if (TOP && edge_index >= 0) push_candidate(count, keys, v, (uint32_t)edge_index);
    }
    const SoftmaxPart mine = t.warp_part();
    if (lane == 0) warp_part[parity][warp] = mine;
    __syncthreads();

    // Everybody has read the row before's count on the way here; its place is used again by the row after the next, which begins
    // behind the next one's barrier.
    if (TOP && threadIdx.x == 0) top.count[third == 0 ? 2 : third - 1] = 0;
    bool listed = true;                                   // the candidates are in the list
    if (TOP && *count > kLpCandidates) listed = collect_again<T>(z, share.first(rank), share.behind(rank, size, cols), top, count, keys, a.top_k);

    SoftmaxPart part = {-INFINITY, 0.0f, 0.0f};
    if (warp == finisher) {
      if (lane < kLpWarps) part = warp_part[parity][lane];
      part = join_lanes<kLpWarps>(part);
      if (TOP && listed) select_largest(keys, *count, top.best, a.top_k);
      if (size > 1 && lane == 0) cta_part = part;
    }
    if (size > 1) cluster_barrier();
    if (warp == finisher && rank == 0) {
      if (size > 1) {
        part = {-INFINITY, 0.0f, 0.0f};
        if (lane < (int)size) {
          const uint32_t at = peer_address(&cta_part, lane);
          part = {peer_float(at), peer_float(at + 4), peer_float(at + 8)};
        }
        part = join_lanes<kLpMaxCluster>(part);
        if (TOP) {
          __syncwarp();
          for (int i = lane; i < (int)size * a.top_k; i += 32) keys[i] = peer_key(peer_address(&top.best[i % a.top_k], i / a.top_k));
          __syncwarp();
          select_largest(keys, (int)size * a.top_k, top.best, a.top_k);
        }
      }
      part.peak = __shfl_sync(0xffffffffu, part.peak, 0);
      part.s = __shfl_sync(0xffffffffu, part.s, 0);
      part.a = __shfl_sync(0xffffffffu, part.a, 0);
      const bool empty = part.peak == -INFINITY && part.s == 0.0f;
      const float log_s = empty ? 0.0f : logf(part.s);
      if (lane == 0) {
        if (a.peak) a.peak[row] = part.peak;
        if (a.log_sum) a.log_sum[row] = log_s;
        if (a.entropy) a.entropy[row] = empty ? 0.0f : log_s - kLn2 * (part.a / part.s);
        if (a.targets && a.logp) {
          float lp = 0.0f;
          if (target >= a.cols) lp = NAN;
          else if (target >= 0) lp = empty ? -INFINITY : (target_logit - part.peak) - log_s;
          a.logp[row] = lp;
        }
      }
      if (TOP && lane < a.top_k) {
        const unsigned long long key = top.best[lane];
        a.top_ids[row * a.top_k + lane] = key_index(key);
        a.top_logp[row * a.top_k + lane] = empty ? -INFINITY : (key_value(key) - part.peak) - log_s;
      }
    }
    if (size > 1) cluster_barrier();                      // the first CTA has read the others' shared memory
    parity ^= 1;
    third = third == 2 ? 0 : third + 1;
    finisher = finisher + 1 == kLpWarps ? 0 : finisher + 1;
  }
}

// ---- many or short rows: a warp a row --------------------------------------------------------------------------------------
// Nothing in a row then waits for another warp, and the serial work at a row's end (and for its likeliest tokens) of one warp
// hides behind the others' streams; but a warp alone takes its time over a row, so there have to be the more rows the longer they
// are, up to 12 per SM.  Measured, bfloat16, CTA a row against warp a row in us: 8192 x 32768 107 / 91; 1200 x 16000 13.0 / 11.9;
// 600 x 8000 6.4 / 6.3; 300 x 4000 4.9 / 4.5; 75 x 4000 4.0 / 4.1; 16 x 2000 3.9 / 3.5; with 8 likeliest tokens 1776 x 50000 68 / 68;
// 1200 x 8000 17.5 / 17.1; 600 x 4000 11.3 / 10.1; 300 x 4000 7.3 / 9.4; 300 x 2000 7.2 / 6.5; 16 x 1000 6.2 / 5.1.
// The candidates are a warp's own: filtered as above with the lanes' maxima for groups - with many to find, of the first stretch
// the maxima of quarters, and then what is left of the list: of the 32 lanes' maxima the 32nd is the smallest -, appended by
// ballots, and pruned to little more than k when the list is full.
constexpr int kLpWarpRows = 12;
static bool logprob_by_warps(int64_t rows, int64_t cols, bool top, int sms) {
  const int64_t span = top ? 1024 : 2048;      // columns that a row may have for every row per SM; up to it any number of rows will do
  return cols <= span || rows >= (int64_t)sms * kLpWarpRows || rows * span >= cols * sms;
}
constexpr int kLpWarpList = 256;               // candidates
template <typename T>
constexpr int lp_warp_words = 32 / Word16<T>::kCount;                    // words of a lane in an iteration: 32 elements
// CTAs of eight warps on an SM.  Two suffice the plain sums of two-byte logits (8192 x 32768 bfloat16 takes 101 us with three, 91 with
// two, 16384 x 16384 90 and 85: the last round of rows is fuller), and for likeliest tokens of float32 ones three would have to
// share the memory of the lists (2047 x 50001 with 20, lists of half the length: 91 us, 85 with two); float32 sums (2047 x 50001: 72
// us, 74 with two) and likeliest tokens of two-byte logits (8192 x 32768 with 8: 162 us, 164 with two) take three.
template <typename T, bool TOP>
constexpr int lp_warp_ctas = (sizeof(T) == 4) == TOP ? 2 : 3;
template <typename T, bool TOP>
constexpr int lp_warp_stages = sizeof(T) == 4 ? 2 : TOP ? 3 : 4;      // iterations' words in shared memory

// A lower bound of the k-th largest of the lanes' values (order bits): exact in the upper 16 bits.
__device__ __forceinline__ uint32_t kth_largest_bound(uint32_t mine, int k) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t trial = bound | (1u << bit);
    if (__popc(__ballot_sync(0xffffffffu, mine >= trial)) >= k) bound = trial;
  }
  return bound;
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads, (lp_warp_ctas<T, TOP>)) logprob_warp_kernel(LogprobArgs a) {
  constexpr int kVec = Word16<T>::kCount;
  constexpr int kWords = lp_warp_words<T>;
  constexpr int kStages = lp_warp_stages<T, TOP>;
  constexpr int kChunk = 32 * kWords;                     // words of an iteration
  constexpr uint32_t kNone = Word16<T>::kMinusInf;
  extern __shared__ __align__(16) uint4 shared[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint4* ring = shared + warp * kStages * kChunk + lane;
  unsigned long long* list = reinterpret_cast<unsigned long long*>(shared + kLpWarps * kStages * kChunk) + warp * (kLpWarpList + SOLON_MAX_TOP);
  unsigned long long* best = list + kLpWarpList;
  const int cols = (int)a.cols, k = a.top_k;
  const int64_t stride = (int64_t)gridDim.x * kLpWarps;

  int64_t row = (int64_t)warp * gridDim.x + blockIdx.x;   // (neighbouring rows to different SMs)
  int64_t ahead_row = row;                                // what is copied next: the row, the lane's word, the words from there on
  const uint4* ahead = nullptr;
  int ahead_left = 0;
  auto ahead_from = [&]() {
    while (ahead_row < a.rows) {
      const RowShare<T> share(a, ahead_row, 0, 1);
      ahead = share.body() + lane;
      ahead_left = share.words - lane;
      if (share.words > 0) return;
      ahead_row += stride;
    }
  };
  ahead_from();
  auto issue = [&](uint4* to) {
    if (ahead_row < a.rows) {
      if (ahead_left + lane >= kChunk) {
#pragma unroll
        for (int u = 0; u < kWords; ++u) copy16_async(to + u * 32, ahead + u * 32);
      } else {
#pragma unroll
        for (int u = 0; u < kWords; ++u)
          if (u * 32 < ahead_left) copy16_async(to + u * 32, ahead + u * 32);
      }
      ahead += kChunk;
      ahead_left -= kChunk;
      if (ahead_left + lane <= 0) {
        ahead_row += stride;
        ahead_from();
      }
    }
    copies_commit();
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) issue(ring + s * kChunk);
  const bool with_target = a.targets && a.logp;
  int64_t next_target = with_target && row < a.rows ? a.targets[row] : -1;
  uint4* stage = ring;

  for (; row < a.rows; row += stride) {
    const RowShare<T> share(a, row, 0, 1);
    const T* z = share.z;
    const int tail = share.head + share.words * kVec;
    // from memory, for the row's end: the elements outside the words (head in lanes 0 .., tail in lanes 16 ..) and the target
    const int edge_index = lane < share.head ? lane : lane >= 16 && lane - 16 < cols - tail ? tail + lane - 16 : -1;
    T edge = from_float<T>(-INFINITY), target_logit = from_float<T>(0.0f);
    if (edge_index >= 0) edge = z[edge_index];
    const int64_t target = next_target;
    if (target >= 0 && target < a.cols) target_logit = z[target];
    if (with_target && row + stride < a.rows) next_target = a.targets[row + stride];

    LogprobThread<T> t;
    t.init();
    int listed = 0, next_refresh = 1, iteration = 0;
    float threshold = -INFINITY;                          // candidates are above it, or (see above) not below it
    auto prune = [&]() {                                  // to the k largest and a half as many again
      uint32_t smallest;
      listed = trim_keys(list, listed, k, k + (k >> 1), &smallest);
      threshold = fmaxf(threshold, order_value(smallest));
    };
    auto append = [&](bool wanted, float v, int index) {
      const uint32_t mask = __ballot_sync(0xffffffffu, wanted);
      if (listed + __popc(mask) > kLpWarpList) {
        prune();
      }
      if (wanted) list[listed + __popc(mask & ((1u << lane) - 1u))] = rank_key(v, (uint32_t)index);
      listed += __popc(mask);
      __syncwarp();
    };
    for (int base = 0; base < share.words; base += kChunk, ++iteration) {
      copies_wait<kStages - 1>();
      uint4 w[kWords];
#pragma unroll
      for (int u = 0; u < kWords; ++u) w[u] = stage[u * 32];
      const bool last = base + kChunk > share.words;
      if (last) {
#pragma unroll
        for (int u = 0; u < kWords; ++u)
          if (base + u * 32 + lane >= share.words) w[u] = make_uint4(kNone, kNone, kNone, kNone);
      }
      const float biggest = largest_of<T>(w);
      t.peak = fmaxf(t.peak, biggest);
      bool added = false;
      if (__any_sync(0xffffffffu, !(biggest <= t.limit))) {
        t.move_reference(biggest);
        if (t.differences()) {
#pragma unroll
          for (int u = 0; u < kWords; ++u) t.add_word_far(w[u]);
          added = true;
        }
      }
      if (!added) {
#pragma unroll
        for (int u = 0; u < kWords; ++u) t.add_word(w[u]);
      }
      if constexpr (TOP) {
        const bool first = iteration == 0;
        if (first) {                                      // compared with its own threshold: equal values enter
          uint32_t bound;
          if (k <= 16) {
            bound = kth_largest_bound(lane < share.words ? order_bits(t.peak) : 0u, k);
          } else {                                        // of the maxima of a quarter of a lane's elements each
            uint32_t quarter[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              quarter[u] = order_bits(Word16<T>::largest(w[u]));
              if constexpr (kWords == 8) quarter[u] = max(quarter[u], order_bits(Word16<T>::largest(w[u + 4])));
            }
            bound = kth_largest(make_uint4(quarter[0], quarter[1], quarter[2], quarter[3]), k);
          }
          if (bound >= 0x00800000u) threshold = order_value(bound);      // (below: fewer than k lanes have a finite value; all enter)
        }
        if (__any_sync(0xffffffffu, first ? !(biggest < threshold) : !(biggest <= threshold))) {
          uint32_t bits = candidate_bits<T>(w, threshold, first);
          if (last) {                                     // (not the -infinities behind the row's end)
#pragma unroll
            for (int u = 0; u < kWords; ++u)
              if (base + u * 32 + lane >= share.words) bits &= ~(((1u << kVec) - 1u) << (u * kVec));
          }
          // (all picked with one threshold: one that is raised on the way, by pruning, counts from the next stretch on)
          while (__any_sync(0xffffffffu, bits != 0)) {
            const int e = bits ? __ffs(bits) - 1 : 0, u = e / kVec, j = e % kVec;
            const float v = to_float(reinterpret_cast<const T*>(stage + u * 32)[j]);
            append(bits != 0, v, share.head + (base + u * 32 + lane) * kVec + j);
            bits &= bits - 1;
          }
        }
        if (iteration + 1 == next_refresh && base + kChunk < share.words) {
          if (k > 24) {
            if (listed > k + (k >> 1)) prune();
          } else if (!first) threshold = fmaxf(threshold, order_value(kth_largest_bound(order_bits(t.peak), k)));      // (NaN: below -infinity)
          next_refresh *= 2;
        }
      }
      issue(stage);                                       // into the words just read
      stage = stage == ring + (kStages - 1) * kChunk ? ring : stage + kChunk;
    }
    if (__any_sync(0xffffffffu, edge_index >= 0)) {
      const float v = to_float(edge);
      t.peak = fmaxf(t.peak, v);
      if (__any_sync(0xffffffffu, !(v <= t.limit))) t.move_reference(v);
      if (t.differences()) t.add_pair_far(v, -INFINITY);
      else t.add_word(make_uint4(Word16<T>::first(edge), kNone, kNone, kNone));
      if (TOP) append(edge_index >= 0, v, edge_index);
    }
    const SoftmaxPart part = t.warp_part();
    const bool empty = part.peak == -INFINITY && part.s == 0.0f;
    const float log_s = empty ? 0.0f : logf(part.s);
    if (lane == 0) {
      if (a.peak) a.peak[row] = part.peak;
      if (a.log_sum) a.log_sum[row] = log_s;
      if (a.entropy) a.entropy[row] = empty ? 0.0f : log_s - kLn2 * (part.a / part.s);
      if (with_target) {
        float lp = 0.0f;
        if (target >= a.cols) lp = NAN;
        else if (target >= 0) lp = empty ? -INFINITY : (to_float(target_logit) - part.peak) - log_s;
        a.logp[row] = lp;
      }
    }
    if constexpr (TOP) {
      __syncwarp();
      select_largest(list, listed, best, k);
      if (lane < k) {
        const unsigned long long key = best[lane];
        a.top_ids[row * k + lane] = key_index(key);
        a.top_logp[row * k + lane] = empty ? -INFINITY : (key_value(key) - part.peak) - log_s;
      }
      __syncwarp();
    }
  }
}

struct LogprobGradArgs {
  const void* logits;
  const int64_t* targets;      // nullptr: none
  const float* peak;
  const float* log_sum;
  const float* entropy;        // nullptr unless g_entropy
  const float* g_logp;         // nullptr: none
  const float* g_entropy;      // nullptr: none
  void* dz;
  int64_t rows, cols, pitch, dz_pitch;
};

// The terms of a row that do not depend on the column.
struct RowGrad {
  float m, log_s, g, gh, h;
  int64_t target;              // -1: none
  bool zero;
};

__device__ __forceinline__ RowGrad row_grad(const LogprobGradArgs& a, int64_t row) {
  RowGrad r;
  r.m = a.peak[row];
  r.log_s = a.log_sum[row];
  r.target = a.targets ? a.targets[row] : -1;
  r.g = r.target >= 0 && a.g_logp ? a.g_logp[row] : 0.0f;
  if (r.target >= a.cols) {
    r.target = -1;
    r.g = NAN;
  }
  r.gh = a.g_entropy ? a.g_entropy[row] : 0.0f;
  r.h = a.g_entropy ? a.entropy[row] : 0.0f;
  r.zero = (r.m == -INFINITY && r.log_s == 0.0f) || (r.g == 0.0f && r.gh == 0.0f);
  return r;
}

// -p (g + gh (log p + H)); log p is held at -200 or more, where p is 0 and the product defined.
__device__ __forceinline__ float logit_grad(const RowGrad& r, float z) {
  const float lp = max_nan((z - r.m) - r.log_s, -200.0f);
  return -exp2_fast(lp * kLog2e) * fmaf(r.gh, lp + r.h, r.g);
}

// A CTA per stretch of kLpThreads * kLpWords words of a row.
template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprob_grad_kernel(LogprobGradArgs a) {
  constexpr int kVec = Word16<T>::kCount;
  const int cols = (int)a.cols;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const T* z = static_cast<const T*>(a.logits) + row * a.pitch;
    T* dz = static_cast<T*>(a.dz) + row * a.dz_pitch;
    const RowGrad r = row_grad(a, row);
    auto one = [&](int c) { dz[c] = r.zero ? from_float<T>(0.0f) : from_float<T>(logit_grad(r, to_float(z[c])) + (c == r.target ? r.g : 0.0f)); };
    if (((uintptr_t)z ^ (uintptr_t)dz) & 15) {            // the two rows lie differently between 16-byte boundaries
      const int begin = blockIdx.x * (kLpThreads * kLpWords * kVec);
#pragma unroll 4
      for (int i = 0; i < kLpWords * kVec; ++i) {
        const int c = begin + i * kLpThreads + threadIdx.x;
        if (c < cols) one(c);
      }
      continue;
    }
    const int to_boundary = (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T);
    const int head = to_boundary < cols ? to_boundary : cols;
    const int words = (cols - head) / kVec, tail = head + words * kVec;
    if (blockIdx.x == 0) {
      if ((int)threadIdx.x < head) one(threadIdx.x);
      if ((int)threadIdx.x < cols - tail) one(tail + threadIdx.x);
    }
    const uint4* from = reinterpret_cast<const uint4*>(z + head);
    uint4* to = reinterpret_cast<uint4*>(dz + head);
    const int first = blockIdx.x * (kLpThreads * kLpWords) + threadIdx.x;
    uint4 w[kLpWords];
    if (!r.zero) {
#pragma unroll
      for (int u = 0; u < kLpWords; ++u)
        if (first + u * kLpThreads < words) w[u] = load16_once(from + first + u * kLpThreads);
    }
#pragma unroll
    for (int u = 0; u < kLpWords; ++u) {
      const int i = first + u * kLpThreads;
      if (i >= words) break;
      if (r.zero) {
        to[i] = make_uint4(0u, 0u, 0u, 0u);
        continue;
      }
      float x[kVec];
      Word16<T>::unpack(w[u], x);
      const int64_t hit = r.target - (head + (int64_t)i * kVec);
#pragma unroll
      for (int j = 0; j < kVec; ++j) x[j] = logit_grad(r, x[j]);
      if (hit >= 0 && hit < kVec) {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (j == (int)hit) x[j] += r.g;
      }
      to[i] = Word16<T>::pack(x);
    }
  }
}

// CTAs per row: as many as bring the grid to four per SM, as long as each has an iteration's words to read.
static int logprob_cluster(int64_t rows, int64_t cols, size_t size, int sms) {
  int cluster = 1;
  while (cluster < kLpMaxCluster && rows * cluster * 2 <= (int64_t)sms * 4 && cols * (int64_t)size >= (int64_t)cluster * 2 * kLpChunk * 16) cluster *= 2;
  return cluster;
}

template <typename T, bool TOP>
static int logprob_launch_top(const LogprobArgs& a, int cluster, int sms, cudaStream_t stream) {
  constexpr size_t kSmem = (size_t)lp_stages<TOP> * kLpChunk * 16;
  SOLON_SHARED_MEMORY_ONCE((logprob_kernel<T, TOP>), kSmem);
  const int64_t resident = (int64_t)sms * kLpCtasPerSm / cluster;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((a.rows < resident ? a.rows : resident) * cluster));
  cfg.blockDim = dim3(kLpThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  SOLON_CUDA_TRY(cudaLaunchKernelEx(&cfg, logprob_kernel<T, TOP>, a));
  return SOLON_OK;
}

template <typename T, bool TOP>
static int logprob_launch_warps(const LogprobArgs& a, int sms, cudaStream_t stream) {
  constexpr size_t kPerWarp = lp_warp_stages<T, TOP> * 32 * lp_warp_words<T> * 16 + (TOP ? (kLpWarpList + SOLON_MAX_TOP) * 8 : 0);
  constexpr size_t kSmem = kLpWarps * kPerWarp;
  SOLON_SHARED_MEMORY_ONCE((logprob_warp_kernel<T, TOP>), kSmem);
  const int64_t resident = (int64_t)sms * lp_warp_ctas<T, TOP>;      // (a CTA may have fewer rows than warps: the SMs get equally many)
  logprob_warp_kernel<T, TOP><<<(unsigned)(a.rows < resident ? a.rows : resident), kLpThreads, kSmem, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T>
static int logprob_launch(const LogprobArgs& a, int sms, cudaStream_t stream) {
  if (logprob_by_warps(a.rows, a.cols, a.top_k > 0, sms))
    return a.top_k > 0 ? logprob_launch_warps<T, true>(a, sms, stream) : logprob_launch_warps<T, false>(a, sms, stream);
  const int cluster = logprob_cluster(a.rows, a.cols, sizeof(T), sms);
  return a.top_k > 0 ? logprob_launch_top<T, true>(a, cluster, sms, stream) : logprob_launch_top<T, false>(a, cluster, sms, stream);
}

template <typename T>
static int logprob_grad_launch(const LogprobGradArgs& a, cudaStream_t stream) {
  const int64_t stretch = (int64_t)kLpThreads * kLpWords * Word16<T>::kCount;
  const int64_t x = (a.cols + stretch - 1) / stretch;
  logprob_grad_kernel<T><<<dim3((unsigned)x, (unsigned)(a.rows < 65535 ? a.rows : 65535)), kLpThreads, 0, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

}  // namespace solon

using namespace solon;

extern "C" {

int solon_token_logprobs(const void* logits, int64_t pitch, int dtype, const int64_t* targets, int64_t rows, int64_t vocab, int top_k, float* logp,
                         float* entropy, float* peak, float* log_sum, int64_t* top_ids, float* top_logp, void* cuda_stream) {
  if (!token_dtype(dtype) || rows < 0 || vocab < 1 || vocab > SOLON_MAX_COLS) return SOLON_ERR_INVALID_ARG;
  if (top_k < 0 || top_k > SOLON_MAX_TOP || top_k > vocab || (top_k > 0 && rows > 0 && (!top_ids || !top_logp))) return SOLON_ERR_INVALID_ARG;
  if (rows == 0) return SOLON_OK;
  if (rows > 0x7FFFFFFF / kLpMaxCluster || !matrix_ok(logits, pitch, rows, vocab, dtype) || (logp && !targets)) return SOLON_ERR_INVALID_ARG;
  if (((uintptr_t)logp | (uintptr_t)entropy | (uintptr_t)peak | (uintptr_t)log_sum | (uintptr_t)top_logp) & 3 || ((uintptr_t)targets | (uintptr_t)top_ids) & 7)
    return SOLON_ERR_INVALID_ARG;
  int sms = 0, rc;
  if ((rc = current_sms(&sms))) return rc;
  const LogprobArgs a = {logits, targets, logp, entropy, peak, log_sum, top_ids, top_logp, rows, vocab, pitch, top_k};
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SOLON_F32) return logprob_launch<float>(a, sms, stream);
  if (dtype == SOLON_BF16) return logprob_launch<__nv_bfloat16>(a, sms, stream);
  return logprob_launch<__half>(a, sms, stream);
}

int solon_token_logprobs_backward(const void* logits, int64_t pitch, int dtype, const int64_t* targets, int64_t rows, int64_t vocab, const float* peak,
                                  const float* log_sum, const float* entropy, const float* grad_logp, const float* grad_entropy, void* dlogits, int64_t dlogits_pitch,
                                  void* cuda_stream) {
  if (!token_dtype(dtype) || rows < 0 || vocab < 1 || vocab > SOLON_MAX_COLS) return SOLON_ERR_INVALID_ARG;
  if ((grad_logp && !targets) || (grad_entropy && !entropy)) return SOLON_ERR_INVALID_ARG;
  if (rows == 0) return SOLON_OK;
  if (!matrix_ok(logits, pitch, rows, vocab, dtype) || !matrix_ok(dlogits, dlogits_pitch, rows, vocab, dtype) || !peak || !log_sum) return SOLON_ERR_INVALID_ARG;
  if (((uintptr_t)peak | (uintptr_t)log_sum | (uintptr_t)entropy | (uintptr_t)grad_logp | (uintptr_t)grad_entropy) & 3 || ((uintptr_t)targets & 7)) return SOLON_ERR_INVALID_ARG;
  if (logits == dlogits && pitch != dlogits_pitch && rows > 1) return SOLON_ERR_INVALID_ARG;
  const LogprobGradArgs a = {logits, targets, peak, log_sum, entropy, grad_logp, grad_entropy, dlogits, rows, vocab, pitch, dlogits_pitch};
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SOLON_F32) return logprob_grad_launch<float>(a, stream);
  if (dtype == SOLON_BF16) return logprob_grad_launch<__nv_bfloat16>(a, stream);
  return logprob_grad_launch<__half>(a, stream);
}

}  // extern "C"
