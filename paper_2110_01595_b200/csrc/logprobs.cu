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
// gradient; a target beyond the vocabulary is not read and has logp NaN; NaN and +infinity make the row's results NaN.
#include <math.h>

#include "elements.cuh"
#include "solon_internal.h"
#include "token_args.h"

namespace solon {

// Bound by memory, with the exponentials close behind (one a logit: at 16 a clock and SM 60 % of the time that bfloat16 logits
// take to arrive), so the arithmetic beside them is kept short: two values an instruction where there is one for it, sums
// against a reference value that need not be the maximum, and one comparison per 16 bytes for everything that is rare.
constexpr int kLpThreads = 256;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpUnroll = 4;                   // 16-byte words a thread has in flight
constexpr int kLpMaxCluster = 8;
constexpr int kLpCandidates = 2048;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Order of the likeliest tokens as one integer: value first (NaN above all, -0 = +0), of equal values the lower index.
__device__ __forceinline__ uint32_t order_bits(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return z != z ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : (b | 0x80000000u);      // > 0 for every value
}
__device__ __forceinline__ unsigned long long rank_key(float z, uint32_t index) {
  return ((unsigned long long)order_bits(z) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long key) { return 0xFFFFFFFFu - (uint32_t)key; }
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return o == 0xFFFFFFFFu ? NAN : __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

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

// Softmax sums of a part of a row: largest logit, and against a reference r (in base 2, t = (z - r) log2 e)
// s = sum 2^t, a = sum 2^t t.
struct SoftmaxPart {
  float peak, ref, s, a;
};

// The same sums against another reference: t' = t + d, d = (r - r') log2 e.  A part whose terms all vanish adds nothing; one
// without terms has no reference to move from.
__device__ __forceinline__ void shift_part(SoftmaxPart& p, float ref) {
  if (p.s == 0.0f) {
    p.ref = ref;
    return;
  }
  const float d = (p.ref - ref) * kLog2e, f = exp2_fast(d);
  p.a = f > 0.0f ? f * (p.a + d * p.s) : (p.s != p.s ? p.s : 0.0f);
  p.s *= f;
  p.ref = ref;
}

// What a thread carries through its share of a row.  Sums run against `ref`, one of the values seen; it is replaced (and the
// sums rescaled) only when a value exceeds it by 8 in base 2, which spares the rescaling in almost every word and costs the
// sums nothing but a factor of at most 256.  `peak` is the largest value itself.
struct LogprobThread {
  float peak, ref, limit;      // limit: values above it need the reference moved (-infinity until there is a reference)
  Float2 s, a;

  __device__ __forceinline__ void init() {
    peak = -INFINITY;
    ref = 0.0f;
    limit = -INFINITY;
    s = a = pack2(0.0f, 0.0f);
  }
  __device__ __forceinline__ SoftmaxPart part() const {
    float s0, s1, a0, a1;
    unpack2(s, s0, s1);
    unpack2(a, a0, a1);
    return {peak, ref, s0 + s1, a0 + a1};
  }
  __device__ __forceinline__ void move_reference(float to) {
    SoftmaxPart p = part();
    shift_part(p, to);
    if (!(to < INFINITY)) p.s = NAN;             // +infinity or NaN: the row has no softmax
    s = pack2(p.s, 0.0f);
    a = pack2(p.a, 0.0f);
    ref = to;
    limit = to + 8.0f / kLog2e;
  }
  // N values of which none is above `limit`.  t is held at -200 or more, where 2^t is 0 and t 2^t defined.
  template <int N>
  __device__ __forceinline__ void add(const float (&z)[N]) {
    const Float2 minus_ref = pack2(-ref, -ref), scale = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float t0, t1;
      unpack2(mul2(add2(pack2(z[i], z[i + 1]), minus_ref), scale), t0, t1);
      t0 = max_nan(t0, -200.0f);
      t1 = max_nan(t1, -200.0f);
      const Float2 e = pack2(exp2_fast(t0), exp2_fast(t1));
      s = add2(s, e);
      a = fma2(e, pack2(t0, t1), a);
    }
  }
};

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
// threshold is the k-th largest of the maxima of 32 groups of eight threads, taken anew whenever the part of the row that
// has been seen has doubled, with all threads at the same place of the row.  The k largest are picked from the candidates at
// the end.  Should they overflow (a row that rises throughout), the k largest are found by going through the row k times.
struct LogprobTop {
  unsigned long long key[kLpCandidates];
  unsigned long long best[SOLON_MAX_TOP];      // this CTA's k largest, in falling order (0: fewer)
  unsigned long long scratch[kLpWarps];
  uint32_t group_max[32];
  float threshold;
  uint32_t threshold_order;
  int count;
};

__device__ __forceinline__ void push_candidate(LogprobTop& top, float z, uint32_t index) {
  const int at = atomicAdd(&top.count, 1);
  if (at < kLpCandidates) top.key[at] = rank_key(z, index);
}

// New threshold from the threads' maxima (order bits, 0: has seen nothing).  All threads call it, at the same place of the row.
__device__ __forceinline__ void refresh_threshold(LogprobTop& top, uint32_t seen, int k) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) seen = max(seen, __shfl_xor_sync(0xffffffffu, seen, off));
  if ((lane & 7) == 0) top.group_max[warp * 4 + (lane >> 3)] = seen;
  __syncthreads();
  if (warp == 0) {
    const uint32_t mine = top.group_max[lane];
    int rank = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const uint32_t other = __shfl_sync(0xffffffffu, mine, j);
      rank += other > mine || (other == mine && j < lane);
    }
    if (rank == k - 1) {
      top.threshold_order = mine;
      top.threshold = key_value((unsigned long long)mine << 32);
    }
  }
  __syncthreads();
}

// Sorts the largest k of n keys (all different, beside zeros) into out, zeros behind them.
__device__ __forceinline__ void select_largest(const unsigned long long* keys, int n, unsigned long long* out, int k) {
  for (int i = threadIdx.x; i < k; i += kLpThreads) out[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kLpThreads) {
    const unsigned long long mine = keys[i];
    if (mine == 0) continue;
    int rank = 0;
    for (int j = 0; j < n && rank < k; ++j) rank += keys[j] > mine;
    if (rank < k) out[rank] = mine;
  }
  __syncthreads();
}

// A row is read by a cluster of 1 to 8 CTAs, each taking a stretch of it.  Elements before the row's first and behind its last
// 16-byte boundary go one by one to the first and the last CTA.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kLpThreads, 4) logprob_kernel(LogprobArgs a) {
  constexpr int kVec = Word16<T>::kCount;
  constexpr int kChunk = kLpThreads * kLpUnroll;          // words of an iteration
  __shared__ SoftmaxPart warp_part[kLpWarps];
  __shared__ SoftmaxPart cta_part;
  __shared__ float row_stats[2];                          // peak, log sum
  __shared__ __align__(16) unsigned char top_bytes[TOP ? sizeof(LogprobTop) : 16];
  LogprobTop& top = *reinterpret_cast<LogprobTop*>(top_bytes);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const int64_t row = blockIdx.x / size;
  const T* z = static_cast<const T*>(a.logits) + row * a.pitch;
  const int cols = (int)a.cols;
  const int to_boundary = (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T);
  const int head = to_boundary < cols ? to_boundary : cols;
  const int words = (cols - head) / kVec;
  const int begin = (int)((int64_t)words * rank / size), end = (int)((int64_t)words * (rank + 1) / size);
  const uint4* body = reinterpret_cast<const uint4*>(z + head);

  LogprobThread t;
  t.init();
  auto add_one = [&](int c) {                             // an element outside the words
    const float v = to_float(z[c]);
    t.peak = fmaxf(t.peak, v);
    if (!(v <= t.limit)) t.move_reference(v);
    const float pair[2] = {v, -INFINITY};
    t.add(pair);
    if (TOP) push_candidate(top, v, (uint32_t)c);
  };
  if (TOP) {
    if (threadIdx.x == 0) top.count = 0;
    __syncthreads();
  }
  if (rank == 0 && (int)threadIdx.x < head) add_one(threadIdx.x);

  float threshold = -INFINITY;                            // candidates are above it; +infinity in a sweep without candidates
  auto add_word = [&](const uint4& w, int index, bool candidates) {
    const float big = Word16<T>::largest(w);
    float x[kVec];
    Word16<T>::unpack(w, x);
    t.peak = fmaxf(t.peak, big);
    if (!(big <= t.limit)) t.move_reference(big);
    t.add(x);
    if (TOP && candidates && !(big <= threshold)) {
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (!(x[j] <= threshold)) push_candidate(top, x[j], (uint32_t)(head + index * kVec + j));
    }
  };

  int next_refresh = 1, iteration = 0;
  for (int base = begin; base < end; base += kChunk, ++iteration) {
    uint4 w[kLpUnroll];
    if (base + kChunk <= end) {
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u) w[u] = load16_once(body + base + u * kLpThreads + threadIdx.x);
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u) add_word(w[u], base + u * kLpThreads + threadIdx.x, iteration > 0);
    } else {
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u) {
        const int i = base + u * kLpThreads + threadIdx.x;
        if (i < end) w[u] = load16_once(body + i);
      }
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u) {
        const int i = base + u * kLpThreads + threadIdx.x;
        if (i < end) add_word(w[u], i, iteration > 0);
      }
    }
    if constexpr (TOP) {
      if (iteration == 0) {
        // the first stretch is compared with its own threshold, so values equal to it count too; where they are many (a
        // masked row), only those of the first 1024 elements, if that leaves k
        refresh_threshold(top, begin + (int)threadIdx.x < end ? order_bits(t.peak) : 0u, a.top_k);
        const uint32_t at_least = top.threshold_order;
        const int before = top.count;
        __syncthreads();
        for (int pass = 0; pass < 2; ++pass) {
          const int ties_until = pass == 0 ? 0x7FFFFFFF : begin * kVec + 1024;
#pragma unroll
          for (int u = 0; u < kLpUnroll; ++u) {
            const int i = base + u * kLpThreads + threadIdx.x;
            if (i < end) {
              float x[kVec];
              Word16<T>::unpack(w[u], x);
#pragma unroll
              for (int j = 0; j < kVec; ++j) {
                const uint32_t o = order_bits(x[j]);
                if (o > at_least || (o == at_least && i * kVec + j < ties_until)) push_candidate(top, x[j], (uint32_t)(head + i * kVec + j));
              }
            }
          }
          __syncthreads();
          const int found = top.count;
          __syncthreads();
          if (found <= kLpCandidates || pass == 1) {
            // (too few after the second pass cannot pass for a result: the count says overflow)
            if (pass == 1 && found - before < a.top_k && threadIdx.x == 0) top.count = kLpCandidates + 1;
            break;
          }
          if (threadIdx.x == 0) top.count = before;
          __syncthreads();
        }
        __syncthreads();
        threshold = top.threshold;
        next_refresh = 2;
      } else if (iteration + 1 == next_refresh && base + kChunk < end) {
        refresh_threshold(top, order_bits(t.peak), a.top_k);
        threshold = top.threshold;
        next_refresh *= 2;
      }
    }
  }

  // behind everything else: the threshold takes what it has seen to be of lower index than what it is compared with
  if (rank == size - 1 && (int)threadIdx.x < cols - head - words * kVec) add_one(head + words * kVec + threadIdx.x);

  // the CTA's sums: everything against the warp's, then the CTA's largest value
  SoftmaxPart p = t.part();
  float peak = p.peak;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) peak = fmaxf(peak, __shfl_xor_sync(0xffffffffu, peak, off));
  p.peak = peak;
  if (peak > -INFINITY) shift_part(p, peak);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    p.s += __shfl_xor_sync(0xffffffffu, p.s, off);
    p.a += __shfl_xor_sync(0xffffffffu, p.a, off);
  }
  if (lane == 0) warp_part[warp] = p;
  __syncthreads();
  auto join = [](SoftmaxPart& sum, SoftmaxPart q, float to) {
    if (to > -INFINITY) shift_part(q, to);
    sum.s += q.s;
    sum.a += q.a;
  };
  SoftmaxPart cta = {-INFINITY, 0.0f, 0.0f, 0.0f};
  if (threadIdx.x == 0) {
    for (int i = 0; i < kLpWarps; ++i) cta.peak = fmaxf(cta.peak, warp_part[i].peak);
    cta.ref = cta.peak;
    for (int i = 0; i < kLpWarps; ++i) join(cta, warp_part[i], cta.peak);
    cta_part = cta;
  }

  if constexpr (TOP) {
    __syncthreads();
    const int count = top.count;
    if (count <= kLpCandidates) {
      select_largest(top.key, count, top.best, a.top_k);
    } else {
      unsigned long long last = ~0ull;
      for (int k = 0; k < a.top_k; ++k) {                 // the largest key below the one before
        unsigned long long best = 0;
        const int first = rank == 0 ? 0 : head + begin * kVec, behind = rank == size - 1 ? cols : head + end * kVec;
        for (int c = first + threadIdx.x; c < behind; c += kLpThreads) {
          const unsigned long long key = rank_key(to_float(z[c]), (uint32_t)c);
          if (key < last && key > best) best = key;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, off));
        if (lane == 0) top.scratch[warp] = best;
        __syncthreads();
        for (int i = 0; i < kLpWarps; ++i) best = max(best, top.scratch[i]);
        if (threadIdx.x == 0) top.best[k] = best;
        last = best;
        __syncthreads();
      }
    }
  }

  if (size > 1) cluster_barrier();
  if (rank == 0) {
    if (threadIdx.x == 0) {
      for (uint32_t r = 1; r < size; ++r) {
        const uint32_t at = peer_address(&cta_part, r);
        const SoftmaxPart q = {peer_float(at), peer_float(at + 4), peer_float(at + 8), peer_float(at + 12)};
        const float big = fmaxf(cta.peak, q.peak);
        if (big > -INFINITY) shift_part(cta, big);
        cta.peak = big;
        join(cta, q, big);
      }
      const bool empty = cta.peak == -INFINITY && cta.s == 0.0f;
      const float log_s = empty ? 0.0f : logf(cta.s);
      row_stats[0] = cta.peak;
      row_stats[1] = log_s;
      if (a.peak) a.peak[row] = cta.peak;
      if (a.log_sum) a.log_sum[row] = log_s;
      if (a.entropy) a.entropy[row] = empty ? 0.0f : log_s - kLn2 * (cta.a / cta.s);
      if (a.targets && a.logp) {
        const int64_t target = a.targets[row];
        float lp = 0.0f;
        if (target >= a.cols) lp = NAN;
        else if (target >= 0) lp = empty ? -INFINITY : (to_float(z[target]) - cta.peak) - log_s;
        a.logp[row] = lp;
      }
    }
    if constexpr (TOP) {
      __syncthreads();
      if (size > 1) {
        for (int i = threadIdx.x; i < (int)size * a.top_k; i += kLpThreads) top.key[i] = peer_key(peer_address(&top.best[i % a.top_k], i / a.top_k));
        __syncthreads();
        select_largest(top.key, (int)size * a.top_k, top.best, a.top_k);
      }
      for (int i = threadIdx.x; i < a.top_k; i += kLpThreads) {
        const unsigned long long key = top.best[i];
        a.top_ids[row * a.top_k + i] = key_index(key);
        a.top_logp[row * a.top_k + i] = row_stats[0] == -INFINITY && row_stats[1] == 0.0f ? -INFINITY : (key_value(key) - row_stats[0]) - row_stats[1];
      }
    }
  }
  if (size > 1) cluster_barrier();        // the first CTA has read the others' shared memory
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

// A CTA per stretch of kLpThreads * kLpUnroll words of a row.
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
      const int begin = blockIdx.x * (kLpThreads * kLpUnroll * kVec);
#pragma unroll 4
      for (int i = 0; i < kLpUnroll * kVec; ++i) {
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
    const int first = blockIdx.x * (kLpThreads * kLpUnroll) + threadIdx.x;
    uint4 w[kLpUnroll];
    if (!r.zero) {
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u)
        if (first + u * kLpThreads < words) w[u] = load16_once(from + first + u * kLpThreads);
    }
#pragma unroll
    for (int u = 0; u < kLpUnroll; ++u) {
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
  while (cluster < kLpMaxCluster && rows * cluster * 2 <= (int64_t)sms * 4 && cols * (int64_t)size >= (int64_t)cluster * 2 * kLpThreads * kLpUnroll * 16) cluster *= 2;
  return cluster;
}

template <typename T, bool TOP>
static int logprob_launch_top(const LogprobArgs& a, int cluster, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.rows * cluster));
  cfg.blockDim = dim3(kLpThreads);
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

template <typename T>
static int logprob_launch(const LogprobArgs& a, int sms, cudaStream_t stream) {
  const int cluster = logprob_cluster(a.rows, a.cols, sizeof(T), sms);
  return a.top_k > 0 ? logprob_launch_top<T, true>(a, cluster, stream) : logprob_launch_top<T, false>(a, cluster, stream);
}

template <typename T>
static int logprob_grad_launch(const LogprobGradArgs& a, cudaStream_t stream) {
  const int64_t stretch = (int64_t)kLpThreads * kLpUnroll * Word16<T>::kCount;
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
