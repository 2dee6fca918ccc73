// AdamW over all tensors of a model at once (solon_adamw_*): what a parameter server does with the aggregate that
// solon_decode returns.  Per weight, with g' = grad_scale * clip * g:
//     m <- b1 m + (1 - b1) g'          v <- b2 v + (1 - b2) g'^2
//     p <- p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// All of it in float32; b1^t and b2^t are kept in float64 on the device, so that a replayed CUDA graph counts its steps.  The
// moments are formed as written, every product and sum rounded by itself (g' = (grad_scale g) clip, ((1 - b2) g') g', no
// multiply-adds): the 8-bit state's codes can hang on a moment's last bit, and so they are those of one elementary operation
// after the other.  (With multiply-adds 9 to 19 codes of 50 M came out otherwise per step, and a quarter of the moments in their last bit.)
//
// Bound by memory: a weight with float32 gradient moves 28 bytes (32-bit states) or 16 (8-bit states) against about 20 flops.
// Measured on 50 M weights: 32-bit states 204 us (6.9 TB/s); 8-bit states 144 to 147 us (5.5 TB/s; codes and random bits keep the
// integer pipe busy 61 % of the time), with float64 gradients 155 to 158 us (6.4 TB/s); the norm 65 us of 400 MB of float64
// gradients, 31 us of float32 ones, which the update then partly finds in L2.
//
// Work: the state is laid out in blocks of 256 elements, every tensor starting a block of its own; one warp owns a block, one
// CTA eight consecutive blocks of a tensor (a chunk).  Three launches at most: the gradient's squared norm (only when it is
// clipped), one CTA that turns it into the clip factor, checks the guard and counts the step, and the update itself.
#include <math.h>

#include <new>

#include "elements.cuh"
#include "solon_internal.h"

namespace solon {

constexpr int kAdamBlock = 256;                        // elements of a state block (one warp, eight per lane)
constexpr int kAdamChunkBlocks = 8;                    // blocks of a chunk (one CTA of eight warps)
constexpr int kAdamThreads = 32 * kAdamChunkBlocks;
constexpr int kAdamChunk = kAdamBlock * kAdamChunkBlocks;

// All that a CTA needs to know of its chunk, in one 64-byte record: one trip to memory before the data, not two.
struct alignas(64) AdamChunk {
  float* p;                  // the chunk's first element
  __nv_bfloat16* copy;       // nullptr: none
  const void* grad;          // bound gradient of the chunk's first element
  int64_t offset;            // first element in the concatenated order
  int64_t slot;              // first element in the state
  int count;                 // elements
  float weight_decay;
  int starts;                // the tensor's first chunk
  int behind;                // elements of the tensor behind the chunk, up to three
};

// What the update reads, written by the control kernel of the same step.
struct AdamScalars {
  double b1t, b2t;           // b1^t, b2^t of the last step that was applied
  long long applied, skipped;
  float inv_bc1, inv_sqrt_bc2, grad_scale, clip;      // (the first two with the quotient's power of two)
  int skip;
  unsigned key;              // of the step's random words
};

}  // namespace solon

struct solon_adamw {
  int n_tensors, bits, device, num_sms;
  double beta1, beta2, eps;
  uint64_t seed;
  int64_t total, n_blocks, n_chunks;
  int grads_bound, grad_dtype;             // bound gradients and their type
  void *exp_avg, *exp_avg_sq;
  int16_t* base;
  std::vector<int64_t> numel;
  std::vector<solon::AdamChunk> chunks;
  solon::AdamChunk* d_chunks;
  solon::AdamScalars* d_scalars;
  double* d_partials;                      // norm kernel: one sum per CTA
  int norm_grid;
};

namespace solon {

// MurmurHash3's 32-bit finaliser (Appleby): every input bit reaches every output bit.
__host__ __device__ __forceinline__ uint32_t mix32_but_last(uint32_t h) {
  h ^= h >> 16;
  h *= 0x85EBCA6Bu;
  h ^= h >> 13;
  return h * 0xC2B2AE35u;
}
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t h) {
  h = mix32_but_last(h);
  return h ^ (h >> 16);
}

// The 32 random bits of a state slot in a step are mix32((hash start of the slot) ^ key), key: step and seed; the low half
// rounds m, the high half v.  Slots 0 .. n behind one add n kSlotFactor to its start (a block of 256 does not cross 2^32).
constexpr uint32_t kSlotFactor = 0x9E3779B1u;
__device__ __forceinline__ uint32_t slot_hash_start(int64_t slot) {
  return (uint32_t)slot * kSlotFactor + (uint32_t)((uint64_t)slot >> 32) * 0x85EBCA77u;
}

// ---- the 8-bit state -------------------------------------------------------------------------------------------
// The float32 numbers with three mantissa bits are those whose low 20 bits are zero; their rank is bits >> 20.  A block
// of 256 values holds `base` and, per value, an 8-bit code: rank - base, 0 for zero.  The window of 127 (m, beside its
// sign) or 255 (v) ranks ends at the block's largest magnitude, rounded up: 15.9 and 31.9 binades, the same range of
// gradients for both.  Because the grid is the same for every block, a window that moves with the block's maximum
// re-rounds nothing.
//
// Rounding is stochastic: 16 random bits, added to the upper 16 of the 20 that are cut (within a binade, and across its end, a
// float's value is linear in its bits).  The four lowest bits take no part, so the mean of a rounding is off by at most 15 / 2^20
// of a grid step, towards 0.  Rounding to nearest would leave v standing still: with b2 = 0.999 a step moves it by up to
// 0.1 %, half a grid step is 3 - 6 %.  Two exceptions: what lies below the window becomes 0 for m and the smallest code for
// v, which is never 0 unless v is - a zero v under a moving m would divide by eps.  Non-finite values take the top code
// and have no part in the choice of the window, so they spoil no other element of their block.
constexpr uint32_t kTopFinite = 0x7F7u;                // rank of the largest finite value of the grid

// Largest finite magnitude of the block as bits (float order = integer order for non-negative floats).
__device__ __forceinline__ uint32_t finite_bits(uint32_t bits) { return bits < 0x7F800000u ? bits : 0u; }

__device__ __forceinline__ int window_base(uint32_t max_bits, uint32_t levels) {
  uint32_t top = (max_bits + 0xFFFFFu) >> 20;
  top = top < kTopFinite ? top : kTopFinite;
  return top > levels ? (int)(top - levels) : 0;
}

__device__ __forceinline__ int state_code(uint32_t bits, uint32_t random20, int base, int levels) {
  const int code = (int)((bits + random20) >> 20) - base;
  return code < levels ? code : levels;
}

// ---- control: one CTA before the update -----------------------------------------------------------------------------

struct AdamControlArgs {
  AdamScalars* s;
  const double* partials;      // squared norm of the unscaled gradient, per CTA of the norm kernel
  int n_partials;              // 0: no clipping
  float* norm_out;             // nullptr: not wanted
  double grad_scale, max_norm, beta1, beta2;
  double quotient_scale;       // a power of two for both sides of the step's quotient (its eps has it already)
  uint64_t seed;
  const int* guard_status;     // plan's status words (nullptr: no guard)
  const int* guard_t;          // per group: accepted error count, -1 undecodable
  int guard_groups;
};

__global__ void __launch_bounds__(256) adam_control_kernel(AdamControlArgs a) {
  __shared__ double part_s[8];
  pdl_trigger();
  pdl_wait();
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.n_partials; i += 256) sum += a.partials[i];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  if ((threadIdx.x & 31) == 0) part_s[threadIdx.x >> 5] = sum;
  int bad = 0;
  if (a.guard_t) {
    for (int i = threadIdx.x; i < a.guard_groups; i += 256) bad |= a.guard_t[i] < 0;
    if (threadIdx.x < 2) bad |= a.guard_status[threadIdx.x] & kStatusWaitExpired;
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x != 0) return;
  double scale = a.grad_scale;
  float clip = 1.0f;
  if (a.n_partials > 0) {
    sum = 0.0;
    for (int w = 0; w < 8; ++w) sum += part_s[w];
    const double norm = sqrt(sum) * fabs(a.grad_scale);
    if (a.norm_out) *a.norm_out = (float)norm;
    if (!(norm < INFINITY)) bad = 1;               // NaN or infinite: there is nothing to clip to
    // From the norm that is handed back, in float32 like everything that the moments are made of.  Beyond its range in float64,
    // with a power of two moved from one factor to the other: the clip factor alone could be subnormal.
    const float narrow = (float)norm;
    if (narrow < INFINITY) {
      clip = fminf(__fmul_rn((float)a.max_norm, __frcp_rn(__fadd_rn(narrow, 1e-6f))), 1.0f);
    } else {
      clip = (float)(fmin(a.max_norm / norm, 1.0) * 0x1p64);
      scale *= 0x1p-64;
    }
  }
  AdamScalars* s = a.s;
  s->skip = bad;
  if (bad) {
    s->skipped += 1;
    return;
  }
  const double b1t = s->b1t * a.beta1, b2t = s->b2t * a.beta2;
  const long long t = s->applied + 1;
  s->b1t = b1t;
  s->b2t = b2t;
  s->applied = t;
  s->inv_bc1 = (float)(a.quotient_scale / (1.0 - b1t));
  s->inv_sqrt_bc2 = (float)(a.quotient_scale / sqrt(1.0 - b2t));
  s->grad_scale = (float)scale;
  s->clip = clip;
  s->key = mix32((uint32_t)t * 0x9E3779B1u + (uint32_t)a.seed) ^ (uint32_t)(a.seed >> 32);
}

// ---- squared norm of the gradient ----------------------------------------------------------------------------------
// Squares and sums in float64 (of the values rounded to float32, as the update takes them), so that neither a square overflows
// nor the order of the sums shows in the result.  A conversion and a multiply-add per element stay below the time that the
// gradient takes to arrive.

__device__ __forceinline__ void norm_finish(double acc, double* partials) {
  __shared__ double part_s[kAdamChunkBlocks];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
  if ((threadIdx.x & 31) == 0) part_s[threadIdx.x >> 5] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int w = 0; w < kAdamChunkBlocks; ++w) total += part_s[w];
    partials[blockIdx.x] = total;
  }
}

// A flat gradient: eight 16-byte words a thread at a time (50 M float64: 64 us, with four 93), of two-byte elements four (50 M: 23
// us, with eight, which spill, 49), a contiguous stretch per CTA and turn.
template <typename G>
__global__ void __launch_bounds__(kAdamThreads, 4) adam_norm_flat_kernel(const G* __restrict__ grad, int64_t n, double* __restrict__ partials) {
  constexpr int kVec = 16 / sizeof(G);
  constexpr int kUnroll = sizeof(G) == 2 ? 4 : 8;
  pdl_trigger();
  pdl_wait();
  const int64_t to_boundary = (int64_t)((16 - ((uintptr_t)grad & 15)) & 15) / (int64_t)sizeof(G);
  const int64_t head = to_boundary < n ? to_boundary : n;
  const int64_t words = (n - head) / kVec, tail = head + words * kVec;
  const G* body = grad + head;
  double acc = 0.0;
  if (blockIdx.x == 0) {
    double x = (int64_t)threadIdx.x < head ? (double)to_float(grad[threadIdx.x]) : 0.0;
    acc = x * x;
    x = (int64_t)threadIdx.x < n - tail ? (double)to_float(grad[tail + threadIdx.x]) : 0.0;
    acc = fma(x, x, acc);
  }
  double part[kVec];
#pragma unroll
  for (int k = 0; k < kVec; ++k) part[k] = 0.0;
  for (int64_t base = (int64_t)blockIdx.x * kAdamThreads * kUnroll; base < words; base += (int64_t)gridDim.x * kAdamThreads * kUnroll) {
    Pack<G, kVec> v[kUnroll];
    const int64_t first = base + threadIdx.x;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (first + u * kAdamThreads < words) v[u] = load_pack<G, kVec>(body + (first + u * kAdamThreads) * kVec);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (first + u * kAdamThreads < words) {
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          const double x = (double)to_float(v[u].e[k]);
          part[k] = fma(x, x, part[k]);
        }
      }
  }
#pragma unroll
  for (int k = 0; k < kVec; ++k) acc += part[k];
  norm_finish(acc, partials);
}

// Gradients in tensors of their own: chunk by chunk, one element a thread and access (50 M float32, step with clipping: 252 us, from
// a flat gradient 235; 8-bit states 195 and 180).
template <typename G>
__global__ void __launch_bounds__(kAdamThreads) adam_norm_bound_kernel(const AdamChunk* __restrict__ chunks, int64_t n_chunks, double* __restrict__ partials) {
  pdl_trigger();
  pdl_wait();
  double acc = 0.0;
  for (int64_t c = blockIdx.x; c < n_chunks; c += gridDim.x) {
    const G* g = static_cast<const G*>(chunks[c].grad);
    const int left = chunks[c].count;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = i * kAdamThreads + threadIdx.x;
      x[i] = e < left ? to_float(g[e]) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = fma((double)x[i], (double)x[i], acc);
  }
  norm_finish(acc, partials);
}

// ---- the update ------------------------------------------------------------------------------------------------------

struct AdamStepArgs {
  const AdamChunk* chunks;
  const void* flat;            // nullptr: the chunks' bound gradients
  void* exp_avg;
  void* exp_avg_sq;
  int16_t* base;               // two per block: m's, v's (8-bit states)
  const AdamScalars* scalars;
  float beta1, one_minus_beta1, beta2, one_minus_beta2, eps, lr;
};

// How a warp goes through its block.  A lane has two groups of four consecutive elements; where parameters or gradients do not
// start on the groups' boundaries (tensors that are pieces of one vector, at any offset: what the aggregate's users have), a
// group is put together from the two aligned words that hold it, and parameters go back as aligned words too.  Single
// accesses of four bytes move the same bytes in four times as many requests, which caps what is on the way: 11.2 M weights of
// an odd offset take 63 us that way, 55 us from aligned words, 49 us where they are aligned.  The aligned words reach up to three
// elements beyond the block, so a tensor's first block, full blocks with fewer than three elements of the tensor behind them, and
// blocks that are not full go element by element (every 32nd a lane's).
enum BlockMode { kSingle, kAligned, kShifted };

template <bool VEC>
__device__ __forceinline__ int lane_element(int lane, int i) {
  return VEC ? ((i >> 2) * 32 + lane) * 4 + (i & 3) : i * 32 + lane;
}

// Four consecutive elements at p from 16-byte words; delta: elements from the word that holds the first to p.
__device__ __forceinline__ void select4(float (&x)[4], const float4& a, const float4& b, int delta) {
  const float e[7] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z};
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = delta < 2 ? (delta == 0 ? e[k] : e[k + 1 < 7 ? k + 1 : 6]) : (delta == 2 ? e[k + 2 < 7 ? k + 2 : 6] : e[k + 3]);
}
template <typename T>
__device__ __forceinline__ void load8_shifted(T (&x)[8], const T* p, int lane) {
  if constexpr (sizeof(T) == 4) {
    const int delta = (int)(((uintptr_t)p >> 2) & 3);
    const float4* w = reinterpret_cast<const float4*>(p - delta);
    float4 a[2], b[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      a[h] = w[h * 32 + lane];
      b[h] = w[h * 32 + lane + (delta ? 1 : 0)];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float q[4];
      select4(q, a[h], b[h], delta);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[h * 4 + k] = q[k];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[lane_element<true>(lane, i)];
  }
}
// Word j of the shifted block holds the last delta elements of group j - 1 and the first 4 - delta of group j; the block's first
// and last word are shared with its neighbours, so their elements go one by one.
__device__ __forceinline__ void store8_shifted(float* p, const float (&x)[8], int lane) {
  const int delta = (int)(((uintptr_t)p >> 2) & 3);
  float4* w = reinterpret_cast<float4*>(p - delta);
  if (delta == 0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h * 32 + lane] = make_float4(x[h * 4], x[h * 4 + 1], x[h * 4 + 2], x[h * 4 + 3]);
    return;
  }
  float before[2][3];                          // elements 1 .. 3 of the group before
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float last = __shfl_sync(0xffffffffu, x[k + 1], 31);
#pragma unroll
    for (int h = 0; h < 2; ++h) before[h][k] = __shfl_up_sync(0xffffffffu, x[h * 4 + k + 1], 1);
    if (lane == 0) before[1][k] = last;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float e[7] = {before[h][0], before[h][1], before[h][2], x[h * 4], x[h * 4 + 1], x[h * 4 + 2], x[h * 4 + 3]};
    float q[4];                                // elements -delta .. 3 - delta of the group
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = delta == 1 ? e[k + 2 < 7 ? k + 2 : 6] : delta == 2 ? e[k + 1] : e[k];
    if (h > 0 || lane > 0) w[h * 32 + lane] = make_float4(q[0], q[1], q[2], q[3]);
  }
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (k < 4 - delta) p[k] = x[k];
  }
  if (lane == 31) {
#pragma unroll
    for (int k = 1; k < 4; ++k)
      if (k >= 4 - delta) p[252 + k] = x[4 + k];
  }
}

template <bool VEC, typename T>
__device__ __forceinline__ void load8(T (&x)[8], const T* p, int lane, int n) {
  if constexpr (VEC) {
    constexpr int kVec = sizeof(T) <= 4 ? 4 : 2;       // at most 16 bytes an access
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 4 / kVec; ++q) {
        const Pack<T, kVec> v = load_pack<T, kVec>(p + (h * 32 + lane) * 4 + q * kVec);
#pragma unroll
        for (int k = 0; k < kVec; ++k) x[h * 4 + q * kVec + k] = v.e[k];
      }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = i * 32 + lane;
      x[i] = e < n ? p[e] : T(0.0f);
    }
  }
}

template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, const T (&x)[8], int lane, int n) {
  if constexpr (VEC) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      Pack<T, 4> v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v.e[k] = x[h * 4 + k];
      store_pack<T, 4>(p + (h * 32 + lane) * 4, v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = i * 32 + lane;
      if (e < n) p[e] = x[i];
    }
  }
}

// The hardware's square root and quotient (one and two units in the last place): the update is rounded by far less than
// the state's own width, and the exact forms cost a quarter of the 8-bit step's instructions.  The quotient asks for a denominator
// between 2^-126 and 2^126 (above, it is 0): sqrt(v) stays below 2^64 and its factor below 2^27, so only eps can leave that range;
// then both sides carry a power of two (solon_adamw_step).
__device__ __forceinline__ float sqrt_fast(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A lane's eight codes of m and of v: two 32-bit words of four neighbours each (VEC), or eight single bytes.
template <bool VEC>
struct LaneCodes {
  uint32_t m[VEC ? 2 : 8], v[VEC ? 2 : 8];

  __device__ __forceinline__ void load(const uint8_t* mp, const uint8_t* vp, int lane) {
#pragma unroll
    for (int i = 0; i < (VEC ? 2 : 8); ++i) {
      m[i] = VEC ? reinterpret_cast<const uint32_t*>(mp)[i * 32 + lane] : mp[i * 32 + lane];
      v[i] = VEC ? reinterpret_cast<const uint32_t*>(vp)[i * 32 + lane] : vp[i * 32 + lane];
    }
  }
  __device__ __forceinline__ void store(uint8_t* mp, uint8_t* vp, int lane) const {
#pragma unroll
    for (int i = 0; i < (VEC ? 2 : 8); ++i) {
      if constexpr (VEC) {
        reinterpret_cast<uint32_t*>(mp)[i * 32 + lane] = m[i];
        reinterpret_cast<uint32_t*>(vp)[i * 32 + lane] = v[i];
      } else {
        mp[i * 32 + lane] = (uint8_t)m[i];
        vp[i * 32 + lane] = (uint8_t)v[i];
      }
    }
  }
  // Whether no code in the warp stands for zero (nearly always so: every weight that has had a gradient).
  __device__ __forceinline__ bool none_zero() const {
    uint32_t all = 0x80808080u;
#pragma unroll
    for (int i = 0; i < (VEC ? 2 : 8); ++i) {      // the top bit of a byte of the sums says that the byte is not 0
      const uint32_t mm = (m[i] & 0x7F7F7F7Fu) + 0x7F7F7F7Fu, vv = ((v[i] & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | v[i];
      all &= mm & vv;
    }
    return __all_sync(0xffffffffu, VEC ? all == 0x80808080u : (all & 0x80u) != 0);
  }
  __device__ __forceinline__ uint32_t m_at(int i) const { return VEC ? (m[i / 4 % 2] >> (8 * (i % 4))) & 0xFFu : m[i % (VEC ? 2 : 8)]; }
  __device__ __forceinline__ uint32_t v_at(int i) const { return VEC ? (v[i / 4 % 2] >> (8 * (i % 4))) & 0xFFu : v[i % (VEC ? 2 : 8)]; }

  __device__ __forceinline__ void decode(float (&mf)[8], float (&vf)[8], uint32_t mb, uint32_t vb, bool no_zeros) const {
    if (no_zeros) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (VEC) {                       // the byte to bits 16 .. 23, four up, plus the base; the sign byte on top
          const uint32_t mag = __byte_perm(m[i / 4] & 0x7F7F7F7Fu, 0u, 0x4044 | (i % 4) << 8), sign = __byte_perm(m[i / 4], 0u, 0x0444 | (i % 4) << 12);
          mf[i] = __uint_as_float(((mag << 4) + mb) | (sign & 0x80000000u));
          vf[i] = __uint_as_float((__byte_perm(v[i / 4], 0u, 0x4044 | (i % 4) << 8) << 4) + vb);
        } else {
          mf[i] = __uint_as_float((((m[i] & 127u) << 20) + mb) | ((m[i] & 128u) << 24));
          vf[i] = __uint_as_float((v[i] << 20) + vb);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t c = m_at(i), mag = c & 127u, q = v_at(i);
        mf[i] = __uint_as_float((mag ? (mag << 20) + mb : 0u) | ((c & 128u) << 24));
        vf[i] = __uint_as_float(q ? (q << 20) + vb : 0u);
      }
    }
  }

  // `simple`: every value is finite and no v is 0, which allows the shorter forms of the same codes.
  __device__ __forceinline__ void encode(const float (&mf)[8], const float (&vf)[8], int mbase, int vbase, int64_t slot, uint32_t key, int lane, bool simple) {
    const uint32_t hash0 = slot_hash_start(slot);
    uint32_t cm[8], cv[8];
    if (simple) {
      const uint32_t mshift = (uint32_t)mbase << 20, vshift = ((uint32_t)vbase + 1u) << 20;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (the last step of mix32 leaves the upper half alone, so both halves come from the step before it)
        const uint32_t h = mix32_but_last((hash0 + (uint32_t)lane_element<VEC>(lane, i) * kSlotFactor) ^ key), upper = h >> 16;
        const uint32_t mbits = __float_as_uint(mf[i]) & 0x7FFFFFFFu;
        cm[i] = (uint32_t)__vimin_s32_relu((int)((((h ^ upper) & 0xFFFFu) << 4) + (mbits - mshift)) >> 20, 127);
        cv[i] = (uint32_t)__vimin_s32_relu((int)((upper << 4) + (__float_as_uint(vf[i]) - vshift)) >> 20, 254);     // one less
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t r = mix32((hash0 + (uint32_t)lane_element<VEC>(lane, i) * kSlotFactor) ^ key);
        cm[i] = (uint32_t)max(state_code(__float_as_uint(mf[i]) & 0x7FFFFFFFu, (r & 0xFFFFu) << 4, mbase, 127), 0);
        cv[i] = (uint32_t)max(state_code(__float_as_uint(vf[i]) & 0x7FFFFFFFu, (r >> 16) << 4, vbase, 255), vf[i] != 0.0f ? 1 : 0);
      }
    }
    if constexpr (VEC) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        auto four = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t pick) {      // one byte of each
          return __byte_perm(__byte_perm(a, b, pick), __byte_perm(c, d, pick), 0x5410);
        };
        const uint32_t mag = four(cm[4 * h], cm[4 * h + 1], cm[4 * h + 2], cm[4 * h + 3], 0x0040);
        const uint32_t sign = four(__float_as_uint(mf[4 * h]), __float_as_uint(mf[4 * h + 1]), __float_as_uint(mf[4 * h + 2]), __float_as_uint(mf[4 * h + 3]), 0x0073);
        m[h] = mag | (sign & (mag + 0x7F7F7F7Fu) & 0x80808080u);                             // no sign on a zero
        v[h] = four(cv[4 * h], cv[4 * h + 1], cv[4 * h + 2], cv[4 * h + 3], 0x0040) + (simple ? 0x01010101u : 0u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[i] = cm[i] | (cm[i] ? (__float_as_uint(mf[i]) >> 24) & 128u : 0u);
        v[i] = cv[i] + (simple ? 1u : 0u);
      }
    }
  }
};

template <int BITS, typename G, BlockMode MODE>
__device__ __forceinline__ void adam_block(const AdamStepArgs& a, const AdamChunk& ch, const G* grad, int first, int lane, int n) {
  constexpr bool VEC = MODE != kSingle;
  float p[8], m[8], v[8];
  G g[8];
  const int64_t slot = ch.slot + first;
  const int64_t block = slot / kAdamBlock;
  if constexpr (MODE == kShifted) {
    load8_shifted(p, (const float*)ch.p + first, lane);
    load8_shifted(g, grad + first, lane);
  } else {
    load8<VEC>(p, (const float*)ch.p + first, lane, n);
    load8<VEC>(g, grad + first, lane, n);
  }
  LaneCodes<VEC> codes;
  Pack<int16_t, 2> base;
  if constexpr (BITS == 32) {
    load8<VEC>(m, (const float*)a.exp_avg + slot, lane, kAdamBlock);
    load8<VEC>(v, (const float*)a.exp_avg_sq + slot, lane, kAdamBlock);
  } else {
    codes.load((const uint8_t*)a.exp_avg + slot, (const uint8_t*)a.exp_avg_sq + slot, lane);
    base = load_pack<int16_t, 2>(a.base + 2 * block);
  }
  const float inv_sqrt_bc2 = a.scalars->inv_sqrt_bc2;
  const Float2 grad_scale = pack2(a.scalars->grad_scale, a.scalars->grad_scale), clip = pack2(a.scalars->clip, a.scalars->clip);
  const Float2 b1 = pack2(a.beta1, a.beta1), c1 = pack2(a.one_minus_beta1, a.one_minus_beta1);
  const Float2 b2 = pack2(a.beta2, a.beta2), c2 = pack2(a.one_minus_beta2, a.one_minus_beta2);
  const float minus_step = -a.lr * a.scalars->inv_bc1;
  const float decay = 1.0f - a.lr * ch.weight_decay;
  bool simple = false;
  if constexpr (BITS == 8) {
    simple = codes.none_zero();
    codes.decode(m, v, (uint32_t)(int)base.e[0] << 20, (uint32_t)(int)base.e[1] << 20, simple);
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const Float2 gi = mul2(mul2(pack2(to_float(g[i]), to_float(g[i + 1])), grad_scale), clip);
    float kept[2], added[2];                   // (added one by one: a packed sum of packed products becomes a multiply-add)
    unpack2(mul2(b1, pack2(m[i], m[i + 1])), kept[0], kept[1]);
    unpack2(mul2(c1, gi), added[0], added[1]);
    m[i] = __fadd_rn(kept[0], added[0]);
    m[i + 1] = __fadd_rn(kept[1], added[1]);
    unpack2(mul2(b2, pack2(v[i], v[i + 1])), kept[0], kept[1]);
    unpack2(mul2(mul2(c2, gi), gi), added[0], added[1]);
    v[i] = __fadd_rn(kept[0], added[0]);
    v[i + 1] = __fadd_rn(kept[1], added[1]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = fmaf(p[i], decay, __fdividef(minus_step * m[i], fmaf(sqrt_fast(v[i]), inv_sqrt_bc2, a.eps)));
  }
  if constexpr (MODE == kShifted) store8_shifted(ch.p + first, p, lane);
  else store8<VEC>(ch.p + first, p, lane, n);
  if (ch.copy) {
    __nv_bfloat16 c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = from_float<__nv_bfloat16>(p[i]);
    __nv_bfloat16* copy = ch.copy + first;
    if (MODE == kShifted && ((uintptr_t)copy & 7) != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) copy[lane_element<true>(lane, i)] = c[i];
    } else {
      store8<VEC>(copy, c, lane, n);
    }
  }
  if constexpr (BITS == 32) {
    store8<VEC>((float*)a.exp_avg + slot, m, lane, kAdamBlock);
    store8<VEC>((float*)a.exp_avg_sq + slot, v, lane, kAdamBlock);
  } else {
    uint32_t mbits = 0, vbits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mbits = max(mbits, __float_as_uint(m[i]) & 0x7FFFFFFFu);
      vbits = max(vbits, __float_as_uint(v[i]));
    }
    mbits = __reduce_max_sync(0xffffffffu, mbits);
    vbits = __reduce_max_sync(0xffffffffu, vbits);
    if (max(mbits, vbits) >= 0x7F800000u) {          // something is not finite: the largest of the others
      simple = false;
      mbits = vbits = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mbits = max(mbits, finite_bits(__float_as_uint(m[i]) & 0x7FFFFFFFu));
        vbits = max(vbits, finite_bits(__float_as_uint(v[i]) & 0x7FFFFFFFu));
      }
      mbits = __reduce_max_sync(0xffffffffu, mbits);
      vbits = __reduce_max_sync(0xffffffffu, vbits);
    }
    // (v was not 0 and beta2 leaves it so: a quarter of the smallest value of the grid is still a float32)
    simple = simple && a.beta2 >= 0.25f;
    base.e[0] = (int16_t)window_base(mbits, 127u);
    base.e[1] = (int16_t)window_base(vbits, 255u);
    codes.encode(m, v, base.e[0], base.e[1], slot, a.scalars->key, lane, simple);
    codes.store((uint8_t*)a.exp_avg + slot, (uint8_t*)a.exp_avg_sq + slot, lane);
    if (lane == 0) store_pack<int16_t, 2>(a.base + 2 * block, base);
  }
}

// Chunks go from the last to the first: what the norm kernel read last is still in L2.
template <int BITS, typename G>
__global__ void __launch_bounds__(kAdamThreads, 4) adam_step_kernel(AdamStepArgs a) {
  const AdamChunk ch = a.chunks[gridDim.x - 1 - blockIdx.x];
  const int lane = threadIdx.x & 31, first = (threadIdx.x >> 5) * kAdamBlock;
  const int left = ch.count - first;
  const G* grad = a.flat ? static_cast<const G*>(a.flat) + ch.offset : static_cast<const G*>(ch.grad);
  const bool aligned = ((uintptr_t)ch.p & 15) == 0 && ((uintptr_t)ch.copy & 7) == 0 && ((uintptr_t)grad & (sizeof(G) < 4 ? 7 : 15)) == 0;
  const bool full = left >= kAdamBlock;
  const bool inside = full && !(first == 0 && ch.starts) && left - kAdamBlock + ch.behind >= 3;
  pdl_wait();
  if (left <= 0 || a.scalars->skip) return;
  if (aligned && full) adam_block<BITS, G, kAligned>(a, ch, grad, first, lane, kAdamBlock);
  else if (inside) adam_block<BITS, G, kShifted>(a, ch, grad, first, lane, kAdamBlock);
  else adam_block<BITS, G, kSingle>(a, ch, grad, first, lane, full ? kAdamBlock : left);
}

// What the 8-bit state stands for, as bfloat16: blocks x 256.  A value of the grid has zeros in the low 20 of its float32's
// bits, so the upper 16 are its bfloat16: (code + base) << 4, two to a word.  16 codes a thread.
__device__ __forceinline__ uint32_t two_moments(uint32_t c, uint32_t base2, uint32_t mask) {      // codes in bytes 0 and 2
  const uint32_t mag = c & mask;
  const uint32_t nonzero = ((mag + 0x00FF00FFu) >> 8) & 0x00010001u;
  return (((mag + base2) << 4) & (nonzero * 0xFFFFu)) | ((c & ~mask & 0x00800080u) << 8);
}
__device__ __forceinline__ uint4 eight_moments(uint32_t lo, uint32_t hi, uint32_t base2, uint32_t mask) {
  return make_uint4(two_moments(__byte_perm(lo, 0u, 0x4140), base2, mask), two_moments(__byte_perm(lo, 0u, 0x4342), base2, mask),
                    two_moments(__byte_perm(hi, 0u, 0x4140), base2, mask), two_moments(__byte_perm(hi, 0u, 0x4342), base2, mask));
}
__global__ void __launch_bounds__(256) adam_moments_kernel(const uint4* __restrict__ m, const uint4* __restrict__ v, const uint32_t* __restrict__ base,
                                                           int64_t n_words, uint4* __restrict__ m_out, uint4* __restrict__ v_out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_words) return;
  const uint4 mc = m[i], vc = v[i];
  const uint32_t b = base[i / (kAdamBlock / 16)];
  const uint32_t mb = __byte_perm(b, 0u, 0x1010), vb = __byte_perm(b, 0u, 0x3232);
  m_out[2 * i] = eight_moments(mc.x, mc.y, mb, 0x007F007Fu);
  m_out[2 * i + 1] = eight_moments(mc.z, mc.w, mb, 0x007F007Fu);
  v_out[2 * i] = eight_moments(vc.x, vc.y, vb, 0x00FF00FFu);
  v_out[2 * i + 1] = eight_moments(vc.z, vc.w, vb, 0x00FF00FFu);
}

// ---- host ------------------------------------------------------------------------------------------------------------

// A copy to the device that has arrived when the call returns, whichever stream the next step goes to: from pageable memory
// cudaMemcpy alone may return when the bytes are staged, and streams made without blocking are not ordered behind it.
static int adam_upload(void* to, const void* from, size_t bytes) {
  if (bytes) SOLON_CUDA_TRY(cudaMemcpy(to, from, bytes, cudaMemcpyHostToDevice));
  SOLON_CUDA_TRY(cudaDeviceSynchronize());
  return SOLON_OK;
}

static int adam_upload_scalars(solon_adamw* o, int64_t step) {
  AdamScalars s = {};
  s.b1t = pow(o->beta1, (double)step);
  s.b2t = pow(o->beta2, (double)step);
  s.applied = step;
  return adam_upload(o->d_scalars, &s, sizeof(s));
}

static void adam_free(solon_adamw* o) {
  cudaFree(o->d_chunks);
  cudaFree(o->d_scalars);
  cudaFree(o->d_partials);
  (void)cudaGetLastError();
}

template <typename T>
static int adam_alloc(T** ptr, size_t count) {
  cudaError_t err = cudaMalloc((void**)ptr, (count ? count : 1) * sizeof(T));
  if (err == cudaSuccess) return SOLON_OK;
  (void)cudaGetLastError();
  *ptr = nullptr;
  return err == cudaErrorMemoryAllocation ? SOLON_ERR_NOMEM : SOLON_ERR_CUDA;
}

static int64_t adam_blocks(int64_t numel) { return (numel + kAdamBlock - 1) / kAdamBlock; }

static int adam_upload_chunks(solon_adamw* o) {
  return adam_upload(o->d_chunks, o->chunks.data(), o->chunks.size() * sizeof(AdamChunk));
}

static int adam_create(solon_adamw* o, const int64_t* numel, float* const* params, void* const* copies, const float* weight_decay) {
  o->numel.assign(numel, numel + o->n_tensors);
  for (int i = 0; i < o->n_tensors; ++i) {
    for (int64_t first = 0; first < numel[i]; first += kAdamChunk) {
      AdamChunk c = {};
      c.p = params[i] + first;
      c.copy = copies && copies[i] ? static_cast<__nv_bfloat16*>(copies[i]) + first : nullptr;
      c.offset = o->total + first;
      c.slot = o->n_blocks * kAdamBlock + first;
      c.count = (int)(numel[i] - first < kAdamChunk ? numel[i] - first : kAdamChunk);
      c.weight_decay = weight_decay ? weight_decay[i] : 0.0f;
      c.starts = first == 0;
      const int64_t behind = numel[i] - first - c.count;
      c.behind = (int)(behind < 3 ? behind : 3);
      o->chunks.push_back(c);
    }
    o->total += numel[i];
    o->n_blocks += adam_blocks(numel[i]);
  }
  o->n_chunks = (int64_t)o->chunks.size();      // (at most one a block: below 2^31)
  o->norm_grid = o->num_sms * 4;
  if (o->norm_grid > o->n_chunks) o->norm_grid = o->n_chunks ? (int)o->n_chunks : 1;
  int rc;
  if ((rc = adam_alloc(&o->d_chunks, o->chunks.size()))) return rc;
  if ((rc = adam_alloc(&o->d_scalars, 1))) return rc;
  if ((rc = adam_alloc(&o->d_partials, (size_t)o->norm_grid))) return rc;
  if ((rc = adam_upload_chunks(o))) return rc;
  return adam_upload_scalars(o, 0);
}

template <typename G>
static int adam_norm(solon_adamw* o, const void* flat, cudaStream_t stream) {
  const dim3 grid((unsigned)o->norm_grid), block(kAdamThreads);
  if (flat) return launch_dependent(adam_norm_flat_kernel<G>, grid, block, 0, stream, static_cast<const G*>(flat), o->total, o->d_partials);
  return launch_dependent(adam_norm_bound_kernel<G>, grid, block, 0, stream, (const AdamChunk*)o->d_chunks, o->n_chunks, o->d_partials);
}

template <typename G>
static int adam_update(solon_adamw* o, const AdamStepArgs& a, cudaStream_t stream) {
  const dim3 grid((unsigned)o->n_chunks), block(kAdamThreads);
  if (o->bits == 32) return launch_dependent(adam_step_kernel<32, G>, grid, block, 0, stream, a);
  return launch_dependent(adam_step_kernel<8, G>, grid, block, 0, stream, a);
}

}  // namespace solon

using namespace solon;

extern "C" {

int64_t solon_adamw_state_blocks(int n_tensors, const int64_t* numel) {
  if (n_tensors < 1 || !numel) return SOLON_ERR_INVALID_ARG;
  int64_t blocks = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (numel[i] < 0 || numel[i] > SOLON_ADAMW_MAX_NUMEL) return SOLON_ERR_INVALID_ARG;
    blocks += adam_blocks(numel[i]);
    if (blocks > SOLON_ADAMW_MAX_NUMEL / kAdamBlock) return SOLON_ERR_INVALID_ARG;
  }
  return blocks;
}

int solon_adamw_create(int n_tensors, const int64_t* numel, float* const* params, void* const* copies, const float* weight_decay, int state_bits,
                       void* exp_avg, void* exp_avg_sq, int16_t* base, double beta1, double beta2, double eps, uint64_t seed, solon_adamw** out) {
  if (!out) return SOLON_ERR_INVALID_ARG;
  *out = nullptr;
  if (!params || !exp_avg || !exp_avg_sq || (state_bits != 32 && state_bits != 8) || (state_bits == 8 && !base)) return SOLON_ERR_INVALID_ARG;
  if (solon_adamw_state_blocks(n_tensors, numel) < 0) return SOLON_ERR_INVALID_ARG;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps > 0.0f && eps < INFINITY)) return SOLON_ERR_INVALID_ARG;
  if (((uintptr_t)exp_avg | (uintptr_t)exp_avg_sq) & 15 || ((uintptr_t)base & 3)) return SOLON_ERR_INVALID_ARG;
  for (int i = 0; i < n_tensors; ++i) {
    if (numel[i] > 0 && (!params[i] || ((uintptr_t)params[i] & 3))) return SOLON_ERR_INVALID_ARG;
    if (copies && copies[i] && ((uintptr_t)copies[i] & 1)) return SOLON_ERR_INVALID_ARG;
    if (weight_decay && !(weight_decay[i] >= 0.0f && weight_decay[i] < INFINITY)) return SOLON_ERR_INVALID_ARG;
  }
  int device = 0, sms = 0;
  SOLON_CUDA_TRY(cudaGetDevice(&device));
  SOLON_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  solon_adamw* o = new (std::nothrow) solon_adamw();
  if (!o) return SOLON_ERR_NOMEM;
  o->n_tensors = n_tensors;
  o->bits = state_bits;
  o->device = device;
  o->num_sms = sms;
  o->beta1 = beta1;
  o->beta2 = beta2;
  o->eps = eps;
  o->seed = seed;
  o->exp_avg = exp_avg;
  o->exp_avg_sq = exp_avg_sq;
  o->base = base;
  int rc;
  try {
    rc = adam_create(o, numel, params, copies, weight_decay);
  } catch (...) {
    rc = SOLON_ERR_NOMEM;
  }
  if (rc) {
    adam_free(o);
    delete o;
    return rc;
  }
  *out = o;
  return SOLON_OK;
}

int solon_adamw_destroy(solon_adamw* opt) {
  if (!opt) return SOLON_ERR_INVALID_ARG;
  adam_free(opt);      // cudaFree waits for work in flight
  delete opt;
  return SOLON_OK;
}

int solon_adamw_bind_grads(solon_adamw* opt, const void* const* grads, int grad_dtype) {
  if (!opt || !grads || (grad_dtype != SOLON_F32 && grad_dtype != SOLON_F64 && grad_dtype != SOLON_BF16)) return SOLON_ERR_INVALID_ARG;
  const uintptr_t size = grad_dtype == SOLON_F64 ? 8 : grad_dtype == SOLON_F32 ? 4 : 2;
  for (int i = 0; i < opt->n_tensors; ++i)
    if (opt->numel[(size_t)i] > 0 && (!grads[i] || ((uintptr_t)grads[i] & (size - 1)))) return SOLON_ERR_INVALID_ARG;
  SOLON_CUDA_TRY(cudaDeviceSynchronize());     // steps in flight read the table
  opt->grads_bound = 0;                        // until the new ones have arrived: a copy that fails may leave some of each
  size_t chunk = 0;
  for (int i = 0; i < opt->n_tensors; ++i)
    for (int64_t first = 0; first < opt->numel[(size_t)i]; first += kAdamChunk) opt->chunks[chunk++].grad = static_cast<const char*>(grads[i]) + first * (int64_t)size;
  int rc;
  if ((rc = adam_upload_chunks(opt))) return rc;
  opt->grads_bound = 1;
  opt->grad_dtype = grad_dtype;
  return SOLON_OK;
}

int solon_adamw_set_step(solon_adamw* opt, int64_t step) {
  if (!opt || step < 0) return SOLON_ERR_INVALID_ARG;
  SOLON_CUDA_TRY(cudaDeviceSynchronize());
  return adam_upload_scalars(opt, step);
}

int solon_adamw_get_steps(solon_adamw* opt, int64_t* applied, int64_t* skipped) {
  if (!opt || !applied || !skipped) return SOLON_ERR_INVALID_ARG;
  AdamScalars s;
  SOLON_CUDA_TRY(cudaDeviceSynchronize());
  SOLON_CUDA_TRY(cudaMemcpy(&s, opt->d_scalars, sizeof(s), cudaMemcpyDeviceToHost));
  *applied = s.applied;
  *skipped = s.skipped;
  return SOLON_OK;
}

int solon_adamw_step(solon_adamw* opt, const void* grad, int grad_dtype, double grad_scale, double lr, double max_norm, float* grad_norm,
                     const solon_plan* guard, void* cuda_stream) {
  if (!opt) return SOLON_ERR_INVALID_ARG;
  if (!grad) {
    if (!opt->grads_bound) return SOLON_ERR_INVALID_ARG;
    grad_dtype = opt->grad_dtype;
  }
  if (grad_dtype != SOLON_F32 && grad_dtype != SOLON_F64 && grad_dtype != SOLON_BF16) return SOLON_ERR_INVALID_ARG;
  const uintptr_t size = grad_dtype == SOLON_F64 ? 8 : grad_dtype == SOLON_F32 ? 4 : 2;
  if ((uintptr_t)grad & (size - 1) || ((uintptr_t)grad_norm & 3)) return SOLON_ERR_INVALID_ARG;
  if (!(fabs(grad_scale) < INFINITY) || !(lr >= 0.0 && lr < INFINITY) || !(max_norm >= 0.0 && max_norm < INFINITY)) return SOLON_ERR_INVALID_ARG;
  if (grad_norm && max_norm == 0.0) return SOLON_ERR_INVALID_ARG;
  if (guard && guard->device != opt->device) return SOLON_ERR_INVALID_ARG;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  int rc;
  AdamControlArgs c = {};
  c.s = opt->d_scalars;
  c.partials = opt->d_partials;
  c.n_partials = max_norm > 0.0 ? opt->norm_grid : 0;
  c.norm_out = grad_norm;
  c.grad_scale = grad_scale;
  c.max_norm = max_norm;
  c.beta1 = opt->beta1;
  c.beta2 = opt->beta2;
  c.quotient_scale = opt->eps > 0x1p100 ? 0x1p-28 : opt->eps < 0x1p-100 ? 0x1p28 : 1.0;      // eps: 2^-149 .. 2^128 to 2^-121 .. 2^100
  c.seed = opt->seed;
  if (guard) {
    c.guard_status = guard->d_status;
    c.guard_t = guard->d_t_acc;
    c.guard_groups = guard->q;
  }
  if (max_norm > 0.0) {
    rc = grad_dtype == SOLON_F32 ? adam_norm<float>(opt, grad, stream) : grad_dtype == SOLON_F64 ? adam_norm<double>(opt, grad, stream)
                                                                                                  : adam_norm<__nv_bfloat16>(opt, grad, stream);
    if (rc) return rc;
  }
  if ((rc = launch_dependent(adam_control_kernel, dim3(1), dim3(256), 0, stream, c))) return rc;
  if (opt->n_chunks == 0) return SOLON_OK;
  AdamStepArgs a = {};
  a.chunks = opt->d_chunks;
  a.flat = grad;
  a.exp_avg = opt->exp_avg;
  a.exp_avg_sq = opt->exp_avg_sq;
  a.base = opt->base;
  a.scalars = opt->d_scalars;
  a.beta1 = (float)opt->beta1;
  a.one_minus_beta1 = (float)(1.0 - opt->beta1);
  a.beta2 = (float)opt->beta2;
  a.one_minus_beta2 = (float)(1.0 - opt->beta2);
  a.eps = (float)(opt->eps * c.quotient_scale);
  a.lr = (float)lr;
  return grad_dtype == SOLON_F32 ? adam_update<float>(opt, a, stream) : grad_dtype == SOLON_F64 ? adam_update<double>(opt, a, stream)
                                                                                                 : adam_update<__nv_bfloat16>(opt, a, stream);
}

int solon_adamw_moments(solon_adamw* opt, void* exp_avg_out, void* exp_avg_sq_out, void* cuda_stream) {
  if (!opt || opt->bits != 8 || !exp_avg_out || !exp_avg_sq_out) return SOLON_ERR_INVALID_ARG;
  if (((uintptr_t)exp_avg_out | (uintptr_t)exp_avg_sq_out) & 15) return SOLON_ERR_INVALID_ARG;
  const int64_t words = opt->n_blocks * (kAdamBlock / 16);
  if (words == 0) return SOLON_OK;
  adam_moments_kernel<<<(unsigned)((words + 255) / 256), 256, 0, (cudaStream_t)cuda_stream>>>(
      (const uint4*)opt->exp_avg, (const uint4*)opt->exp_avg_sq, (const uint32_t*)opt->base, words, (uint4*)exp_avg_out, (uint4*)exp_avg_sq_out);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

}  // extern "C"
