// Layer norm over the rows of a matrix, forward and backward, with the gradients of weight and bias summed per partition
// straight into the rows of the partition-gradient matrix that solon_encode reads.
//     mu = mean x, rstd = (mean (x - mu)^2 + eps)^(-1/2), xh = (x - mu) rstd, y = w xh + b
//     a = w dy,   dx = rstd (a - mean a - xh mean(a xh)),   dw_k = sum dy xh,   db_k = sum dy   (rows of partition k)
// The variance is summed over the differences from the mean (a second sweep over values that sit in registers), not as a
// difference of two sums; statistics and sums are float32.
//
// Bound by memory: 2 (forward) and 3 (backward) accesses of the matrix against about 8 and 14 flops an element.  Measured, call
// after call on the same tensors, and with cold caches: forward 16384 x 4096 bfloat16 48 to 51 us (5.3 to 5.6 TB/s), 52 cold, 8192 x
// 8192 float32 83 (6.4 TB/s), 87 cold; backward 15 x 2048 rows of 2048 bfloat16 67 us (5.6 TB/s), 73 cold, 3.5 of them for the
// partial sums, 8192 x 8192 float32 135 (6.0 TB/s), 132 cold.  What keeps it from the copy rate is 16 warps
// an SM (the registers of a column's parameters and sums), each with a barrier or two a row.
//
// Layout: a row belongs to a team of TPR threads that hold 16 or 32 elements each (fewer in short rows), so that a team's
// reductions cost little beside the work on the elements.  Teams of one warp meet in shuffles only, larger ones
// also in shared memory.  CTAs stay for many rows; every thread copies its own words of the next rows into shared memory
// ahead of time (cp.async: it waits for its own copies only, no barrier), which keeps enough bytes on the way without registers
// for them.  The weight's gradient is summed in registers over all rows of a CTA; only one partial sum per CTA and column
// leaves it, added up per partition by a second kernel in a fixed order.
#include <math.h>

#include <type_traits>

#include "elements.cuh"
#include "solon_internal.h"
#include "token_args.h"

namespace solon {

constexpr int kLnThreads = 256;                // threads of a CTA, or one team if that is larger
constexpr int kLnMaxCols = 16384;              // 1024 threads of 16 float32; wider rows take the streaming kernels

// Rows on the way per team beside the one that is worked on: four, or what 96 KB (of a CTA of which two share an SM) or 192 KB
// of shared memory hold.
constexpr int ln_stages_for(int threads, int row_bytes_per_thread) {
  const int fit = (threads <= kLnThreads ? 98304 : 196608) / (threads * row_bytes_per_thread);
  return fit < 1 ? 1 : fit < 4 ? fit : 4;
}
template <typename T, int TPR, int ELEMS, int ROWS>
constexpr int ln_stages = ln_stages_for(TPR < kLnThreads ? kLnThreads : TPR, ROWS * ELEMS * (int)sizeof(T));
template <int TPR>
__device__ __forceinline__ void team_barrier(int team = 0) {
  if constexpr (TPR == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(TPR) : "memory");
}
// Sum over the team, the result in every thread.  Teams of several warps alternate between two slots, so one barrier a
// sum is enough: a slot is written again only after everybody has passed the barrier of the sum in between.  (The slots are read
// in packs of 16 bytes, which their type is aligned for.)
template <int N>
struct alignas(16) SumSlots {
  float v[2 * 32 * N];
};
template <int TPR, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], SumSlots<N>& slots, int& turn, int team) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], off);
  if constexpr (TPR > 32) {
    constexpr int kWarps = TPR / 32;
    const int warp = (threadIdx.x & (TPR - 1)) >> 5;
    float* s = slots.v + (turn * (blockDim.x >> 5) + team * kWarps) * N;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) s[k * kWarps + warp] = v[k];
    }
    team_barrier<TPR>(team);
    if constexpr (kWarps == 32) {              // a lane a warp's sum: 32 warps that each read 32 sums would queue for shared memory
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = s[k * kWarps + (threadIdx.x & 31)];
#pragma unroll
      for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], off);
      return;
    }
    constexpr int kRead = kWarps < 4 ? kWarps : 4;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; w += kRead) {
        const Pack<float, kRead> q = load_pack<float, kRead>(s + k * kWarps + w);
#pragma unroll
        for (int j = 0; j < kRead; ++j) sum += q.e[j];
      }
      v[k] = sum;
    }
  }
}

__device__ __forceinline__ float param_at(const void* p, int is_f32, int dtype, int64_t c) {
  if (is_f32) return static_cast<const float*>(p)[c];
  if (dtype == SOLON_BF16) return to_float(static_cast<const __nv_bfloat16*>(p)[c]);
  return to_float(static_cast<const __half*>(p)[c]);
}

struct LnForwardArgs {
  const void* x;
  const void* weight;
  const void* bias;
  void* y;
  float* mean;
  float* rstd;
  int64_t rows, cols, x_pitch, y_pitch;
  float eps;
  int param_f32, dtype;
};

// How a thread sees a row: ELEMS elements in groups of VEC neighbours - 16-byte words, or, where rows are not made of 16-byte
// words at 16-byte boundaries, pairs or single elements.  Single elements are loaded straight into registers: no asynchronous copy
// moves two bytes, and with four a copy per element costs more than it hides (backward 15 x 1000 x 2001 float32 78 us straight, 98
// copied).  Pairs gain by the ring (30000 x 2002 bfloat16 70 -> 54 us, backward 45 x 700 x 1002 63 -> 54).  Two elements share an
// instruction.
template <typename T, int VEC, int TPR, int ELEMS>
struct LnRow {
  static constexpr int kGroups = ELEMS / VEC;
  static constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
  static constexpr int kTeam = TPR, kTeams = kBlock / TPR;
  static constexpr bool kRing = VEC > 1;
  using Group = Pack<T, VEC>;
  static constexpr int kStageGroups = kGroups * kBlock;      // of a stage: one row of every team
  // Elements can be gone through in steps of a few, and those left out in which a warp has no column of the row.  What that
  // saves, and the order of loads and sums that comes with it, pays where the functions below say so.
  static constexpr int kStep = VEC > 4 ? VEC : ELEMS < 4 ? ELEMS : 4, kSteps = ELEMS / kStep, kStepGroups = kStep / VEC;

  static __device__ __forceinline__ int column(int group, int tid) { return (group * TPR + tid) * VEC; }
  static __device__ __forceinline__ int steps(int cols, int tid) {
    int n = 1;
#pragma unroll
    for (int s = 1; s < kSteps; ++s) n += column(s * kStepGroups, tid & ~31) < cols;
    return n;
  }

  // the copies of a row's groups into a stage of the ring (groups x threads)
  static __device__ __forceinline__ void issue(Group* stage, const T* row, int cols, int tid, int steps) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      if (i >= kStepGroups && i / kStepGroups >= steps) break;
      const int c = column(i, tid);
      copy_async<(int)sizeof(Group)>(stage + i * kBlock + threadIdx.x, c < cols ? row + c : row, c < cols);
    }
  }
  static __device__ __forceinline__ void take(Float2 (&v)[ELEMS / 2], const Group* stage, const T* row, int cols, int tid, int steps) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (s > 0 && s >= steps) break;
      if constexpr (VEC * sizeof(T) == 16) {
#pragma unroll
        for (int i = s * kStepGroups; i < (s + 1) * kStepGroups; ++i) {
          float part[VEC];
          Word16<T>::unpack(reinterpret_cast<const uint4&>(stage[i * kBlock + threadIdx.x]), part);
#pragma unroll
          for (int k = 0; k < VEC; k += 2) v[(i * VEC + k) / 2] = pack2(part[k], part[k + 1]);
        }
      } else {
        Group part[kStepGroups];
#pragma unroll
        for (int i = 0; i < kStepGroups; ++i) {
          const int group = s * kStepGroups + i;
          if constexpr (kRing) part[i] = stage[group * kBlock + threadIdx.x];
          else part[i].e[0] = column(group, tid) < cols ? row[column(group, tid)] : from_float<T>(0.0f);
        }
#pragma unroll
        for (int i = 0; i < kStep; i += 2) v[(s * kStep + i) / 2] = pack2(to_float(part[i / VEC].e[i % VEC]), to_float(part[(i + 1) / VEC].e[(i + 1) % VEC]));
      }
    }
  }
  static __device__ __forceinline__ void store(T* row, const Float2 (&v)[ELEMS / 2], int cols, int tid) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int c = column(i, tid);
      if constexpr (VEC * sizeof(T) == 16) {
        float part[VEC];
#pragma unroll
        for (int k = 0; k < VEC; k += 2) unpack2(v[(i * VEC + k) / 2], part[k], part[k + 1]);
        if (c < cols) *reinterpret_cast<uint4*>(row + c) = Word16<T>::pack(part);
      } else {
        float part[2];
        unpack2(v[i * VEC / 2], part[0], part[1]);
        Group p;
#pragma unroll
        for (int k = 0; k < VEC; ++k) p.e[k] = from_float<T>(part[(i * VEC + k) % 2]);
        if (c < cols) store_pack<T, VEC>(row + c, p);
      }
    }
  }
  // weight or bias of the thread's columns (once per CTA)
  static __device__ __forceinline__ void params(Float2 (&w)[ELEMS / 2], const void* p, int is_f32, int dtype, float absent, int cols, int tid) {
    float e[ELEMS];
    if constexpr (VEC >= 4) {
      if (p && is_f32 && ((uintptr_t)p & 15) == 0) {
#pragma unroll
        for (int i = 0; i < ELEMS; i += 4) {
          const int c = column(i / VEC, tid) + i % VEC;
          const float4 v = c < cols ? *reinterpret_cast<const float4*>(static_cast<const float*>(p) + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          w[i / 2] = pack2(v.x, v.y);
          w[i / 2 + 1] = pack2(v.z, v.w);
        }
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < ELEMS; ++i) {
      const int c = column(i / VEC, tid) + i % VEC;
      e[i] = c < cols ? (p ? param_at(p, is_f32, dtype, c) : absent) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < ELEMS; i += 2) w[i / 2] = pack2(e[i], e[i + 1]);
  }
};

__device__ __forceinline__ Float2 both(float x) { return pack2(x, x); }
__device__ __forceinline__ float sum_of(Float2 x) {
  float a, b;
  unpack2(x, a, b);
  return a + b;
}

// Which steps without columns are left out - of the copies, of the loads, of the work.  Measured with and without, us, caches
// cold.  Forward: words of float32 8192 x 8192 88, 97 (of two-byte elements the same, or 55, 53 with 4000 x 16384); single float32
// elements 4000 x 15001 130, 155.  Backward: teams up to 128 15 x 2048 x 2048 bfloat16 73, 78; of 256, the work alone, 16384 x 2560
// 68, 70; of 512, loads and work, 8192 x 5120 bfloat16 70, 74, but 8192 x 8192 85, 82, float32 131, 136; single float32 elements
// 30000 x 2001 134, 145 (two-byte ones 270, 109: their loads then wait for one another).
struct LnSkip {
  bool copies, loads, work;
};
template <typename T, int VEC>
constexpr LnSkip ln_forward_skip = {VEC == 4 && sizeof(T) == 4, VEC == 1 && sizeof(T) == 4, VEC != 2 && sizeof(T) == 4};
template <typename T, int VEC, int TPR>
constexpr LnSkip ln_backward_skip = VEC == 1   ? LnSkip{false, sizeof(T) == 4, sizeof(T) == 4}
                                    : VEC == 2 ? LnSkip{false, false, false}
                                               : LnSkip{TPR <= 128, TPR > 256, true};

// CTAs of the forward pass on an SM: with single elements a third one pays (30000 x 2001 bfloat16 81 -> 71 us, float32 98 -> 91).
template <int VEC, int TPR, int ELEMS>
constexpr int ln_forward_ctas = TPR >= 512 ? 1 : VEC > 1 || ELEMS > 16 ? 2 : 3;

template <typename T, int VEC, int TPR, int ELEMS>
__global__ void __launch_bounds__(TPR < kLnThreads ? kLnThreads : TPR, ln_forward_ctas<VEC, TPR, ELEMS>) ln_forward_kernel(LnForwardArgs a) {
  using Row = LnRow<T, VEC, TPR, ELEMS>;
  constexpr int kStages = ln_stages<T, TPR, ELEMS, 1>;
  extern __shared__ __align__(16) uint4 ring_memory[];
  typename Row::Group* ring = reinterpret_cast<typename Row::Group*>(ring_memory);      // stages x groups x threads
  __shared__ SumSlots<1> slots;
  const int tid = threadIdx.x & (TPR - 1), team = threadIdx.x / TPR, cols = (int)a.cols;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  constexpr LnSkip kSkip = ln_forward_skip<T, VEC>;
  const int with_columns = Row::steps(cols, tid);
  const int copy_steps = kSkip.copies ? with_columns : Row::kSteps, load_steps = kSkip.loads ? with_columns : Row::kSteps;
  const int steps = kSkip.work ? with_columns : Row::kSteps;
  const float inv_n = 1.0f / (float)cols;
  const int64_t stride = (int64_t)gridDim.x * Row::kTeams;
  int64_t row = (int64_t)blockIdx.x * Row::kTeams + team;
  if constexpr (Row::kRing) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) {
      if (row + s * stride < a.rows) Row::issue(ring + s * Row::kStageGroups, x + (row + s * stride) * a.x_pitch, cols, tid, copy_steps);
      copies_commit();
    }
  }
  Float2 w[ELEMS / 2], b[ELEMS / 2];
  Row::params(w, a.weight, a.param_f32, a.dtype, 1.0f, cols, tid);
  Row::params(b, a.bias, a.param_f32, a.dtype, 0.0f, cols, tid);
  int turn = 0, stage = 0;
  for (; row < a.rows; row += stride) {
    Float2 v[ELEMS / 2];
    typename Row::Group* words = ring + stage * Row::kStageGroups;
    if constexpr (Row::kRing) copies_wait<kStages - 1>();
    Row::take(v, words, x + row * a.x_pitch, cols, tid, load_steps);
    if constexpr (Row::kRing) {
      const int64_t ahead = row + kStages * stride;       // into the words just read
      if (ahead < a.rows) Row::issue(words, x + ahead * a.x_pitch, cols, tid, copy_steps);
      copies_commit();
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    Float2 acc = both(0.0f);
#pragma unroll
    for (int s = 0; s < Row::kSteps; ++s) {
      if (s > 0 && s >= steps) break;
#pragma unroll
      for (int i = s * Row::kStep / 2; i < (s + 1) * Row::kStep / 2; ++i) acc = add2(acc, v[i]);
    }
    float sum[1] = {sum_of(acc)};
    team_sum<TPR>(sum, slots, turn, team);
    const float mean = sum[0] * inv_n;
    const Float2 minus_mean = both(-mean);
    acc = both(0.0f);
#pragma unroll
    for (int s = 0; s < Row::kSteps; ++s) {
      if (s > 0 && s >= steps) break;
#pragma unroll
      for (int i = s * Row::kStep / 2; i < (s + 1) * Row::kStep / 2; ++i) {
        v[i] = add2(v[i], minus_mean);
        if constexpr (VEC > 1) {                            // a group lies inside the row or outside
          if (Row::column(2 * i / VEC, tid) < cols) acc = fma2(v[i], v[i], acc);
        } else {
          float e0, e1;
          unpack2(v[i], e0, e1);
          e0 = Row::column(2 * i, tid) < cols ? e0 : 0.0f;
          e1 = Row::column(2 * i + 1, tid) < cols ? e1 : 0.0f;
          const Float2 e = pack2(e0, e1);
          acc = fma2(e, e, acc);
        }
      }
    }
    float sq[1] = {sum_of(acc)};
    team_sum<TPR>(sq, slots, turn, team);
    const float rstd = rsqrtf(sq[0] * inv_n + a.eps);
    const Float2 scale = both(rstd);
#pragma unroll
    for (int s = 0; s < Row::kSteps; ++s) {
      if (s > 0 && s >= steps) break;
#pragma unroll
      for (int i = s * Row::kStep / 2; i < (s + 1) * Row::kStep / 2; ++i) v[i] = fma2(mul2(v[i], scale), w[i], b[i]);
    }
    Row::store(y + row * a.y_pitch, v, cols, tid);
    if (tid == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

struct LnBackwardArgs {
  const void* dy;
  const void* x;
  const void* weight;
  const float* mean;
  const float* rstd;
  void* dx;                    // nullptr: not wanted
  void* dweight;               // partitions rows of grad_pitch elements (nullptr: not wanted)
  void* dbias;
  float* partials;             // partitions x splits x 2 x cols (splits > 1)
  int64_t rows_per_part, cols, dy_pitch, x_pitch, dx_pitch, grad_pitch;
  int splits, param_f32, dtype, grad_f64;
};

__device__ __forceinline__ void store_grad(void* p, int f64, int64_t i, float v) {
  if (f64) static_cast<double*>(p)[i] = (double)v;
  else static_cast<float*>(p)[i] = v;
}

// A team's sums for weight and bias: the partition's gradient, or a partial sum where several CTAs share the partition.  `line`:
// shared memory for a float of each of the team's columns.
template <typename Row, int VEC, int ELEMS>
__device__ __forceinline__ void put_param_sums(const LnBackwardArgs& a, const float (&sums)[2][ELEMS], float* line, int part, int split, int tid) {
  const int cols = (int)a.cols;
  if (a.splits > 1) {
    constexpr int kStore = VEC < 4 ? VEC : 4;  // a row of groups of VEC elements is a row of groups of kStore
    float* out = a.partials + ((int64_t)part * a.splits + split) * 2 * a.cols;
#pragma unroll
    for (int i = 0; i < ELEMS; i += kStore) {
      const int c = Row::column(i / VEC, tid) + i % VEC;
      if (c >= cols) continue;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        float* to = out + which * cols + c;
        const float* v = &sums[which][i];
        if constexpr (kStore == 4) *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
        else if constexpr (kStore == 2) *reinterpret_cast<float2*>(to) = make_float2(v[0], v[1]);
        else *to = *v;
      }
    }
    return;
  }
  if constexpr (VEC >= 4) {                    // by way of shared memory, so that neighbouring threads store neighbouring elements
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      void* dst = which ? a.dbias : a.dweight;
      if (!dst) continue;
      team_barrier<Row::kTeam>();              // (only the first team is here)
#pragma unroll
      for (int i = 0; i < ELEMS; i += 4) {
        const float* v = &sums[which][i];
        *reinterpret_cast<float4*>(line + Row::column(i / VEC, tid) + i % VEC) = make_float4(v[0], v[1], v[2], v[3]);
      }
      team_barrier<Row::kTeam>();
      for (int c = tid; c < cols; c += Row::kTeam) store_grad(dst, a.grad_f64, part * a.grad_pitch + c, line[c]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < ELEMS; ++i) {
      const int c = Row::column(i / VEC, tid) + i % VEC;
      if (c >= cols) continue;
      if (a.dweight) store_grad(a.dweight, a.grad_f64, part * a.grad_pitch + c, sums[0][i]);
      if (a.dbias) store_grad(a.dbias, a.grad_f64, part * a.grad_pitch + c, sums[1][i]);
    }
  }
}

// CTA (split, partition): rows split * teams + team, stepping by splits * teams, of its partition.
template <typename T, int VEC, int TPR, int ELEMS>
__global__ void __launch_bounds__(TPR < kLnThreads ? kLnThreads : TPR, TPR < 512 ? 2 : 1) ln_backward_kernel(LnBackwardArgs a) {
  using Row = LnRow<T, VEC, TPR, ELEMS>;
  constexpr int kTeams = Row::kTeams;
  constexpr int kStages = ln_stages<T, TPR, ELEMS, 2>;
  extern __shared__ __align__(16) uint4 ring_memory[];
  typename Row::Group* ring = reinterpret_cast<typename Row::Group*>(ring_memory);      // stages x 2 (x, dy) x groups x threads
  __shared__ SumSlots<2> slots;
  const int tid = threadIdx.x & (TPR - 1), team = threadIdx.x / TPR, cols = (int)a.cols;
  const int split = blockIdx.x, part = blockIdx.y;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.dx);
  constexpr LnSkip kSkip = ln_backward_skip<T, VEC, TPR>;
  const int with_columns = Row::steps(cols, tid);
  const int copy_steps = kSkip.copies ? with_columns : Row::kSteps, load_steps = kSkip.loads ? with_columns : Row::kSteps;
  const int steps = kSkip.work ? with_columns : Row::kSteps;
  const float inv_n = 1.0f / (float)cols;
  const int64_t stride = (int64_t)a.splits * kTeams, end = (int64_t)(part + 1) * a.rows_per_part;
  int64_t row = (int64_t)part * a.rows_per_part + (int64_t)split * kTeams + team;
  if constexpr (Row::kRing) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) {
      const int64_t at = row + s * stride;
      if (at < end) {
        Row::issue(ring + s * 2 * Row::kStageGroups, x + at * a.x_pitch, cols, tid, copy_steps);
        Row::issue(ring + (s * 2 + 1) * Row::kStageGroups, dy + at * a.dy_pitch, cols, tid, copy_steps);
      }
      copies_commit();
    }
  }
  float next_mean = 0.0f, next_rstd = 0.0f;               // of the row after the one that is worked on
  if (row < end) {
    next_mean = a.mean[row];
    next_rstd = a.rstd[row];
  }
  Float2 w[ELEMS / 2], dw[ELEMS / 2], db[ELEMS / 2];
  Row::params(w, a.weight, a.param_f32, a.dtype, 1.0f, cols, tid);
#pragma unroll
  for (int i = 0; i < ELEMS / 2; ++i) dw[i] = db[i] = both(0.0f);
  int turn = 0, stage = 0;
  for (; row < end; row += stride) {
    const float mean = next_mean, rstd = next_rstd;
    if (row + stride < end) {
      next_mean = a.mean[row + stride];
      next_rstd = a.rstd[row + stride];
    }
    const Float2 minus_mean = both(-mean), scale = both(rstd);
    Float2 s0 = both(0.0f), s1 = both(0.0f);
    typename Row::Group* words = ring + stage * 2 * Row::kStageGroups;
    Float2 xh[ELEMS / 2], g[ELEMS / 2];
    if constexpr (Row::kRing) copies_wait<kStages - 1>();
    Row::take(xh, words, x + row * a.x_pitch, cols, tid, load_steps);
    Row::take(g, words + Row::kStageGroups, dy + row * a.dy_pitch, cols, tid, load_steps);
    if constexpr (Row::kRing) {
      const int64_t ahead = row + kStages * stride;       // into the words just read
      if (ahead < end) {
        Row::issue(words, x + ahead * a.x_pitch, cols, tid, copy_steps);
        Row::issue(words + Row::kStageGroups, dy + ahead * a.dy_pitch, cols, tid, copy_steps);
      }
      copies_commit();
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }
#pragma unroll
    for (int s = 0; s < Row::kSteps; ++s) {
      if (s > 0 && s >= steps) break;
#pragma unroll
      for (int i = s * Row::kStep / 2; i < (s + 1) * Row::kStep / 2; ++i) {               // (outside the row dy and w are 0)
        xh[i] = mul2(add2(xh[i], minus_mean), scale);
        dw[i] = fma2(g[i], xh[i], dw[i]);
        db[i] = add2(db[i], g[i]);
        g[i] = mul2(g[i], w[i]);
        s0 = add2(s0, g[i]);
        s1 = fma2(g[i], xh[i], s1);
      }
    }
    if (dx) {
      float sums[2] = {sum_of(s0), sum_of(s1)};
      team_sum<TPR>(sums, slots, turn, team);
      const Float2 minus_m0 = both(-sums[0] * inv_n), minus_m1 = both(-sums[1] * inv_n);
#pragma unroll
      for (int s = 0; s < Row::kSteps; ++s) {
        if (s > 0 && s >= steps) break;
#pragma unroll
        for (int i = s * Row::kStep / 2; i < (s + 1) * Row::kStep / 2; ++i) g[i] = mul2(fma2(xh[i], minus_m1, add2(g[i], minus_m0)), scale);
      }
      Row::store(dx + row * a.dx_pitch, g, cols, tid);
    }
  }
  pdl_trigger();                               // the kernel that adds up the partial sums may take its place (it waits for this one)
  if (!a.dweight && !a.dbias) return;
  float sums[2][ELEMS];                        // weight, bias
#pragma unroll
  for (int i = 0; i < ELEMS; i += 2) {
    unpack2(dw[i / 2], sums[0][i], sums[0][i + 1]);
    unpack2(db[i / 2], sums[1][i], sums[1][i + 1]);
  }
  if constexpr (kTeams > 1) {                  // add the teams' sums, in team order
    float* combine = reinterpret_cast<float*>(ring_memory);
    if constexpr (VEC > 1) copies_wait<0>();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < ELEMS; ++i) combine[(team * ELEMS + i) * TPR + tid] = sums[which][i];
      __syncthreads();
      if (team == 0) {
#pragma unroll
        for (int i = 0; i < ELEMS; ++i)
          for (int t = 1; t < kTeams; ++t) sums[which][i] += combine[(t * ELEMS + i) * TPR + tid];
      }
    }
    if (team != 0) return;
  }
  put_param_sums<Row, VEC, ELEMS>(a, sums, reinterpret_cast<float*>(ring_memory), part, split, tid);
}

// Rows of 8193 .. 16384 elements: a row a CTA of 1024 threads, whose 64 registers hold the sums of 16 columns but not the row and
// the weight beside them.  So the weight sits in shared memory, and the row is taken from the ring twice: for the sums, and
// again, piece by piece, for dx; each piece of the ring is refilled as soon as it has been taken for the second time.
// (15 x 64 rows of 12000 bfloat16 with all of it in registers, which spilled 312 bytes a thread: 49 us; so: 30 to 32.  Pieces of a
// word or four elements: 4000 x 15001 float32 190 us, of two 240; 4000 x 15002 bfloat16 131, of two 136; of eight 211, 130.)
template <typename T>
constexpr int ln_broad_stages = sizeof(T) == 2 ? 2 : 1;      // 64 KB of weights and 64 or 128 KB a stage
template <typename T, int VEC>
__global__ void __launch_bounds__(1024) ln_backward_broad_kernel(LnBackwardArgs a) {
  constexpr int kTeam = 1024, kElems = 16, kPiece = VEC < 4 ? 4 : VEC, kPieces = kElems / kPiece, kSpan = kPiece * kTeam;
  constexpr int kStages = ln_broad_stages<T>;
  using Row = LnRow<T, VEC, kTeam, kElems>;
  using Piece = LnRow<T, VEC, kTeam, kPiece>;                // piece k: the row's columns from k * kSpan on
  extern __shared__ __align__(16) uint4 ring_memory[];
  Float2* weights = reinterpret_cast<Float2*>(ring_memory);                             // [kElems / 2][threads]
  typename Row::Group* ring = reinterpret_cast<typename Row::Group*>(weights + kElems / 2 * kTeam);
  __shared__ SumSlots<2> slots;
  const int tid = threadIdx.x, cols = (int)a.cols, split = blockIdx.x, part = blockIdx.y;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.dx);
  const float inv_n = 1.0f / (float)cols;
  const int64_t end = (int64_t)(part + 1) * a.rows_per_part;
  int64_t row = (int64_t)part * a.rows_per_part + split;
  auto issue = [&](int stage, int k, int64_t at) {
    typename Row::Group* words = ring + stage * 2 * Row::kStageGroups + k * Piece::kStageGroups;
    const int from = k * kSpan < cols ? k * kSpan : 0, left = cols - k * kSpan;
    Piece::issue(words, x + at * a.x_pitch + from, left, tid, Piece::kSteps);
    Piece::issue(words + Row::kStageGroups, dy + at * a.dy_pitch + from, left, tid, Piece::kSteps);
  };
  if constexpr (Row::kRing) {
#pragma unroll
    for (int s = 0; s < kStages; ++s) {
      const int64_t at = row + (int64_t)s * a.splits;
      if (at < end) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) issue(s, k, at);
      }
      copies_commit();
    }
  }
  {
    Float2 w[kElems / 2];
    Row::params(w, a.weight, a.param_f32, a.dtype, 1.0f, cols, tid);
#pragma unroll
    for (int i = 0; i < kElems / 2; ++i) weights[i * kTeam + tid] = w[i];               // read by this thread only
  }
  Float2 dw[kElems / 2], db[kElems / 2];
#pragma unroll
  for (int i = 0; i < kElems / 2; ++i) dw[i] = db[i] = both(0.0f);
  int turn = 0, stage = 0;
  for (; row < end; row += a.splits) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    const Float2 minus_mean = both(-mean), scale = both(rstd);
    Float2 s0 = both(0.0f), s1 = both(0.0f);
    const typename Row::Group* words = ring + stage * 2 * Row::kStageGroups;
    const T* x_row = x + row * a.x_pitch;
    const T* dy_row = dy + row * a.dy_pitch;
    if constexpr (Row::kRing) copies_wait<kStages - 1>();
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      Float2 xh[kPiece / 2], g[kPiece / 2];
      Piece::take(xh, words + k * Piece::kStageGroups, x_row + k * kSpan, cols - k * kSpan, tid, Piece::kSteps);
      Piece::take(g, words + Row::kStageGroups + k * Piece::kStageGroups, dy_row + k * kSpan, cols - k * kSpan, tid, Piece::kSteps);
#pragma unroll
      for (int i = 0; i < kPiece / 2; ++i) {
        const int e = k * kPiece / 2 + i;
        xh[i] = mul2(add2(xh[i], minus_mean), scale);
        dw[e] = fma2(g[i], xh[i], dw[e]);
        db[e] = add2(db[e], g[i]);
        g[i] = mul2(g[i], weights[e * kTeam + tid]);
        s0 = add2(s0, g[i]);
        s1 = fma2(g[i], xh[i], s1);
      }
    }
    float s[2] = {sum_of(s0), sum_of(s1)};
    if (dx) team_sum<kTeam>(s, slots, turn, 0);
    const Float2 minus_m0 = both(-s[0] * inv_n), minus_m1 = both(-s[1] * inv_n);
    const int64_t ahead = row + (int64_t)kStages * a.splits;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      if (dx) {
        Float2 xh[kPiece / 2], g[kPiece / 2];
        Piece::take(xh, words + k * Piece::kStageGroups, x_row + k * kSpan, cols - k * kSpan, tid, Piece::kSteps);
        Piece::take(g, words + Row::kStageGroups + k * Piece::kStageGroups, dy_row + k * kSpan, cols - k * kSpan, tid, Piece::kSteps);
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) {
          xh[i] = mul2(add2(xh[i], minus_mean), scale);
          g[i] = mul2(g[i], weights[(k * kPiece / 2 + i) * kTeam + tid]);
          g[i] = mul2(fma2(xh[i], minus_m1, add2(g[i], minus_m0)), scale);
        }
        Piece::store(dx + row * a.dx_pitch + k * kSpan, g, cols - k * kSpan, tid);
      }
      if constexpr (Row::kRing) {
        if (ahead < end) issue(stage, k, ahead);
      }
    }
    if constexpr (Row::kRing) {
      copies_commit();
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }
  }
  pdl_trigger();
  if (!a.dweight && !a.dbias) return;
  float sums[2][kElems];
#pragma unroll
  for (int i = 0; i < kElems; i += 2) {
    unpack2(dw[i / 2], sums[0][i], sums[0][i + 1]);
    unpack2(db[i / 2], sums[1][i], sums[1][i + 1]);
  }
  put_param_sums<Row, VEC, kElems>(a, sums, reinterpret_cast<float*>(ring_memory), part, split, tid);
}

// Sums of the CTAs' partial sums, in a fixed order: a lane takes two columns, the splits are dealt to WARPS warps.
template <int WARPS>
__global__ void __launch_bounds__(WARPS < 8 ? 256 : WARPS * 32) ln_param_grad_kernel(LnBackwardArgs a) {
  const int part = blockIdx.y, warp = WARPS == 1 ? 0 : threadIdx.x >> 5;
  const int64_t all = 2 * a.cols;                                      // 0 .. cols - 1: weight, then bias
  const int64_t first = WARPS == 1 ? ((int64_t)blockIdx.x * 256 + threadIdx.x) * 2 : (int64_t)blockIdx.x * 64 + (threadIdx.x & 31) * 2;
  pdl_wait();
  float2 sum = make_float2(0.0f, 0.0f);
  if (first < all) {
    const float* src = a.partials + (int64_t)part * a.splits * all + first;
#pragma unroll 4
    for (int s = warp; s < a.splits; s += WARPS) {
      const float2 v = *reinterpret_cast<const float2*>(src + s * all);
      sum.x += v.x;
      sum.y += v.y;
    }
  }
  auto put = [&](int64_t c, float v) {
    if (c >= all) return;
    void* dst = c < a.cols ? a.dweight : a.dbias;
    if (dst) store_grad(dst, a.grad_f64, part * a.grad_pitch + (c < a.cols ? c : c - a.cols), v);
  };
  if constexpr (WARPS == 1) {
    put(first, sum.x);
    put(first + 1, sum.y);
  } else {
    __shared__ float2 part_s[WARPS][32];
    part_s[warp][threadIdx.x & 31] = sum;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const float* column = reinterpret_cast<const float*>(part_s) + threadIdx.x;
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) total += column[w * 64];
    put((int64_t)blockIdx.x * 64 + threadIdx.x, total);
  }
}

// ---- rows too wide for registers: one CTA a row, the row read again for every sweep (it stays in L2) ----------------------
// (Single elements, whatever the alignment: forward 4000 x 20000 bfloat16 138 us (2.3 TB/s), 512 x 20000 23; backward 45 x 8 rows of 20000
// 33 to 38.  No path of this library has rows this wide.)

constexpr int kLnWideThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kLnWideThreads) ln_forward_wide_kernel(LnForwardArgs a) {
  __shared__ SumSlots<1> slots;
  int turn = 0;
  const float inv_n = 1.0f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
    T* y = static_cast<T*>(a.y) + row * a.y_pitch;
    float sum[1] = {0.0f};
    for (int64_t c = threadIdx.x; c < a.cols; c += kLnWideThreads) sum[0] += to_float(x[c]);
    team_sum<kLnWideThreads>(sum, slots, turn, 0);
    const float mean = sum[0] * inv_n;
    float sq[1] = {0.0f};
    for (int64_t c = threadIdx.x; c < a.cols; c += kLnWideThreads) {
      const float d = to_float(x[c]) - mean;
      sq[0] = fmaf(d, d, sq[0]);
    }
    team_sum<kLnWideThreads>(sq, slots, turn, 0);
    const float rstd = rsqrtf(sq[0] * inv_n + a.eps);
    for (int64_t c = threadIdx.x; c < a.cols; c += kLnWideThreads) {
      const float w = a.weight ? param_at(a.weight, a.param_f32, a.dtype, c) : 1.0f;
      const float b = a.bias ? param_at(a.bias, a.param_f32, a.dtype, c) : 0.0f;
      y[c] = from_float<T>(fmaf((to_float(x[c]) - mean) * rstd, w, b));
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kLnWideThreads) ln_backward_wide_kernel(LnBackwardArgs a, int64_t rows) {
  __shared__ SumSlots<2> slots;
  int turn = 0;
  const float inv_n = 1.0f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
    const T* dy = static_cast<const T*>(a.dy) + row * a.dy_pitch;
    T* dx = static_cast<T*>(a.dx) + row * a.dx_pitch;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.0f, 0.0f};
    for (int64_t c = threadIdx.x; c < a.cols; c += kLnWideThreads) {
      const float g = to_float(dy[c]) * (a.weight ? param_at(a.weight, a.param_f32, a.dtype, c) : 1.0f);
      s[0] += g;
      s[1] = fmaf(g, (to_float(x[c]) - mean) * rstd, s[1]);
    }
    team_sum<kLnWideThreads>(s, slots, turn, 0);
    const float m0 = s[0] * inv_n, m1 = s[1] * inv_n;
    for (int64_t c = threadIdx.x; c < a.cols; c += kLnWideThreads) {
      const float g = to_float(dy[c]) * (a.weight ? param_at(a.weight, a.param_f32, a.dtype, c) : 1.0f);
      dx[c] = from_float<T>(rstd * (g - m0 - (to_float(x[c]) - mean) * rstd * m1));
    }
  }
}

// The parameters' partial sums of rows too wide for registers: a thread a column, a slice of a partition's rows a CTA.
template <typename T>
__global__ void __launch_bounds__(256) ln_param_partials_wide_kernel(LnBackwardArgs a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int split = blockIdx.y, part = blockIdx.z;
  if (c >= a.cols) return;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  float dw = 0.0f, db = 0.0f;
  for (int64_t r = split; r < a.rows_per_part; r += a.splits) {
    const int64_t row = (int64_t)part * a.rows_per_part + r;
    const float g = to_float(dy[row * a.dy_pitch + c]);
    dw = fmaf(g, (to_float(x[row * a.x_pitch + c]) - a.mean[row]) * a.rstd[row], dw);
    db += g;
  }
  if (a.splits > 1) {
    float* out = a.partials + ((int64_t)part * a.splits + split) * 2 * a.cols;
    out[c] = dw;
    out[a.cols + c] = db;
  } else {
    if (a.dweight) store_grad(a.dweight, a.grad_f64, part * a.grad_pitch + c, dw);
    if (a.dbias) store_grad(a.dbias, a.grad_f64, part * a.grad_pitch + c, db);
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------

// Threads of a team for rows of `cols` elements, `most` of which a thread takes at most; short rows take a half or a quarter.
struct LnTeam {
  int threads, elems;
};
static LnTeam ln_team(int64_t cols, int most) {
  if (cols <= 32 * (most / 4)) return {32, most / 4};
  if (cols <= 32 * (most / 2)) return {32, most / 2};
  int team = 32;
  while ((int64_t)team * most < cols) team *= 2;
  return {team, most};
}

static int64_t ln_min(int64_t a, int64_t b) { return a < b ? a : b; }

// CTAs that share a partition's rows.  One a SM in all, as long as every team has a row; the partitions share them evenly
// (rounded down: one more and the last CTAs would run after all others).  Two a SM where two fit (CTAs of 256 threads), if
// that leaves 8 rows to a CTA: below, writing and adding up twice the partial sums costs more than the second CTA brings
// (us with one and two, bfloat16: 45 x 16 rows of 4096 10.0, 11.1; 45 x 64 19.1, 18.0; 1 x 1024 10.3, 12.1).
// Wider rows, of which a CTA takes 256 columns: sixteen a SM, with 24 rows or more (45 x 8 rows of 20000 33 us with one, 42 with two).
constexpr int kLnSms = 148;
static int ln_splits(int64_t rows_per_part, int64_t cols, int partitions) {
  if (cols > kLnMaxCols) {
    const int64_t splits = ln_min(16 * kLnSms / (partitions * ((cols + 255) / 256)), rows_per_part / 24);
    return splits < 1 ? 1 : (int)splits;
  }
  const int team = ln_team(cols, 16).threads;
  const int teams = team < kLnThreads ? kLnThreads / team : 1;
  const int64_t two = 2 * kLnSms / partitions;
  const int64_t want = team <= kLnThreads && two * 8 <= rows_per_part ? two : kLnSms / partitions;
  const int64_t most = (rows_per_part + teams - 1) / teams;
  const int64_t splits = ln_min(want, most);
  return splits < 1 ? 1 : (int)splits;
}

// Whether rows consist of groups of `vec` elements that start on multiples of their size.
static bool grouped_rows(const void* p, int64_t pitch, int64_t cols, int dtype, int vec) {
  return ((uintptr_t)p & (vec * element_size(dtype) - 1)) == 0 && pitch % vec == 0 && cols % vec == 0;
}

template <typename T, int VEC, int TPR, int ELEMS>
static int ln_forward_launch(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
  constexpr int kTeams = kBlock / TPR;
  constexpr size_t kSmem = LnRow<T, VEC, TPR, ELEMS>::kRing ? (size_t)ln_stages<T, TPR, ELEMS, 1> * ELEMS * sizeof(T) * kBlock : 0;
  if constexpr (kSmem > 40 * 1024) SOLON_SHARED_MEMORY_ONCE((ln_forward_kernel<T, VEC, TPR, ELEMS>), kSmem);
  const int64_t want = (a.rows + kTeams - 1) / kTeams, cap = (int64_t)sms * ln_forward_ctas<VEC, TPR, ELEMS>;
  ln_forward_kernel<T, VEC, TPR, ELEMS><<<(unsigned)ln_min(want, cap), kBlock, kSmem, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T, int VEC, int TPR, int ELEMS>
static int ln_backward_launch(const LnBackwardArgs& a, int partitions, cudaStream_t stream) {
  if constexpr (TPR == 1024) {
    constexpr size_t kBytes = 1024 * ELEMS * (sizeof(float) + (VEC > 1 ? ln_broad_stages<T> * 2 * sizeof(T) : 0));
    SOLON_SHARED_MEMORY_ONCE((ln_backward_broad_kernel<T, VEC>), kBytes);
    ln_backward_broad_kernel<T, VEC><<<dim3((unsigned)a.splits, (unsigned)partitions), 1024, kBytes, stream>>>(a);
  } else {
    constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
    constexpr size_t kRing = LnRow<T, VEC, TPR, ELEMS>::kRing ? (size_t)ln_stages<T, TPR, ELEMS, 2> * 2 * ELEMS * sizeof(T) * kBlock : 0;
    constexpr size_t kCombine = TPR < kBlock ? (size_t)kBlock * ELEMS * sizeof(float) : 0;
    constexpr size_t kSmem = kRing > kCombine ? kRing : kCombine;
    if constexpr (kSmem > 40 * 1024) SOLON_SHARED_MEMORY_ONCE((ln_backward_kernel<T, VEC, TPR, ELEMS>), kSmem);
    ln_backward_kernel<T, VEC, TPR, ELEMS><<<dim3((unsigned)a.splits, (unsigned)partitions), kBlock, kSmem, stream>>>(a);
  }
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

// Rows of single elements wider than this take 32 a thread, so that two CTAs fit on an SM (8000 x 7001 bfloat16 115 -> 87 us;
// narrower ones lose by it: 30000 x 2001 70 -> 75).
constexpr int kLnWideSingle = 4096;

// f(team size, elements of a thread), both as compile-time constants, for rows of up to LIMIT columns.  A thread takes up to MOST
// elements, at least a group of VEC.
template <int MOST, int VEC, int LIMIT, typename F>
static int ln_by_team(int64_t cols, F f) {
  const LnTeam t = ln_team(cols, MOST);
  constexpr int kLeast = MOST / 4 < VEC ? VEC : MOST / 4;
  using std::integral_constant;
  switch (t.threads) {
    case 32:
      if (t.elems == MOST / 4) return f(integral_constant<int, 32>(), integral_constant<int, kLeast>());
      if (t.elems == MOST / 2) return f(integral_constant<int, 32>(), integral_constant<int, MOST / 2>());
      return f(integral_constant<int, 32>(), integral_constant<int, MOST>());
    case 64: return f(integral_constant<int, 64>(), integral_constant<int, MOST>());
    case 128: return f(integral_constant<int, 128>(), integral_constant<int, MOST>());
    case 256: return f(integral_constant<int, 256>(), integral_constant<int, MOST>());
    case 512:
      if constexpr (256 * MOST < LIMIT) return f(integral_constant<int, 512>(), integral_constant<int, MOST>());
      break;
    case 1024:
      if constexpr (512 * MOST < LIMIT) return f(integral_constant<int, 1024>(), integral_constant<int, MOST>());
      break;
  }
  return SOLON_ERR_INTERNAL;      // (wider than LIMIT)
}

// Rows that are not made of words: pairs or single elements, 16 a thread, 32 in wide rows.
template <typename T, int VEC>
static int ln_forward_loose(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  if (a.cols > 8192) return ln_forward_launch<T, VEC, 512, 32>(a, sms, stream);
  if (a.cols > kLnWideSingle) return ln_forward_launch<T, VEC, 256, 32>(a, sms, stream);
  return ln_by_team<16, VEC, kLnWideSingle>(a.cols, [&](auto team, auto elems) { return ln_forward_launch<T, VEC, team.value, elems.value>(a, sms, stream); });
}

template <typename T>
static int ln_forward_t(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  if (a.cols > kLnMaxCols) {
    const int64_t cap = (int64_t)sms * 4;
    ln_forward_wide_kernel<T><<<(unsigned)ln_min(a.rows, cap), kLnWideThreads, 0, stream>>>(a);
    SOLON_CUDA_TRY(cudaGetLastError());
    return SOLON_OK;
  }
  constexpr int kWord = 16 / (int)sizeof(T);
  auto grouped = [&](int vec) { return grouped_rows(a.x, a.x_pitch, a.cols, a.dtype, vec) && grouped_rows(a.y, a.y_pitch, a.cols, a.dtype, vec); };
  if (grouped(kWord))
    return ln_by_team<64 / (int)sizeof(T), kWord, kLnMaxCols>(a.cols, [&](auto team, auto elems) {
      return ln_forward_launch<T, kWord, team.value, elems.value>(a, sms, stream);
    });
  return grouped(2) ? ln_forward_loose<T, 2>(a, sms, stream) : ln_forward_loose<T, 1>(a, sms, stream);
}

template <typename T>
static int ln_backward_t(const LnBackwardArgs& a, int partitions, int sms, cudaStream_t stream) {
  int rc = SOLON_OK;
  if (a.cols > kLnMaxCols) {
    const int64_t rows = a.rows_per_part * partitions;
    if (a.dweight || a.dbias) {          // before dx, which may be written over dy or x
      ln_param_partials_wide_kernel<T><<<dim3((unsigned)((a.cols + 255) / 256), (unsigned)a.splits, (unsigned)partitions), 256, 0, stream>>>(a);
      SOLON_CUDA_TRY(cudaGetLastError());
    }
    if (a.dx && rows > 0) {
      ln_backward_wide_kernel<T><<<(unsigned)ln_min(rows, (int64_t)sms * 4), kLnWideThreads, 0, stream>>>(a, rows);
      SOLON_CUDA_TRY(cudaGetLastError());
    }
  } else {
    constexpr int kWord = 16 / (int)sizeof(T);
    auto grouped = [&](int vec) {
      return grouped_rows(a.x, a.x_pitch, a.cols, a.dtype, vec) && grouped_rows(a.dy, a.dy_pitch, a.cols, a.dtype, vec) &&
             (!a.dx || grouped_rows(a.dx, a.dx_pitch, a.cols, a.dtype, vec));
    };
    auto single = [&](auto team, auto elems) { return ln_backward_launch<T, 1, team.value, elems.value>(a, partitions, stream); };
    auto pairs = [&](auto team, auto elems) { return ln_backward_launch<T, 2, team.value, elems.value>(a, partitions, stream); };
    auto words = [&](auto team, auto elems) { return ln_backward_launch<T, kWord, team.value, elems.value>(a, partitions, stream); };
    if (!grouped(kWord)) {
      rc = grouped(2) ? ln_by_team<16, 2, kLnMaxCols>(a.cols, pairs) : ln_by_team<16, 1, kLnMaxCols>(a.cols, single);
    } else {
      rc = ln_by_team<16, kWord, kLnMaxCols>(a.cols, words);
    }
  }
  if (rc || a.splits == 1 || (!a.dweight && !a.dbias)) return rc;
  const int64_t columns = 2 * a.cols;
  if (a.splits < 8) return launch_dependent(ln_param_grad_kernel<1>, dim3((unsigned)((columns + 511) / 512), (unsigned)partitions), dim3(256), 0, stream, a);
  const dim3 grid((unsigned)((columns + 63) / 64), (unsigned)partitions);
  if (a.splits < 64) return launch_dependent(ln_param_grad_kernel<8>, grid, dim3(256), 0, stream, a);
  return launch_dependent(ln_param_grad_kernel<32>, grid, dim3(1024), 0, stream, a);
}

}  // namespace solon

using namespace solon;

extern "C" {

int solon_layernorm_forward(const void* x, int64_t x_pitch, int dtype, const void* weight, const void* bias, int param_dtype, int64_t rows, int64_t cols,
                            double eps, void* y, int64_t y_pitch, float* mean, float* rstd, void* cuda_stream) {
  if (!token_dtype(dtype) || (param_dtype != SOLON_F32 && param_dtype != dtype)) return SOLON_ERR_INVALID_ARG;
  if (rows < 0 || cols < 1 || cols > SOLON_MAX_COLS || !((float)eps > 0.0f && eps < INFINITY)) return SOLON_ERR_INVALID_ARG;
  if (rows == 0) return SOLON_OK;
  if (!matrix_ok(x, x_pitch, rows, cols, dtype) || !matrix_ok(y, y_pitch, rows, cols, dtype)) return SOLON_ERR_INVALID_ARG;
  if (!param_ok(weight, param_dtype) || !param_ok(bias, param_dtype) || ((uintptr_t)mean | (uintptr_t)rstd) & 3) return SOLON_ERR_INVALID_ARG;
  int sms = 0, rc;
  if ((rc = current_sms(&sms))) return rc;
  LnForwardArgs a = {x, weight, bias, y, mean, rstd, rows, cols, x_pitch, y_pitch, (float)eps, param_dtype == SOLON_F32, dtype};
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SOLON_F32) return ln_forward_t<float>(a, sms, stream);
  if (dtype == SOLON_BF16) return ln_forward_t<__nv_bfloat16>(a, sms, stream);
  return ln_forward_t<__half>(a, sms, stream);
}

int64_t solon_layernorm_backward_workspace(int64_t rows, int64_t cols, int partitions) {
  if (rows < 0 || cols < 1 || cols > SOLON_MAX_COLS || partitions < 1 || partitions > SOLON_MAX_NODES || rows % partitions) return SOLON_ERR_INVALID_ARG;
  const int splits = ln_splits(rows / partitions, cols, partitions);
  return splits == 1 ? 0 : (int64_t)partitions * splits * 2 * cols * (int64_t)sizeof(float);
}

int solon_layernorm_backward(const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, int dtype, const void* weight, int param_dtype,
                             const float* mean, const float* rstd, int64_t rows, int64_t cols, int partitions, void* dx, int64_t dx_pitch, void* dweight,
                             void* dbias, int64_t grad_pitch, int grad_dtype, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!token_dtype(dtype) || (param_dtype != SOLON_F32 && param_dtype != dtype)) return SOLON_ERR_INVALID_ARG;
  const int64_t need = solon_layernorm_backward_workspace(rows, cols, partitions);
  if (need < 0) return SOLON_ERR_INVALID_ARG;
  if (rows > 0 && (!matrix_ok(dy, dy_pitch, rows, cols, dtype) || !matrix_ok(x, x_pitch, rows, cols, dtype) || !mean || !rstd ||
                   (dx && !matrix_ok(dx, dx_pitch, rows, cols, dtype))))
    return SOLON_ERR_INVALID_ARG;
  if (!param_ok(weight, param_dtype) || ((uintptr_t)mean | (uintptr_t)rstd) & 3) return SOLON_ERR_INVALID_ARG;
  if (dweight || dbias) {
    if (grad_dtype != SOLON_F32 && grad_dtype != SOLON_F64) return SOLON_ERR_INVALID_ARG;
    if (grad_pitch < cols && partitions > 1) return SOLON_ERR_INVALID_ARG;
    if (!param_ok(dweight, grad_dtype) || !param_ok(dbias, grad_dtype)) return SOLON_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))) return SOLON_ERR_INVALID_ARG;
  } else if (!dx || rows == 0) {
    return SOLON_OK;
  }
  int sms = 0, rc;
  if ((rc = current_sms(&sms))) return rc;
  LnBackwardArgs a = {};
  a.dy = dy;
  a.x = x;
  a.weight = weight;
  a.mean = mean;
  a.rstd = rstd;
  a.dx = rows > 0 ? dx : nullptr;
  a.dweight = dweight;
  a.dbias = dbias;
  a.partials = static_cast<float*>(workspace);
  a.rows_per_part = rows / partitions;
  a.cols = cols;
  a.dy_pitch = dy_pitch;
  a.x_pitch = x_pitch;
  a.dx_pitch = dx_pitch;
  a.grad_pitch = grad_pitch;
  a.splits = ln_splits(a.rows_per_part, cols, partitions);
  a.param_f32 = param_dtype == SOLON_F32;
  a.dtype = dtype;
  a.grad_f64 = grad_dtype == SOLON_F64;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SOLON_F32) return ln_backward_t<float>(a, partitions, sms, stream);
  if (dtype == SOLON_BF16) return ln_backward_t<__nv_bfloat16>(a, partitions, sms, stream);
  return ln_backward_t<__half>(a, partitions, sms, stream);
}

}  // extern "C"
