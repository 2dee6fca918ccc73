// Layer norm over the rows of a matrix, forward and backward, with the gradients of weight and bias summed per partition
// straight into the rows of the partition-gradient matrix that solon_encode reads.
//     mu = mean x, rstd = (mean (x - mu)^2 + eps)^(-1/2), xh = (x - mu) rstd, y = w xh + b
//     a = w dy,   dx = rstd (a - mean a - xh mean(a xh)),   dw_k = sum dy xh,   db_k = sum dy   (rows of partition k)
// The variance is summed over the differences from the mean (a second sweep over values that sit in registers), not as a
// difference of two sums; statistics and sums are float32.
//
// Bound by memory: 2 (forward) and 3 (backward) accesses of the matrix against about 8 and 14 flops an element.
//
// Layout: a row belongs to a team of TPR threads, 64 bytes of it each (four 16-byte words; fewer in rows of less than 2 KB), so
// that a team's two reductions cost little beside the work on the elements.  Teams of one warp meet in shuffles only, larger ones
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
constexpr int kLnForwardStages = 2;            // rows on the way per team beside the one that is worked on
// Rows in shared memory per team in the backward pass, the one that is worked on among them.
template <int TPR>
constexpr int ln_backward_stages = TPR < 1024 ? 3 : 1;

// Sum over the team, the result in every thread.  Teams of several warps alternate between two slots, so one barrier a
// sum is enough: a slot is written again only after everybody has passed the barrier of the sum in between.
template <int TPR, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* slots, int& turn, int team) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], off);
  if constexpr (TPR > 32) {
    constexpr int kWarps = TPR / 32;
    const int warp = (threadIdx.x & (TPR - 1)) >> 5;
    float* s = slots + (turn * (blockDim.x >> 5) + team * kWarps) * N;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) s[k * kWarps + warp] = v[k];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(TPR) : "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += s[k * kWarps + w];
      v[k] = sum;
    }
  }
}

__device__ __forceinline__ void copy16_async(void* dst_smem, const void* src, bool inside) {
  const int bytes = inside ? 16 : 0;           // 0: the 16 bytes are filled with zeros, nothing is read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst_smem)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Weight or bias of N neighbouring columns: float32 or the matrix's type, at any alignment.
template <typename T, int N>
__device__ __forceinline__ void param_words(float (&w)[N], const void* p, bool f32, bool aligned, int c) {
  const float* q = static_cast<const float*>(p) + c;
  const T* r = static_cast<const T*>(p) + c;
  if constexpr (N % 4 == 0) {
    if (aligned) {
      if (f32) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const Pack<float, 4> v = load_pack<float, 4>(q + i);
#pragma unroll
          for (int k = 0; k < 4; ++k) w[i + k] = v.e[k];
        }
      } else {
        const Pack<T, N> v = load_pack<T, N>(r);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = to_float(v.e[i]);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = f32 ? q[i] : to_float(r[i]);
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
  int param_f32, dtype, weight_aligned, bias_aligned;
};

// VEC: neighbouring elements an access moves - 16 bytes, or one where rows are not made of 16-byte words at 16-byte
// boundaries; those are loaded straight into registers.
template <typename T, int VEC, int TPR, int ELEMS>
__global__ void __launch_bounds__(TPR < kLnThreads ? kLnThreads : TPR, TPR < 512 ? 4 : TPR < 1024 ? 2 : 1) ln_forward_kernel(LnForwardArgs a) {
  constexpr int kGroups = ELEMS / VEC;         // accesses (with VEC > 1 words of 16 bytes)
  constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
  extern __shared__ __align__(16) uint4 ring[];           // stages x words x threads
  __shared__ __align__(16) float slots[2 * 32];
  const int tid = threadIdx.x & (TPR - 1), team = threadIdx.x / TPR;
  constexpr int kTeams = kBlock / TPR;
  const int cols = (int)a.cols;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  const float inv_n = 1.0f / (float)cols;
  int turn = 0;
  const int64_t stride = (int64_t)gridDim.x * kTeams;
  auto issue = [&](int64_t row, int stage) {
    if constexpr (VEC > 1) {
      if (row < a.rows) {
        const T* from = x + row * a.x_pitch + tid * VEC;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const bool inside = (i * TPR + tid) * VEC < cols;
          copy16_async(ring + (stage * kGroups + i) * kBlock + threadIdx.x, inside ? from + i * TPR * VEC : x, inside);
        }
      }
      copies_commit();
    }
  };
  int64_t row = (int64_t)blockIdx.x * kTeams + team;
  int stage = 0;
#pragma unroll
  for (int s = 0; s < kLnForwardStages; ++s) issue(row + s * stride, s);
  for (; row < a.rows; row += stride) {
    float v[ELEMS];
    if constexpr (VEC > 1) {
      copies_wait<kLnForwardStages - 1>();
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        float part[VEC];
        Word16<T>::unpack(ring[(stage * kGroups + i) * kBlock + threadIdx.x], part);
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[i * VEC + k] = part[k];
      }
      issue(row + kLnForwardStages * stride, stage);      // into the words just read
      stage = stage + 1 == kLnForwardStages ? 0 : stage + 1;
    } else {
      const T* from = x + row * a.x_pitch;
#pragma unroll
      for (int i = 0; i < ELEMS; ++i) v[i] = i * TPR + tid < cols ? to_float(from[i * TPR + tid]) : 0.0f;
    }
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < ELEMS; ++i) sum[0] += v[i];
    team_sum<TPR>(sum, slots, turn, team);
    const float mean = sum[0] * inv_n;
    float sq[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      if ((i * TPR + tid) * VEC < cols) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          v[i * VEC + k] -= mean;
          sq[0] = fmaf(v[i * VEC + k], v[i * VEC + k], sq[0]);
        }
      }
    }
    team_sum<TPR>(sq, slots, turn, team);
    const float rstd = rsqrtf(sq[0] * inv_n + a.eps);
    T* to = y + row * a.y_pitch;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int c = (i * TPR + tid) * VEC;
      if (c < cols) {
        float w[VEC], b[VEC], out[VEC];
        if (a.weight) param_words<T>(w, a.weight, a.param_f32, a.weight_aligned, c);
        if (a.bias) param_words<T>(b, a.bias, a.param_f32, a.bias_aligned, c);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          out[k] = v[i * VEC + k] * rstd;
          out[k] = fmaf(out[k], a.weight ? w[k] : 1.0f, a.bias ? b[k] : 0.0f);
        }
        if constexpr (VEC > 1) *reinterpret_cast<uint4*>(to + c) = Word16<T>::pack(out);
        else to[c] = from_float<T>(out[0]);
      }
    }
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
  int splits, param_f32, dtype, grad_f64, weight_aligned;
};

__device__ __forceinline__ void store_grad(void* p, int f64, int64_t i, float v) {
  if (f64) static_cast<double*>(p)[i] = (double)v;
  else static_cast<float*>(p)[i] = v;
}

// CTA (split, partition): rows split * teams + team, stepping by splits * teams, of its partition.  A row is gone through
// twice, for the sums and for dx: its words stay in shared memory in between, which is what the registers could not hold
// beside the sums of the weight's gradient.
template <typename T, int VEC, int TPR, int ELEMS>
__global__ void __launch_bounds__(TPR < kLnThreads ? kLnThreads : TPR, TPR < 512 ? 2 : 1) ln_backward_kernel(LnBackwardArgs a) {
  constexpr int kGroups = ELEMS / VEC;         // accesses (with VEC > 1 words of 16 bytes)
  constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
  constexpr int kTeams = kBlock / TPR;
  constexpr int kStages = ln_backward_stages<TPR>;
  extern __shared__ __align__(16) uint4 ring[];           // stages x 2 (x, dy) x words x threads; teams' sums at the end
  __shared__ __align__(16) float slots[2 * 32 * 2];
  const int tid = threadIdx.x & (TPR - 1), team = threadIdx.x / TPR;
  const int split = blockIdx.x, part = blockIdx.y, cols = (int)a.cols;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.dx);
  float dw[ELEMS], db[ELEMS];
#pragma unroll
  for (int i = 0; i < ELEMS; ++i) dw[i] = db[i] = 0.0f;
  const float inv_n = 1.0f / (float)cols;
  int turn = 0;
  const int64_t stride = (int64_t)a.splits * kTeams, end = (int64_t)(part + 1) * a.rows_per_part;
  int64_t row = (int64_t)part * a.rows_per_part + (int64_t)split * kTeams + team;
  float next_mean = 0.0f, next_rstd = 0.0f;               // of the row after the one that is worked on
  auto issue = [&](int64_t at, int stage) {
    if constexpr (VEC > 1) {
      if (at < end) {
        const T* from_x = x + at * a.x_pitch + tid * VEC;
        const T* from_dy = dy + at * a.dy_pitch + tid * VEC;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const bool inside = (i * TPR + tid) * VEC < cols;
          uint4* to = ring + (stage * 2 * kGroups + i) * kBlock + threadIdx.x;
          copy16_async(to, inside ? from_x + i * TPR * VEC : x, inside);
          copy16_async(to + kGroups * kBlock, inside ? from_dy + i * TPR * VEC : x, inside);
        }
      }
      copies_commit();
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) issue(row + s * stride, s);
  if (row < end) {
    next_mean = a.mean[row];
    next_rstd = a.rstd[row];
  }
  int stage = 0;
  for (; row < end; row += stride) {
    const float mean = next_mean, rstd = next_rstd;
    if (row + stride < end) {
      next_mean = a.mean[row + stride];
      next_rstd = a.rstd[row + stride];
    }
    const T* row_x = x + row * a.x_pitch;
    const T* row_dy = dy + row * a.dy_pitch;
    float hold_x[VEC > 1 ? 1 : ELEMS], hold_g[VEC > 1 ? 1 : ELEMS];       // rows without words are held in registers
    if constexpr (VEC == 1) {
#pragma unroll
      for (int i = 0; i < ELEMS; ++i) {
        const int c = i * TPR + tid;
        hold_x[i] = c < cols ? to_float(row_x[c]) : mean;
        hold_g[i] = c < cols ? to_float(row_dy[c]) : 0.0f;
      }
    } else {
      const int ahead = stage == 0 ? kStages - 1 : stage - 1;     // the words of the row before
      issue(row + (kStages - 1) * stride, ahead);
      copies_wait<kStages - 1>();
    }
    // group i of the row: xh, dy and w dy
    auto group = [&](int i, float (&xh)[VEC], float (&g)[VEC], float (&wg)[VEC]) {
      if constexpr (VEC > 1) {
        Word16<T>::unpack(ring[(stage * 2 * kGroups + i) * kBlock + threadIdx.x], xh);
        Word16<T>::unpack(ring[((stage * 2 + 1) * kGroups + i) * kBlock + threadIdx.x], g);
      } else {
        xh[0] = hold_x[i];
        g[0] = hold_g[i];
      }
      if (a.weight) {
        float w[VEC];
        const int c = (i * TPR + tid) * VEC;
        param_words<T>(w, a.weight, a.param_f32, a.weight_aligned, c < cols ? c : 0);
#pragma unroll
        for (int k = 0; k < VEC; ++k) wg[k] = g[k] * w[k];
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) wg[k] = g[k];
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) xh[k] = (xh[k] - mean) * rstd;
    };
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {        // (outside the row dy is 0)
      float xh[VEC], g[VEC], wg[VEC];
      group(i, xh, g, wg);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        dw[i * VEC + k] = fmaf(g[k], xh[k], dw[i * VEC + k]);
        db[i * VEC + k] += g[k];
        s[0] += wg[k];
        s[1] = fmaf(wg[k], xh[k], s[1]);
      }
    }
    if (dx) {
      team_sum<TPR>(s, slots, turn, team);
      const float m0 = s[0] * inv_n, m1 = s[1] * inv_n;
      T* to = dx + row * a.dx_pitch;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const int c = (i * TPR + tid) * VEC;
        if (c < cols) {
          float xh[VEC], g[VEC], out[VEC];
          group(i, xh, g, out);
#pragma unroll
          for (int k = 0; k < VEC; ++k) out[k] = rstd * (out[k] - m0 - xh[k] * m1);
          if constexpr (VEC > 1) *reinterpret_cast<uint4*>(to + c) = Word16<T>::pack(out);
          else to[c] = from_float<T>(out[0]);
        }
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  if (!a.dweight && !a.dbias) return;
  if constexpr (kTeams > 1) {                  // add the teams' sums, in team order
    float* combine = reinterpret_cast<float*>(ring);
    if constexpr (VEC > 1) copies_wait<0>();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float* mine = which ? db : dw;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < ELEMS; ++i) combine[(team * ELEMS + i) * TPR + tid] = mine[i];
      __syncthreads();
      if (team == 0) {
#pragma unroll
        for (int i = 0; i < ELEMS; ++i) {
          float sum = mine[i];
          for (int t = 1; t < kTeams; ++t) sum += combine[(t * ELEMS + i) * TPR + tid];
          mine[i] = sum;
        }
      }
    }
    if (team != 0) return;
  }
  float* out = a.splits > 1 ? a.partials + ((int64_t)part * a.splits + split) * 2 * a.cols : nullptr;
#pragma unroll
  for (int i = 0; i < ELEMS; ++i) {
    const int64_t c = ((int64_t)(i / VEC) * TPR + tid) * VEC + i % VEC;
    if (c >= a.cols) continue;
    if (out) {
      out[c] = dw[i];
      out[a.cols + c] = db[i];
    } else {
      if (a.dweight) store_grad(a.dweight, a.grad_f64, part * a.grad_pitch + c, dw[i]);
      if (a.dbias) store_grad(a.dbias, a.grad_f64, part * a.grad_pitch + c, db[i]);
    }
  }
}

// Sums of the CTAs' partial sums: 32 columns a CTA (lanes), the splits dealt to 8 warps and added up in order.
__global__ void __launch_bounds__(256) ln_param_grad_kernel(LnBackwardArgs a) {
  __shared__ float part_s[8][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = blockIdx.y;
  const int64_t c2 = (int64_t)blockIdx.x * 32 + lane;                 // 0 .. cols - 1: weight, then bias
  pdl_wait();
  const float* src = a.partials + (int64_t)part * a.splits * 2 * a.cols + c2;
  float sum = 0.0f;
  if (c2 < 2 * a.cols) {
#pragma unroll 4
    for (int s = warp; s < a.splits; s += 8) sum += src[(int64_t)s * 2 * a.cols];
  }
  part_s[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || c2 >= 2 * a.cols) return;
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += part_s[w][lane];
  const int64_t c = c2 < a.cols ? c2 : c2 - a.cols;
  void* dst = c2 < a.cols ? a.dweight : a.dbias;
  if (dst) store_grad(dst, a.grad_f64, part * a.grad_pitch + c, sum);
}

// ---- rows too wide for registers: one CTA a row, the row read again for every sweep (it stays in L2) ----------------------

constexpr int kLnWideThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kLnWideThreads) ln_forward_wide_kernel(LnForwardArgs a) {
  __shared__ float slots[2 * 32];
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
  __shared__ float slots[2 * 32 * 2];
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

// CTAs that share a partition's rows: as many as run at once (two per SM of 256 threads, one of more), shared by the
// partitions - one more and the last would run alone after all others -, as long as every CTA has a row for each of its teams.
constexpr int kLnSms = 148;
static int ln_splits(int64_t rows_per_part, int64_t cols, int partitions) {
  // (the workspace does not depend on type and alignment, so the number of teams is taken as of the smallest ones)
  const int team = cols > kLnMaxCols ? 1024 : ln_team(cols, 32).threads;
  const int teams = team < kLnThreads ? kLnThreads / team : 1;
  const int64_t want = 2 * kLnSms / partitions;
  const int64_t most = (rows_per_part + teams - 1) / teams;
  const int64_t splits = ln_min(want, most);
  return splits < 1 ? 1 : (int)splits;
}

static bool vector_rows(const void* p, int64_t pitch, int64_t cols, int dtype) {
  const int vec = (int)(16 / element_size(dtype));
  return ((uintptr_t)p & 15) == 0 && pitch % vec == 0 && cols % vec == 0;
}

template <typename T, int VEC, int TPR, int ELEMS>
static int ln_forward_launch(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
  constexpr int kTeams = kBlock / TPR;
  constexpr size_t kSmem = VEC > 1 ? (size_t)kLnForwardStages * (ELEMS / VEC) * 16 * kBlock : 0;
  if constexpr (kSmem > 40 * 1024) SOLON_CUDA_TRY(cudaFuncSetAttribute(ln_forward_kernel<T, VEC, TPR, ELEMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));
  const int64_t want = (a.rows + kTeams - 1) / kTeams, cap = (int64_t)sms * (TPR < 512 ? 4 : TPR < 1024 ? 2 : 1);
  ln_forward_kernel<T, VEC, TPR, ELEMS><<<(unsigned)ln_min(want, cap), kBlock, kSmem, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T, int VEC, int TPR, int ELEMS>
static int ln_backward_launch(const LnBackwardArgs& a, int partitions, cudaStream_t stream) {
  constexpr int kBlock = TPR < kLnThreads ? kLnThreads : TPR;
  constexpr size_t kRing = VEC > 1 ? (size_t)ln_backward_stages<TPR> * 2 * (ELEMS / VEC) * 16 * kBlock : 0;
  constexpr size_t kCombine = TPR < kBlock ? (size_t)kBlock * ELEMS * sizeof(float) : 0;
  constexpr size_t kSmem = kRing > kCombine ? kRing : kCombine;
  if constexpr (kSmem > 40 * 1024) SOLON_CUDA_TRY(cudaFuncSetAttribute(ln_backward_kernel<T, VEC, TPR, ELEMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));
  ln_backward_kernel<T, VEC, TPR, ELEMS><<<dim3((unsigned)a.splits, (unsigned)partitions), kBlock, kSmem, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

// f(team size, elements of a thread), both as compile-time constants.  16 elements with 4-byte types, and where elements are
// loaded one by one; 32 with 16-byte words of two-byte types.
template <int MOST, typename F>
static int ln_by_team(int64_t cols, F f) {
  const LnTeam t = ln_team(cols, MOST);
  switch (t.threads) {
    case 32:
      if (t.elems == MOST / 4) return f(std::integral_constant<int, 32>(), std::integral_constant<int, MOST / 4>());
      if (t.elems == MOST / 2) return f(std::integral_constant<int, 32>(), std::integral_constant<int, MOST / 2>());
      return f(std::integral_constant<int, 32>(), std::integral_constant<int, MOST>());
    case 64: return f(std::integral_constant<int, 64>(), std::integral_constant<int, MOST>());
    case 128: return f(std::integral_constant<int, 128>(), std::integral_constant<int, MOST>());
    case 256: return f(std::integral_constant<int, 256>(), std::integral_constant<int, MOST>());
    case 512: return f(std::integral_constant<int, 512>(), std::integral_constant<int, MOST>());
    default:
      if constexpr (MOST * 1024 <= kLnMaxCols) return f(std::integral_constant<int, 1024>(), std::integral_constant<int, MOST>());
      else return SOLON_ERR_INTERNAL;          // 512 threads of 32 elements hold the widest row
  }
}

template <typename T>
static int ln_forward_t(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  if (a.cols > kLnMaxCols) {
    const int64_t cap = (int64_t)sms * 4;
    ln_forward_wide_kernel<T><<<(unsigned)ln_min(a.rows, cap), kLnWideThreads, 0, stream>>>(a);
    SOLON_CUDA_TRY(cudaGetLastError());
    return SOLON_OK;
  }
  const bool vec = vector_rows(a.x, a.x_pitch, a.cols, a.dtype) && vector_rows(a.y, a.y_pitch, a.cols, a.dtype);
  if (vec)
    return ln_by_team<64 / (int)sizeof(T)>(a.cols, [&](auto team, auto elems) {
      return ln_forward_launch<T, 16 / (int)sizeof(T), team.value, elems.value>(a, sms, stream);
    });
  return ln_by_team<16>(a.cols, [&](auto team, auto elems) { return ln_forward_launch<T, 1, team.value, elems.value>(a, sms, stream); });
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
    const bool vec = vector_rows(a.x, a.x_pitch, a.cols, a.dtype) && vector_rows(a.dy, a.dy_pitch, a.cols, a.dtype) &&
                     (!a.dx || vector_rows(a.dx, a.dx_pitch, a.cols, a.dtype));
    if (vec)
      rc = ln_by_team<64 / (int)sizeof(T)>(a.cols, [&](auto team, auto elems) {
        return ln_backward_launch<T, 16 / (int)sizeof(T), team.value, elems.value>(a, partitions, stream);
      });
    else
      rc = ln_by_team<16>(a.cols, [&](auto team, auto elems) { return ln_backward_launch<T, 1, team.value, elems.value>(a, partitions, stream); });
  }
  if (rc || a.splits == 1 || (!a.dweight && !a.dbias)) return rc;
  return launch_dependent(ln_param_grad_kernel, dim3((unsigned)((2 * a.cols + 31) / 32), (unsigned)partitions), dim3(256), 0, stream, a);
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
  LnForwardArgs a = {x, weight, bias, y, mean, rstd, rows, cols, x_pitch, y_pitch, (float)eps, param_dtype == SOLON_F32, dtype,
                     ((uintptr_t)weight & 15) == 0, ((uintptr_t)bias & 15) == 0};
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
  a.weight_aligned = ((uintptr_t)weight & 15) == 0;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SOLON_F32) return ln_backward_t<float>(a, partitions, sms, stream);
  if (dtype == SOLON_BF16) return ln_backward_t<__nv_bfloat16>(a, partitions, sms, stream);
  return ln_backward_t<__half>(a, partitions, sms, stream);
}

}  // extern "C"
