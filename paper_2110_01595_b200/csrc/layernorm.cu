// Layer norm over the rows of a matrix, forward and backward, with the gradients of weight and bias summed per partition
// straight into the rows of the partition-gradient matrix that solon_encode reads.
//     mu = mean x, rstd = (mean (x - mu)^2 + eps)^(-1/2), xh = (x - mu) rstd, y = w xh + b
//     a = w dy,   dx = rstd (a - mean a - xh mean(a xh)),   dw_k = sum dy xh,   db_k = sum dy   (rows of partition k)
// The variance is summed over the differences from the mean (a second sweep over values that sit in registers), not as a
// difference of two sums; statistics and sums are float32.
//
// Bound by memory: 2 (forward) and 3 (backward) accesses of the matrix against about 8 and 14 flops an element.
//
// Layout: a row belongs to a team of TPR threads that hold it in registers, up to 16 elements each (VEC neighbours an access);
// teams of one warp meet in shuffles only, larger ones also in shared memory.  CTAs stay for many rows, so that weight and
// bias are read once a CTA and the weight's gradient is summed in registers; only one partial sum per CTA and column leaves
// it, added up per partition by a second kernel in a fixed order.
#include <math.h>

#include "elements.cuh"
#include "solon_internal.h"
#include "token_args.h"

namespace solon {

constexpr int kLnElems = 16;                 // elements of a row per thread
constexpr int kLnMaxTeam = 1024;
constexpr int kLnMaxCols = kLnElems * kLnMaxTeam;      // wider rows take the streaming kernels

// Sum over the team, the result in every thread.  Teams of several warps alternate between two slots, so one barrier a
// sum is enough: a slot is written again only after everybody has passed the barrier of the sum in between.
template <int TPR, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* slots, int& turn, int team) {
#pragma unroll
  for (int off = (TPR < 32 ? TPR : 32) / 2; off > 0; off >>= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], off);
  if constexpr (TPR > 32) {
    constexpr int kWarps = TPR / 32;
    const int warp = (threadIdx.x & (TPR - 1)) >> 5;
    float* s = slots + (turn * (blockDim.x >> 5) + team * kWarps) * N;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) s[warp * N + k] = v[k];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(TPR) : "memory");
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += s[w * N + k];
      v[k] = sum;
    }
  }
}

template <typename T, int VEC>
__device__ __forceinline__ void load_row(float (&x)[kLnElems], const T* row, int64_t cols, int tid, int tpr) {
#pragma unroll
  for (int i = 0; i < kLnElems / VEC; ++i) {
    const int64_t c = ((int64_t)i * tpr + tid) * VEC;
    if (c < cols) {
      const Pack<T, VEC> v = load_pack<T, VEC>(row + c);
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[i * VEC + k] = to_float(v.e[k]);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[i * VEC + k] = 0.0f;
    }
  }
}

template <typename T, int VEC>
__device__ __forceinline__ void store_row(T* row, const float (&x)[kLnElems], int64_t cols, int tid, int tpr) {
#pragma unroll
  for (int i = 0; i < kLnElems / VEC; ++i) {
    const int64_t c = ((int64_t)i * tpr + tid) * VEC;
    if (c < cols) {
      Pack<T, VEC> v;
#pragma unroll
      for (int k = 0; k < VEC; ++k) v.e[k] = from_float<T>(x[i * VEC + k]);
      store_pack<T, VEC>(row + c, v);
    }
  }
}

// Weight or bias of a thread's columns: float32 or the matrix's type, read element by element (once per CTA).
__device__ __forceinline__ float param_at(const void* p, int is_f32, int dtype, int64_t c) {
  if (is_f32) return static_cast<const float*>(p)[c];
  if (dtype == SOLON_BF16) return to_float(static_cast<const __nv_bfloat16*>(p)[c]);
  return to_float(static_cast<const __half*>(p)[c]);
}

template <int VEC>
__device__ __forceinline__ void load_params(float (&w)[kLnElems], const void* p, int is_f32, int dtype, float absent, int64_t cols, int tid, int tpr) {
#pragma unroll
  for (int i = 0; i < kLnElems; ++i) {
    const int64_t c = ((int64_t)(i / VEC) * tpr + tid) * VEC + i % VEC;
    w[i] = c < cols ? (p ? param_at(p, is_f32, dtype, c) : absent) : 0.0f;
  }
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

template <typename T, int VEC, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) ln_forward_kernel(LnForwardArgs a) {
  __shared__ float slots[2 * 32];
  const int tid = threadIdx.x & (TPR - 1), team = threadIdx.x / TPR, teams = blockDim.x / TPR;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  float w[kLnElems], b[kLnElems];
  load_params<VEC>(w, a.weight, a.param_f32, a.dtype, 1.0f, a.cols, tid, TPR);
  load_params<VEC>(b, a.bias, a.param_f32, a.dtype, 0.0f, a.cols, tid, TPR);
  const float inv_n = 1.0f / (float)a.cols;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * teams + team; row < a.rows; row += (int64_t)gridDim.x * teams) {
    float v[kLnElems];
    load_row<T, VEC>(v, x + row * a.x_pitch, a.cols, tid, TPR);
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kLnElems; ++i) sum[0] += v[i];
    team_sum<TPR>(sum, slots, turn, team);
    const float mean = sum[0] * inv_n;
    float sq[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kLnElems; ++i) {
      const int64_t c = ((int64_t)(i / VEC) * TPR + tid) * VEC;      // (VEC divides cols: a group is inside or outside)
      v[i] -= mean;
      if (c < a.cols) sq[0] = fmaf(v[i], v[i], sq[0]);
    }
    team_sum<TPR>(sq, slots, turn, team);
    const float rstd = rsqrtf(sq[0] * inv_n + a.eps);
#pragma unroll
    for (int i = 0; i < kLnElems; ++i) v[i] = fmaf(v[i] * rstd, w[i], b[i]);
    store_row<T, VEC>(y + row * a.y_pitch, v, a.cols, tid, TPR);
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

// CTA (split, partition): rows split * teams + team, stepping by splits * teams, of its partition.
template <typename T, int VEC, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) ln_backward_kernel(LnBackwardArgs a) {
  extern __shared__ float combine[];           // teams x TPR x kLnElems (teams > 1)
  __shared__ float slots[2 * 32 * 2];
  const int tid = threadIdx.x & (TPR - 1), team = threadIdx.x / TPR, teams = blockDim.x / TPR;
  const int split = blockIdx.x, part = blockIdx.y;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  T* dx = static_cast<T*>(a.dx);
  float w[kLnElems], dw[kLnElems], db[kLnElems];
  load_params<VEC>(w, a.weight, a.param_f32, a.dtype, 1.0f, a.cols, tid, TPR);
#pragma unroll
  for (int i = 0; i < kLnElems; ++i) dw[i] = db[i] = 0.0f;
  const float inv_n = 1.0f / (float)a.cols;
  int turn = 0;
  for (int64_t r = (int64_t)split * teams + team; r < a.rows_per_part; r += (int64_t)a.splits * teams) {
    const int64_t row = (int64_t)part * a.rows_per_part + r;
    float xv[kLnElems], g[kLnElems];
    load_row<T, VEC>(xv, x + row * a.x_pitch, a.cols, tid, TPR);
    load_row<T, VEC>(g, dy + row * a.dy_pitch, a.cols, tid, TPR);
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kLnElems; ++i) {       // (outside the row g and w are 0)
      xv[i] = (xv[i] - mean) * rstd;
      dw[i] = fmaf(g[i], xv[i], dw[i]);
      db[i] += g[i];
      g[i] *= w[i];
      s[0] += g[i];
      s[1] = fmaf(g[i], xv[i], s[1]);
    }
    if (dx) {
      team_sum<TPR>(s, slots, turn, team);
      const float m0 = s[0] * inv_n, m1 = s[1] * inv_n;
#pragma unroll
      for (int i = 0; i < kLnElems; ++i) g[i] = rstd * (g[i] - m0 - xv[i] * m1);
      store_row<T, VEC>(dx + row * a.dx_pitch, g, a.cols, tid, TPR);
    }
  }
  if (!a.dweight && !a.dbias) return;
  if constexpr (TPR < 256) {                   // add the teams' sums, in team order
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float* mine = which ? db : dw;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kLnElems; ++i) combine[(team * kLnElems + i) * TPR + tid] = mine[i];
      __syncthreads();
      if (team == 0) {
#pragma unroll
        for (int i = 0; i < kLnElems; ++i) {
          float sum = 0.0f;
          for (int t = 0; t < teams; ++t) sum += combine[(t * kLnElems + i) * TPR + tid];
          mine[i] = sum;
        }
      }
    }
    if (team != 0) return;
  }
  float* out = a.splits > 1 ? a.partials + ((int64_t)part * a.splits + split) * 2 * a.cols : nullptr;
#pragma unroll
  for (int i = 0; i < kLnElems; ++i) {
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
  if (c2 < 2 * a.cols)
    for (int s = warp; s < a.splits; s += 8) sum += src[(int64_t)s * 2 * a.cols];
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

static int ln_team(int64_t cols) {
  int team = 32;
  while ((int64_t)team * kLnElems < cols) team *= 2;
  return team;
}

static int64_t ln_min(int64_t a, int64_t b) { return a < b ? a : b; }

// CTAs that share a partition's rows: two per SM over all partitions, as long as every CTA has a row for each of its teams.
static int ln_splits(int64_t rows_per_part, int64_t cols, int partitions) {
  const int teams = cols > kLnMaxCols ? 1 : (ln_team(cols) < 256 ? 256 / ln_team(cols) : 1);
  const int64_t want = (2 * 148 + partitions - 1) / partitions;
  const int64_t most = (rows_per_part + teams - 1) / teams;
  const int64_t splits = ln_min(want, most);
  return splits < 1 ? 1 : (int)splits;
}

static bool vector_rows(const void* p, int64_t pitch, int64_t cols, int dtype) {
  const int vec = (int)(16 / element_size(dtype));
  return ((uintptr_t)p & 15) == 0 && pitch % vec == 0 && cols % vec == 0;
}

template <typename T, int VEC, int TPR>
static int ln_forward_launch(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR;
  constexpr int kTeams = kThreads / TPR;
  const int64_t want = (a.rows + kTeams - 1) / kTeams, cap = (int64_t)sms * (2048 / kThreads);
  ln_forward_kernel<T, VEC, TPR><<<(unsigned)ln_min(want, cap), kThreads, 0, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T, int VEC>
static int ln_forward_team(const LnForwardArgs& a, int sms, cudaStream_t stream) {
  switch (ln_team(a.cols)) {
    case 32: return ln_forward_launch<T, VEC, 32>(a, sms, stream);
    case 64: return ln_forward_launch<T, VEC, 64>(a, sms, stream);
    case 128: return ln_forward_launch<T, VEC, 128>(a, sms, stream);
    case 256: return ln_forward_launch<T, VEC, 256>(a, sms, stream);
    case 512: return ln_forward_launch<T, VEC, 512>(a, sms, stream);
    default: return ln_forward_launch<T, VEC, 1024>(a, sms, stream);
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
  if (vector_rows(a.x, a.x_pitch, a.cols, a.dtype) && vector_rows(a.y, a.y_pitch, a.cols, a.dtype))
    return ln_forward_team<T, 16 / (int)sizeof(T)>(a, sms, stream);
  return ln_forward_team<T, 1>(a, sms, stream);
}

template <typename T, int VEC, int TPR>
static int ln_backward_launch(const LnBackwardArgs& a, int partitions, cudaStream_t stream) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR;
  const size_t smem = TPR < 256 ? (size_t)kThreads * kLnElems * sizeof(float) : 0;
  ln_backward_kernel<T, VEC, TPR><<<dim3((unsigned)a.splits, (unsigned)partitions), kThreads, smem, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T, int VEC>
static int ln_backward_team(const LnBackwardArgs& a, int partitions, cudaStream_t stream) {
  switch (ln_team(a.cols)) {
    case 32: return ln_backward_launch<T, VEC, 32>(a, partitions, stream);
    case 64: return ln_backward_launch<T, VEC, 64>(a, partitions, stream);
    case 128: return ln_backward_launch<T, VEC, 128>(a, partitions, stream);
    case 256: return ln_backward_launch<T, VEC, 256>(a, partitions, stream);
    case 512: return ln_backward_launch<T, VEC, 512>(a, partitions, stream);
    default: return ln_backward_launch<T, VEC, 1024>(a, partitions, stream);
  }
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
    rc = vec ? ln_backward_team<T, 16 / (int)sizeof(T)>(a, partitions, stream) : ln_backward_team<T, 1>(a, partitions, stream);
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
