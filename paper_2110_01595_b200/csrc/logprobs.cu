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

constexpr int kLpThreads = 256;

// Order of the likeliest tokens as one integer: value first (NaN above all, -0 = +0), of equal values the lower index.
__device__ __forceinline__ unsigned long long rank_key(float z, uint32_t index) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  uint32_t order = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
  if (z != z) order = 0xFFFFFFFFu;
  return ((unsigned long long)order << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long key) { return 0xFFFFFFFFu - (uint32_t)key; }

// Running softmax statistics: maximum, sum of e^(z - m), sum of e^(z - m) (z - m).
struct SoftmaxStats {
  float m, s, a;
};

__device__ __forceinline__ void stats_add(SoftmaxStats& t, float z) {
  if (z > t.m || z != z) {           // rescale to the new maximum: (z - m') = (z - m) + (m - m')
    if (t.m > -INFINITY) {
      const float d = t.m - z, f = __expf(d);
      t.a = f > 0.0f ? f * (t.a + d * t.s) : 0.0f;
      t.s *= f;
    }
    t.m = z;
    t.s += (z - z) + 1.0f;           // (NaN for an infinite or NaN logit)
  } else if (z > -INFINITY) {
    const float d = z - t.m, e = __expf(d);
    t.s += e;
    if (e > 0.0f) t.a = fmaf(e, d, t.a);       // (d may be -infinity between a type's lowest and largest values)
  }
}

__device__ __forceinline__ SoftmaxStats stats_join(const SoftmaxStats& x, const SoftmaxStats& y) {
  if (x.s != x.s) return x;
  if (y.s != y.s) return y;
  if (x.m == -INFINITY) return y;
  if (y.m == -INFINITY) return x;
  SoftmaxStats t;
  t.m = fmaxf(x.m, y.m);
  const float dx = x.m - t.m, dy = y.m - t.m, fx = __expf(dx), fy = __expf(dy);
  t.s = x.s * fx + y.s * fy;
  t.a = (fx > 0.0f ? fx * (x.a + dx * x.s) : 0.0f) + (fy > 0.0f ? fy * (y.a + dy * y.s) : 0.0f);
  return t;
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

template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprob_kernel(LogprobArgs a) {
  __shared__ SoftmaxStats stats_s[kLpThreads / 32];
  __shared__ unsigned long long key_s[kLpThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* z = static_cast<const T*>(a.logits) + row * a.pitch;
    SoftmaxStats t = {-INFINITY, 0.0f, 0.0f};
    for (int64_t c = threadIdx.x; c < a.cols; c += kLpThreads) stats_add(t, to_float(z[c]));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      SoftmaxStats o;
      o.m = __shfl_xor_sync(0xffffffffu, t.m, off);
      o.s = __shfl_xor_sync(0xffffffffu, t.s, off);
      o.a = __shfl_xor_sync(0xffffffffu, t.a, off);
      t = stats_join(t, o);
    }
    __syncthreads();
    if (lane == 0) stats_s[warp] = t;
    __syncthreads();
    t = stats_s[0];
    for (int w = 1; w < kLpThreads / 32; ++w) t = stats_join(t, stats_s[w]);
    const bool empty = t.m == -INFINITY;
    const float log_s = empty ? 0.0f : logf(t.s);
    if (threadIdx.x == 0) {
      if (a.peak) a.peak[row] = t.m;
      if (a.log_sum) a.log_sum[row] = log_s;
      if (a.entropy) a.entropy[row] = empty ? 0.0f : log_s - t.a / t.s;
      if (a.targets && a.logp) {
        const int64_t target = a.targets[row];
        float lp = 0.0f;
        if (target >= a.cols) lp = NAN;
        else if (target >= 0) lp = empty ? -INFINITY : (to_float(z[target]) - t.m) - log_s;
        a.logp[row] = lp;
      }
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.top_k; ++k) {            // the largest key below the one before
      unsigned long long best = 0;
      for (int64_t c = threadIdx.x; c < a.cols; c += kLpThreads) {
        const unsigned long long key = rank_key(to_float(z[c]), (uint32_t)c);
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, off));
      __syncthreads();
      if (lane == 0) key_s[warp] = best;
      __syncthreads();
      for (int w = 0; w < kLpThreads / 32; ++w) best = max(best, key_s[w]);
      if (threadIdx.x == 0) {
        const uint32_t c = key_index(best);
        a.top_ids[row * a.top_k + k] = c;
        a.top_logp[row * a.top_k + k] = empty ? -INFINITY : (to_float(z[c]) - t.m) - log_s;
      }
      last = best;
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
  r.zero = r.m == -INFINITY || (r.g == 0.0f && r.gh == 0.0f);
  return r;
}

__device__ __forceinline__ float logit_grad(const RowGrad& r, float z, bool hit) {
  const float lp = (z - r.m) - r.log_s;
  const float p = __expf(lp);
  float d = -r.g * p;
  if (r.gh != 0.0f && !(p == 0.0f)) d -= r.gh * p * (lp + r.h);
  return hit ? d + r.g : d;
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprob_grad_kernel(LogprobGradArgs a) {
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const T* z = static_cast<const T*>(a.logits) + row * a.pitch;
    T* dz = static_cast<T*>(a.dz) + row * a.dz_pitch;
    const RowGrad r = row_grad(a, row);
    for (int64_t c = (int64_t)blockIdx.x * kLpThreads + threadIdx.x; c < a.cols; c += (int64_t)gridDim.x * kLpThreads)
      dz[c] = r.zero ? from_float<T>(0.0f) : from_float<T>(logit_grad(r, to_float(z[c]), c == r.target));
  }
}

template <typename T>
static int logprob_launch(const LogprobArgs& a, int sms, cudaStream_t stream) {
  const int64_t cap = (int64_t)sms * 8;
  logprob_kernel<T><<<(unsigned)(a.rows < cap ? a.rows : cap), kLpThreads, 0, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T>
static int logprob_grad_launch(const LogprobGradArgs& a, cudaStream_t stream) {
  const int64_t x = (a.cols + 8 * kLpThreads - 1) / (8 * kLpThreads);
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
  if (!matrix_ok(logits, pitch, rows, vocab, dtype) || (logp && !targets)) return SOLON_ERR_INVALID_ARG;
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
