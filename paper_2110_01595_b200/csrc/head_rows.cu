// Few float32 rows against an output matrix: logits and gradients by multiply-adds.
//
// The tensor cores would take float32 elements as two float16 pieces, which have to be made first: W read, written and read as often as there are
// products (in the backward pass twice).  With up to 32 rows (16 in the backward pass) the multiply-adds that W's elements go into once they are on the SM cost
// less than that.  Bound: reading W (twice, and writing dW, in the backward pass), or as many multiply-adds an element as there are rows (three times as many: logits, dh,
// dW) at 36 T/s: of 13 rows of 3456 over 37760 tokens 80 us of memory against 47 of multiply-adds.
//
// Logits: a CTA takes a tile of 256 tokens and brings 32 columns at a time into shared memory, two stages (three of 16 columns: 15 to 50 % slower).  Two
// sets of 128 threads share a stage's columns, so that more warps hide what each waits for (13 rows of 3456 over 37760 tokens: 213 us with one set, 167 to 186 with
// two).  A lane owns two tokens (rows 36 floats apart, so that its 16-byte reads meet no bank twice) against all rows, whose elements are broadcast.  Sums of
// 16 products are added to another.  A tile is gone through by one CTA from first to last column, so vocabularies of fewer tiles than half the SMs (below
// 18,944 tokens) take the pieces instead (9 rows of 2307 over 1702 tokens: 190 us here, 60 in pieces).
// Backward: dz of all tokens lies in memory (vocab x rows, small); one kernel then reads W's rows once more, adds dz W to dh in registers and writes dz^T h:
// a thread has four columns, and a CTA a share of the tokens, whose dh a further kernel adds up.

#include <algorithm>

#include "head_rows.h"
#include "head_sums.cuh"
#include "solon_internal.h"
#include "token_args.h"

namespace solon {

constexpr int kColumns = 32;             // of a stage
constexpr int kStride = 36;              // floats between the tokens of a stage
constexpr int kStages = 2;
constexpr int kShareTokens = 32;         // of dz at a time
constexpr int kSmallThreads = 128;       // that share a stage's tokens
constexpr int kHalves = 2;               // sets of threads that share its columns, so that there are warps enough to hide what each waits for
constexpr int kCtaThreads = kHalves * kSmallThreads;

constexpr int kTokens = 2;               // of a lane
constexpr int kTokenTile = kSmallThreads * kTokens;

template <int NR>
struct SmallStage {
  float w[kTokenTile * kStride];
  float h[kColumns * NR];
};

__global__ void __launch_bounds__(256) small_turn_kernel(const float* hidden, int64_t pitch, int rows, int64_t cols, float* out, int nr) {
  const int64_t all = (cols + kColumns - 1) / kColumns * kColumns * nr;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t k = i / nr;
    const int n = (int)(i - k * nr);
    out[i] = n < rows && k < cols ? hidden[n * pitch + k] : 0.0f;
  }
}

// Row n's factors, and whether it has a share: g counts only with a target, and nothing counts in a row of which nothing is left.
__device__ __forceinline__ bool small_share(const HeadSmallArgs& a, int n, float& g, float& gh) {
  const bool there = n < a.rows;
  g = there && a.grad_logp && a.targets[n] >= 0 ? a.grad_logp[n] : 0.0f;
  gh = there && a.grad_entropy ? a.grad_entropy[n] : 0.0f;
  return there && a.peak[n] != -INFINITY && (g != 0.0f || gh != 0.0f);
}

// BACKWARD: dz instead of statistics.  WIDE: W's rows begin at multiples of 16 bytes.
template <int NR, bool BACKWARD, bool WIDE>
__global__ void __launch_bounds__(kCtaThreads, NR <= 16 ? 2 : 1) small_logits_kernel(HeadSmallArgs a) {
  constexpr int kT = kTokens, kTile = kTokenTile;
  extern __shared__ __align__(16) char small_smem[];
  SmallStage<NR>* stages = reinterpret_cast<SmallStage<NR>*>(small_smem);
  const int t = threadIdx.x % kSmallThreads, half = threadIdx.x / kSmallThreads;
  const int64_t v0 = (int64_t)blockIdx.x * kTile;
  const int here = (int)min((int64_t)kTile, a.vocab - v0);
  const float* w = a.weight + v0 * a.weight_pitch;
  const int steps = (int)((a.cols + kColumns - 1) / kColumns);

  auto fetch = [&](int step) {
    SmallStage<NR>& s = stages[step % kStages];
    const int64_t k0 = (int64_t)step * kColumns;
    if (WIDE) {
#pragma unroll 8
      for (int i = threadIdx.x; i < kTile * (kColumns / 4); i += kCtaThreads) {
        const int r = i / (kColumns / 4), c = i % (kColumns / 4) * 4;
        const int64_t left = a.cols - (k0 + c);      // (a group that reaches over the row's end is brought element by element)
        float* to = s.w + r * kStride + c;
        const float* from = w + min(r, here - 1) * a.weight_pitch + k0 + c;
        if (left >= 4) copy16_async(to, from);
        else
#pragma unroll
          for (int e = 0; e < 4; e++) copy_async<4>(to + e, e < left ? from + e : w, e < left);
      }
    } else {
#pragma unroll 8
      for (int i = threadIdx.x; i < kTile * kColumns; i += kCtaThreads) {
        const int r = i / kColumns, c = i % kColumns;
        const bool inside = k0 + c < a.cols;
        copy_async<4>(s.w + r * kStride + c, inside ? w + min(r, here - 1) * a.weight_pitch + k0 + c : w, inside);
      }
    }
    for (int i = threadIdx.x; i < kColumns * NR / 4; i += kCtaThreads) copy16_async(s.h + 4 * i, a.turned + k0 * NR + 4 * i);
    copies_commit();
  };

  Float2 z[kT][NR / 2];
#pragma unroll
  for (int r = 0; r < kT; r++)
#pragma unroll
    for (int n = 0; n < NR / 2; n++) z[r][n] = pack2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < kStages - 1; i++) {
    if (i < steps) fetch(i);
    else copies_commit();
  }
  for (int step = 0; step < steps; step++) {
    copies_wait<kStages - 2>();
    __syncthreads();                         // the stage is here, and the one that is filled next has been gone through
    if (step + kStages - 1 < steps) fetch(step + kStages - 1);
    else copies_commit();
    const SmallStage<NR>& s = stages[step % kStages];
    Float2 sum[kT][NR / 2];
#pragma unroll
    for (int r = 0; r < kT; r++)
#pragma unroll
      for (int n = 0; n < NR / 2; n++) sum[r][n] = pack2(0.0f, 0.0f);
#pragma unroll 2
    for (int k = half * (kColumns / kHalves); k < (half + 1) * (kColumns / kHalves); k += 4) {
      Pack<float, 4> x[kT];
#pragma unroll
      for (int r = 0; r < kT; r++) x[r] = load_pack<float, 4>(s.w + (t + r * kSmallThreads) * kStride + k);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        Float2 twice[kT];
#pragma unroll
        for (int r = 0; r < kT; r++) twice[r] = pack2(x[r].e[j], x[r].e[j]);
#pragma unroll
        for (int n = 0; n < NR; n += 4) {
          const Pack<float, 4> h = load_pack<float, 4>(s.h + (k + j) * NR + n);
#pragma unroll
          for (int r = 0; r < kT; r++) {
            sum[r][n / 2] = fma2(twice[r], pack2(h.e[0], h.e[1]), sum[r][n / 2]);
            sum[r][n / 2 + 1] = fma2(twice[r], pack2(h.e[2], h.e[3]), sum[r][n / 2 + 1]);
          }
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kT; r++)
#pragma unroll
      for (int n = 0; n < NR / 2; n++) z[r][n] = add2(z[r][n], sum[r][n]);
  }
  // the halves' sums
  __syncthreads();
  float* other = reinterpret_cast<float*>(small_smem);
  if (half)
#pragma unroll
    for (int r = 0; r < kT; r++)
#pragma unroll
      for (int n = 0; n < NR / 2; n++) {
        float x, y;
        unpack2(z[r][n], x, y);
        other[(t + r * kSmallThreads) * (NR + 1) + 2 * n] = x;
        other[(t + r * kSmallThreads) * (NR + 1) + 2 * n + 1] = y;
      }
  __syncthreads();
  if (!half)
#pragma unroll
    for (int r = 0; r < kT; r++)
#pragma unroll
      for (int n = 0; n < NR / 2; n++) {
        const float* p = other + (t + r * kSmallThreads) * (NR + 1) + 2 * n;
        z[r][n] = add2(z[r][n], pack2(p[0], p[1]));
      }

  if constexpr (BACKWARD) {
    __shared__ float of_row[6][NR];                  // peak, log_sum, g, g_H, entropy, whether the row has a share
    __shared__ int64_t target[NR];
    if (!half && t < NR) {
      const bool there = t < a.rows;
      const int64_t to = there && a.targets ? a.targets[t] : -1;
      float g, gh;
      of_row[5][t] = small_share(a, t, g, gh) ? 1.0f : 0.0f;
      of_row[0][t] = there ? a.peak[t] : 0.0f;
      of_row[1][t] = there ? a.log_sum[t] : 0.0f;
      of_row[2][t] = g;
      of_row[3][t] = gh;
      of_row[4][t] = there && a.grad_entropy ? a.entropy[t] : 0.0f;
      target[t] = to;
    }
    __syncthreads();
    if (half) return;
#pragma unroll
    for (int r = 0; r < kT; r++) {
      const int64_t v = v0 + t + r * kSmallThreads;
      if (v >= a.vocab) break;
#pragma unroll
      for (int n = 0; n < NR; n += 4) {
        float d[4];
        unpack2(z[r][n / 2], d[0], d[1]);
        unpack2(z[r][n / 2 + 1], d[2], d[3]);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const float g = of_row[2][n + e], lp = (d[e] - of_row[0][n + e]) - of_row[1][n + e], p = exp2_fast(lp * kLog2e);
          float x = -p * fmaf(of_row[3][n + e], fmaxf(lp, kLeastLogp) + of_row[4][n + e], g);
          if (lp != lp) x = lp;
          if (target[n + e] == v) x += g;
          d[e] = of_row[5][n + e] != 0.0f ? x : 0.0f;
        }
        *reinterpret_cast<float4*>(a.dz + v * NR + n) = make_float4(d[0], d[1], d[2], d[3]);
      }
    }
  } else {
    // tokens by rows in shared memory, then a thread takes a row's share of the tile
    constexpr int kSegments = kCtaThreads / NR, kShare = kTile / kSegments;
    __shared__ RowSums part[kSegments][NR];
    float* turned = other;                   // (every thread its own places)
    if (!half)
#pragma unroll
    for (int r = 0; r < kT; r++)
#pragma unroll
      for (int n = 0; n < NR; n += 2) {
        float x, y;
        unpack2(z[r][n / 2], x, y);
        turned[(t + r * kSmallThreads) * (NR + 1) + n] = x;
        turned[(t + r * kSmallThreads) * (NR + 1) + n + 1] = y;
      }
    __syncthreads();
    const int n = threadIdx.x % NR, segment = threadIdx.x / NR, first = segment * kShare, last = min(first + kShare, here);
    RowSums sums = {-INFINITY, 0.0f, 0.0f};
    if (n < a.rows) {
      float m = -INFINITY;
      for (int v = first; v < last; v++) m = max_nan(m, turned[v * (NR + 1) + n]);
      const float ref = m == -INFINITY ? 0.0f : m;
      sums.m = m;
      for (int v = first; v < last; v++) {
        const float c = turned[v * (NR + 1) + n] - ref, e = exp2_fast(c * kLog2e);
        sums.s += e;
        sums.a = fmaf(e, fmaxf(c, -1e30f), sums.a);
      }
      const int64_t to = a.targets ? a.targets[n] - v0 : -1;
      if (to >= first && to < last) a.target_logit[n] = turned[to * (NR + 1) + n];
    }
    part[segment][n] = sums;
    __syncthreads();
    if (!half && t < a.rows) {
      RowSums all = part[0][t];
      for (int i = 1; i < kSegments; i++) all = join(all, part[i][t]);
      float* p = a.partial + (int64_t)blockIdx.x * 3 * a.rows + t;
      p[0] = all.m;
      p[a.rows] = all.s;
      p[2 * a.rows] = all.a;
    }
  }
}

// dh += dz W and dW_k = dz_k^T h_k for a share of the tokens and 1024 columns.  WIDE: a thread's columns lie together (everything at multiples of 16 bytes),
// otherwise 256 apart.  ONE: a single partition, so that no branch stands between the rows.  dz comes 32 tokens at a time through shared memory; W's elements of the next four tokens are on the way.
template <int NR, bool WIDE, bool ONE, typename G>
__global__ void __launch_bounds__(256) small_outer_kernel(HeadSmallArgs a) {
  __shared__ __align__(16) float dz[2][kShareTokens * NR];
  constexpr int kCols = 4;
  const int t = threadIdx.x;
  const int64_t c0 = (int64_t)blockIdx.x * 256 * kCols + (WIDE ? t * kCols : t);
  constexpr int kApart = WIDE ? 1 : 256;
  const int64_t begin = a.vocab * blockIdx.y / gridDim.y, end = a.vocab * (blockIdx.y + 1) / gridDim.y;
  const int each = a.rows / a.partitions;
  float h[NR][kCols], dh[NR][kCols];
#pragma unroll
  for (int n = 0; n < NR; n++) {
    float g, gh;
    const bool counts = small_share(a, n, g, gh);        // (what a row without a share holds may be no number)
#pragma unroll
    for (int c = 0; c < kCols; c++) {
      const int64_t col = c0 + c * kApart;
      h[n][c] = counts && col < a.cols ? a.hidden[n * a.hidden_pitch + col] : 0.0f;
      dh[n][c] = 0.0f;
    }
  }
  auto fetch = [&](int64_t v, int stage) {
    for (int i = t; i < kShareTokens * NR / 4; i += 256) copy16_async(dz[stage] + 4 * i, a.dz + v * NR + 4 * i);      // (dz has room for whole stages)
    copies_commit();
  };
  constexpr int kAhead = 4;
  float next[kAhead][kCols];
  auto load = [&](int64_t v) {
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      const float* p = a.weight + min(v + u, a.vocab - 1) * a.weight_pitch;
      if (WIDE) {
        const float4 x = c0 < a.cols ? *reinterpret_cast<const float4*>(p + c0) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        next[u][0] = x.x, next[u][1] = x.y, next[u][2] = x.z, next[u][3] = x.w;
      } else {
#pragma unroll
        for (int c = 0; c < kCols; c++) next[u][c] = c0 + c * kApart < a.cols ? p[c0 + c * kApart] : 0.0f;
      }
    }
  };
  if (begin < end) {
    fetch(begin, 0);
    load(begin);
  }
  int stage = 0;
  for (int64_t v0 = begin; v0 < end; v0 += kShareTokens, stage ^= 1) {
    if (v0 + kShareTokens < end) {
      fetch(v0 + kShareTokens, stage ^ 1);
      copies_wait<1>();
    } else copies_wait<0>();
    __syncthreads();
    for (int u0 = 0; u0 < kShareTokens && v0 + u0 < end; u0 += kAhead) {
      float w[kAhead][kCols];
#pragma unroll
      for (int u = 0; u < kAhead; u++)
#pragma unroll
        for (int c = 0; c < kCols; c++) w[u][c] = next[u][c];
      load(v0 + u0 + kAhead);
#pragma unroll
      for (int u = 0; u < kAhead; u++) {
        const int64_t v = v0 + u0 + u;
        if (v >= end) break;                 // (the same for all threads)
        float dw[kCols];
        auto store = [&](int part) {
          if (!a.dweight) return;
          G* p = (G*)a.dweight + part * a.grad_pitch + v * a.cols + c0;
          if (WIDE && sizeof(G) * kCols <= 16) {
            if (c0 >= a.cols) return;
            Pack<G, kCols> x;
#pragma unroll
            for (int c = 0; c < kCols; c++) {
              if constexpr (sizeof(G) == 8) x.e[c] = dw[c];
              else x.e[c] = from_float<G>(dw[c]);
            }
            store_pack(p, x);
          } else {
#pragma unroll
            for (int c = 0; c < kCols; c++)
              if (c0 + c * kApart < a.cols) {
                if constexpr (sizeof(G) == 8) p[c * kApart] = dw[c];
                else p[c * kApart] = from_float<G>(dw[c]);
              }
          }
        };
        int part = 0, left = each;
#pragma unroll
        for (int c = 0; c < kCols; c++) dw[c] = 0.0f;
#pragma unroll
        for (int n = 0; n < NR; n += 4) {
          const Pack<float, 4> d = load_pack<float, 4>(dz[stage] + (u0 + u) * NR + n);
#pragma unroll
          for (int e = 0; e < 4; e++) {
#pragma unroll
            for (int c = 0; c < kCols; c++) {
              dh[n + e][c] = fmaf(d.e[e], w[u][c], dh[n + e][c]);
              dw[c] = fmaf(d.e[e], h[n + e][c], dw[c]);
            }
            if (!ONE && --left == 0) {       // a partition's last row
              store(part++);
              left = part < a.partitions ? each : NR + 1;
#pragma unroll
              for (int c = 0; c < kCols; c++) dw[c] = 0.0f;
            }
          }
        }
        if (ONE) store(0);
      }
    }
    __syncthreads();
  }
  if (a.sums)
#pragma unroll
    for (int n = 0; n < NR; n++)
      if (n < a.rows)
#pragma unroll
        for (int c = 0; c < kCols; c++)
          if (c0 + c * kApart < a.cols) a.sums[((int64_t)blockIdx.y * a.rows + n) * a.sums_pitch + c0 + c * kApart] = dh[n][c];
}

// ------------------------------------------------------------------------------------------------------------ host

int small_rows(int64_t rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : 32; }
int64_t small_tile() { return kTokenTile; }

static int64_t small_slices(int64_t cols) { return (cols + 1023) / 1024; }

// 296 CTAs, of at least 64 tokens each: two an SM where the kernel takes 128 registers (up to 8 rows of a single partition at multiples of 16 bytes), otherwise one after
// the other (140 to 148 registers; 198 to 212 up to 16 rows).
int small_splits(int64_t cols, int64_t vocab) {
  const int64_t slices = small_slices(cols);
  return (int)std::max<int64_t>(1, std::min((2 * 148 + slices - 1) / slices, vocab / 64));
}

template <int NR, bool BACKWARD>
static int small_logits(const HeadSmallArgs& a, cudaStream_t stream) {
  const int64_t words = (a.cols + kColumns - 1) / kColumns * kColumns * NR;
  small_turn_kernel<<<(unsigned)std::min<int64_t>((words + 255) / 256, 592), 256, 0, stream>>>(a.hidden, a.hidden_pitch, a.rows, a.cols, a.turned, NR);
  SOLON_CUDA_TRY(cudaGetLastError());
  const unsigned tiles = (unsigned)((a.vocab + kTokenTile - 1) / kTokenTile);
  constexpr int kTurned = kTokenTile * (NR + 1) * 4, bytes = std::max<int>(kStages * sizeof(SmallStage<NR>), kTurned);
  if (!(((uintptr_t)a.weight | (uintptr_t)(a.weight_pitch * 4)) & 15)) {
    SOLON_SHARED_MEMORY_ONCE((small_logits_kernel<NR, BACKWARD, true>), bytes);
    small_logits_kernel<NR, BACKWARD, true><<<tiles, kCtaThreads, bytes, stream>>>(a);
  } else {
    SOLON_SHARED_MEMORY_ONCE((small_logits_kernel<NR, BACKWARD, false>), bytes);
    small_logits_kernel<NR, BACKWARD, false><<<tiles, kCtaThreads, bytes, stream>>>(a);
  }
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

int small_forward(const HeadSmallArgs& a, cudaStream_t stream) {
  switch (small_rows(a.rows)) {
    case 8: return small_logits<8, false>(a, stream);
    case 16: return small_logits<16, false>(a, stream);
    default: return small_logits<32, false>(a, stream);
  }
}

template <int NR, typename G>
static int small_outer(const HeadSmallArgs& a, cudaStream_t stream) {
  const dim3 grid((unsigned)small_slices(a.cols), (unsigned)small_splits(a.cols, a.vocab));
  const bool wide = a.cols % 4 == 0 && !(((uintptr_t)a.weight | (uintptr_t)(a.weight_pitch * 4)) & 15) &&
                    !(((uintptr_t)a.dweight | (uintptr_t)(a.grad_pitch * sizeof(G))) & 15);
  const bool one = a.partitions == 1 || !a.dweight;
  if (wide && one) small_outer_kernel<NR, true, true, G><<<grid, 256, 0, stream>>>(a);
  else if (wide) small_outer_kernel<NR, true, false, G><<<grid, 256, 0, stream>>>(a);
  else if (one) small_outer_kernel<NR, false, true, G><<<grid, 256, 0, stream>>>(a);
  else small_outer_kernel<NR, false, false, G><<<grid, 256, 0, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <int NR>
static int small_backward_n(const HeadSmallArgs& a, cudaStream_t stream) {
  const int rc = small_logits<NR, true>(a, stream);
  if (rc) return rc;
  if (a.grad_dtype == SOLON_F32) return small_outer<NR, float>(a, stream);
  if (a.grad_dtype == SOLON_F64) return small_outer<NR, double>(a, stream);
  return small_outer<NR, __nv_bfloat16>(a, stream);
}

int small_backward(const HeadSmallArgs& a, cudaStream_t stream) {
  return small_rows(a.rows) == 8 ? small_backward_n<8>(a, stream) : small_backward_n<16>(a, stream);
}

}  // namespace solon
