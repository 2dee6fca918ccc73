// Statistics of rows of logits: largest, and sums of e^(z - M) and e^(z - M) (z - M) against it, for the kernels of head.cu and head_rows.cu.
#pragma once

#include "elements.cuh"

namespace solon {

constexpr float kLog2e = 1.44269504088896f;
constexpr float kLeastLogp = -1e4f;      // p is 0 long before: log p below it makes finite products with what p is multiplied by

struct RowSums {
  float m, s, a;
};

// Joins two sets of logits: sums against the larger of the two largest logits.
__device__ __forceinline__ RowSums join(const RowSums& x, const RowSums& y) {
  RowSums r;
  r.m = max_nan(x.m, y.m);
  // (no logits, or none above -infinity: s = a = 0; and a distance that leaves nothing of a set is kept finite times its sum: 0 times infinity would be NaN)
  const float cx = x.m == -INFINITY ? 0.0f : max_nan(x.m - r.m, -1e20f), cy = y.m == -INFINITY ? 0.0f : max_nan(y.m - r.m, -1e20f);
  const float ex = exp2f(cx * kLog2e), ey = exp2f(cy * kLog2e);
  r.s = x.s * ex + y.s * ey;
  r.a = fmaf(x.s, cx, x.a) * ex + fmaf(y.s, cy, y.a) * ey;
  return r;
}

// Says that x is used after y is known: without it the compiler starts so many elements of a row at once that registers do not hold them.
__device__ __forceinline__ void in_turn(Float2& x, const Float2& y) { asm volatile("" : "+l"(x.v) : "l"(y.v)); }

// z = x if `yes`, in a form that no compiler turns into an indexed access: the row would have to lie in memory.
__device__ __forceinline__ void take_if(float& z, float x, bool yes) {
  asm("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p mov.f32 %0, %1;\n\t}" : "+f"(z) : "f"(x), "r"((int)yes));
}

// Sums of one row's part of a tile: its largest logit, S and A against it.
template <int COLUMNS>
__device__ __forceinline__ void row_sums(const float (&v)[COLUMNS], RowSums& sums) {
  float &m = sums.m, &s = sums.s, &a = sums.a;
  float big[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int i = 4; i < COLUMNS; i += 2) asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(big[i / 2 % 4]) : "f"(v[i]), "f"(v[i + 1]));
  m = max_nan(max_nan(big[0], big[1]), max_nan(big[2], big[3]));
  const float ref = m == -INFINITY ? 0.0f : m;
  Float2 minus = pack2(-ref, -ref);
  const Float2 l2e = pack2(kLog2e, kLog2e);
  Float2 s2[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)}, a2[2] = {s2[0], s2[0]};
#pragma unroll
  for (int i = 0; i < COLUMNS; i += 2) {
    if (i % 32 == 0) in_turn(minus, s2[1]);
    const Float2 c = add2(pack2(v[i], v[i + 1]), minus);
    float x, y, cx, cy;
    unpack2(mul2(c, l2e), x, y);
    unpack2(c, cx, cy);
    const Float2 e = pack2(exp2_fast(x), exp2_fast(y));
    s2[i / 2 % 2] = add2(s2[i / 2 % 2], e);
    a2[i / 2 % 2] = fma2(e, pack2(fmaxf(cx, -1e30f), fmaxf(cy, -1e30f)), a2[i / 2 % 2]);      // (0 times -infinity is not wanted; NaN is in s)
  }
  float x, y;
  unpack2(add2(s2[0], s2[1]), x, y);
  s = x + y;
  unpack2(add2(a2[0], a2[1]), x, y);
  a = x + y;
}

}  // namespace solon
