// Element types of the token-model operators: conversion to and from float32, and groups of elements moved by one access.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace solon {

// Everything is computed in float32; a value is rounded to the element type once, to nearest even, where it is stored.
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(double x) { return (float)x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// N consecutive elements, aligned to their size in bytes.
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T e[N];
};

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  return *reinterpret_cast<const Pack<T, N>*>(p);
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& v) {
  *reinterpret_cast<Pack<T, N>*>(p) = v;
}

// ---- 16 bytes of a row that is read once -----------------------------------------------------------------------------

__device__ __forceinline__ uint4 load16_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Copies to shared memory that do not pass registers, in groups that a thread waits for by their number (its own copies only).
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst_smem, const void* src, bool inside) {       // 4, 8 or 16 bytes
  const int bytes = inside ? BYTES : 0;        // 0: the place is filled with zeros, nothing is read
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst_smem)), "l"(src), "r"(bytes) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"((uint32_t)__cvta_generic_to_shared(dst_smem)), "l"(src), "n"(BYTES), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy16_async(void* dst_smem, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst_smem)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The elements of 16 bytes as float32, and their largest value (NaN if there is one).
template <typename T>
struct Word16;

template <>
struct Word16<float> {
  static constexpr int kCount = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
  static constexpr uint32_t kMinusInf = 0xFF800000u;                  // two or one elements of -infinity
  static __device__ __forceinline__ uint32_t first(float v) { return *reinterpret_cast<const uint32_t*>(&v); }
  static __device__ __forceinline__ uint32_t twice(float v) { return __float_as_uint(v); }
  static __device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t low) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(w)), "f"(__uint_as_float(low)));
    return __float_as_uint(r);
  }
  static __device__ __forceinline__ uint32_t max3(uint32_t a, uint32_t b, uint32_t c) {      // (one instruction)
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return __float_as_uint(r);
  }
  static __device__ __forceinline__ float widest(uint32_t w) { return __uint_as_float(w); }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    return widest(at_least(max3(v.x, v.y, v.z), v.w));
  }
};

template <>
struct Word16<__nv_bfloat16> {
  static constexpr int kCount = 8;
  static __device__ __forceinline__ void pair(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    pair(v.x, x[0], x[1]);
    pair(v.y, x[2], x[3]);
    pair(v.z, x[4], x[5]);
    pair(v.w, x[6], x[7]);
  }
  static __device__ __forceinline__ uint32_t join(float a, float b) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) { return make_uint4(join(x[0], x[1]), join(x[2], x[3]), join(x[4], x[5]), join(x[6], x[7])); }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  static constexpr uint32_t kMinusInf = 0xFF80FF80u;
  static __device__ __forceinline__ uint32_t first(__nv_bfloat16 v) { return (kMinusInf & 0xFFFF0000u) | *reinterpret_cast<const uint16_t*>(&v); }
  static __device__ __forceinline__ uint32_t twice(float v) { return join(v, v); }
  static __device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t low) { return max2(w, low); }
  static __device__ __forceinline__ float widest(uint32_t w) {
    float a, b, r;
    pair(w, a, b);
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    return widest(max2(max2(v.x, v.y), max2(v.z, v.w)));
  }
};

template <>
struct Word16<__half> {
  static constexpr int kCount = 8;
  static __device__ __forceinline__ void pair(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    pair(v.x, x[0], x[1]);
    pair(v.y, x[2], x[3]);
    pair(v.z, x[4], x[5]);
    pair(v.w, x[6], x[7]);
  }
  static __device__ __forceinline__ uint32_t join(float a, float b) {
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(b), "f"(a));
    return w;
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) { return make_uint4(join(x[0], x[1]), join(x[2], x[3]), join(x[4], x[5]), join(x[6], x[7])); }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  static constexpr uint32_t kMinusInf = 0xFC00FC00u;
  static __device__ __forceinline__ uint32_t first(__half v) { return (kMinusInf & 0xFFFF0000u) | *reinterpret_cast<const uint16_t*>(&v); }
  static __device__ __forceinline__ uint32_t twice(float v) { return join(v, v); }
  static __device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t low) { return max2(w, low); }
  static __device__ __forceinline__ float widest(uint32_t w) {
    float a, b, r;
    pair(w, a, b);
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    return widest(max2(max2(v.x, v.y), max2(v.z, v.w)));
  }
};

// Two float32 at a time (one instruction each on sm_100).
struct Float2 {
  unsigned long long v;
};
__device__ __forceinline__ Float2 pack2(float a, float b) {
  Float2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(Float2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ Float2 add2(Float2 a, Float2 b) {
  Float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Float2 mul2(Float2 a, Float2 b) {
  Float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Float2 fma2(Float2 a, Float2 b, Float2 c) {
  Float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// 2^x by the hardware's approximation (two units in the last place), 0 below 2^-126.
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

}  // namespace solon
