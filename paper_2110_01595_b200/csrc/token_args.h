// Checks of arguments that the row operators (layer norm, token log probabilities) share.
#pragma once

#include <atomic>

#include "solon_internal.h"

// Raises a kernel's limit of dynamic shared memory, the first time the calling function launches it on a device (the call costs
// about as much as a small launch).  Devices from 64 on are asked every time.
#define SOLON_SHARED_MEMORY_ONCE(kernel, bytes)                                                                              \
  do {                                                                                                                       \
    static std::atomic<uint64_t> solon_done__{0};                                                                            \
    int solon_dev__ = 0;                                                                                                     \
    SOLON_CUDA_TRY(cudaGetDevice(&solon_dev__));                                                                             \
    const uint64_t solon_bit__ = solon_dev__ < 64 ? 1ull << solon_dev__ : 0ull;                                              \
    if (!(solon_done__.load(std::memory_order_relaxed) & solon_bit__)) {                                                     \
      SOLON_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(bytes)));               \
      solon_done__.fetch_or(solon_bit__, std::memory_order_relaxed);                                                         \
    }                                                                                                                        \
  } while (0)

namespace solon {

inline size_t element_size(int dtype) { return dtype == SOLON_F64 ? 8 : dtype == SOLON_F32 ? 4 : 2; }

inline bool token_dtype(int dtype) { return dtype == SOLON_F32 || dtype == SOLON_BF16 || dtype == SOLON_F16; }

// A matrix of rows x cols elements whose rows start `pitch` elements apart.
inline bool matrix_ok(const void* p, int64_t pitch, int64_t rows, int64_t cols, int dtype) {
  return p && ((uintptr_t)p & (element_size(dtype) - 1)) == 0 && (pitch >= cols || rows <= 1);
}

// What a matrix or a vector (rows = 1) takes in memory.
struct Extent {
  const void* p;                         // NULL: nothing
  int64_t rows, row_bytes, pitch_bytes;
};
inline Extent extent(const void* p, int64_t rows, int64_t cols, int64_t pitch, size_t size) {
  return {rows > 0 ? p : nullptr, rows, cols * (int64_t)size, rows > 1 ? pitch * (int64_t)size : cols * (int64_t)size};
}
// Whether two of them share a byte.  Views that lie between one another's rows do not; rows are looked at only where the ranges meet.
inline bool meet(const Extent& x, const Extent& y) {
  if (!x.p || !y.p) return false;
  const Extent &a = x.rows <= y.rows ? x : y, &b = x.rows <= y.rows ? y : x;
  const intptr_t a0 = (intptr_t)a.p, b0 = (intptr_t)b.p;
  const intptr_t a1 = a0 + (a.rows - 1) * a.pitch_bytes + a.row_bytes, b1 = b0 + (b.rows - 1) * b.pitch_bytes + b.row_bytes;
  if (a1 <= b0 || b1 <= a0) return false;
  for (int64_t i = 0; i < a.rows; i++) {
    const intptr_t begin = a0 + i * a.pitch_bytes, end = begin + a.row_bytes;
    if (end <= b0 || begin >= b1) continue;
    const int64_t last = begin <= b0 ? 0 : (begin - b0) / b.pitch_bytes;       // the last row that begins before or where this one does, and the one behind it
    if (begin < b0 + last * b.pitch_bytes + b.row_bytes || (last + 1 < b.rows && b0 + (last + 1) * b.pitch_bytes < end)) return true;
  }
  return false;
}

inline bool param_ok(const void* p, int param_dtype) { return ((uintptr_t)p & (element_size(param_dtype) - 1)) == 0; }

inline int current_sms(int* sms) {
  int device = 0;
  SOLON_CUDA_TRY(cudaGetDevice(&device));
  SOLON_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
  return SOLON_OK;
}

}  // namespace solon
