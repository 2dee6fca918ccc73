// Checks of arguments that the row operators (layer norm, token log probabilities) share.
#pragma once

#include "solon_internal.h"

namespace solon {

inline size_t element_size(int dtype) { return dtype == SOLON_F64 ? 8 : dtype == SOLON_F32 ? 4 : 2; }

inline bool token_dtype(int dtype) { return dtype == SOLON_F32 || dtype == SOLON_BF16 || dtype == SOLON_F16; }

// A matrix of rows x cols elements whose rows start `pitch` elements apart.
inline bool matrix_ok(const void* p, int64_t pitch, int64_t rows, int64_t cols, int dtype) {
  return p && ((uintptr_t)p & (element_size(dtype) - 1)) == 0 && (pitch >= cols || rows <= 1);
}

inline bool param_ok(const void* p, int param_dtype) { return ((uintptr_t)p & (element_size(param_dtype) - 1)) == 0; }

inline int current_sms(int* sms) {
  int device = 0;
  SOLON_CUDA_TRY(cudaGetDevice(&device));
  SOLON_CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
  return SOLON_OK;
}

}  // namespace solon
