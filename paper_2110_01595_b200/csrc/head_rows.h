// Few float32 rows against an output matrix, by multiply-adds (head_rows.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace solon {

struct HeadSmallArgs {
  const float *hidden, *weight;
  int64_t hidden_pitch, weight_pitch, cols, vocab;
  int rows, partitions;
  const int64_t* targets;
  float* turned;                       // up(cols, 32) x NR: hidden, column by column
  // forward
  float *partial, *target_logit;       // slots x 3 x rows; rows
  // backward
  const float *peak, *log_sum, *entropy, *grad_logp, *grad_entropy;
  float* dz;                           // (vocab + 64) x NR
  float* sums;                         // splits x rows x sums_pitch: parts of dhidden (NULL: not wanted)
  int64_t sums_pitch;
  void* dweight;                       // (NULL: not wanted)
  int64_t grad_pitch;
  int grad_dtype;
};

constexpr int kSmallForward = 32, kSmallBackward = 16;      // rows that the kernels take
constexpr int kSmallVocab = 74 * 256;                       // tokens that they are for: fewer tiles than half the SMs are gone through too slowly

int small_rows(int64_t rows);                                // the number of rows that their kernels are built for: 8, 16 or 32
int64_t small_tile();                                        // tokens of a tile of the logits
int small_splits(int64_t cols, int64_t vocab);               // parts of dhidden
int small_forward(const HeadSmallArgs& a, cudaStream_t stream);
int small_backward(const HeadSmallArgs& a, cudaStream_t stream);

}  // namespace solon
