// Declarations shared by the translation units of q8_linear (host side).
#pragma once
#include "q8_internal.h"

namespace q8 {

struct LinearArgs {
  int M, C, K;
  long long ldx, ldw, ldy;
  int x_type, y_type;
  const void* x;
  const float* x_scale;
  const int8_t* w;
  const float* w_scale;
  const float* bias;
  void* y;
  cudaStream_t stream;
};

// Estimated times in microseconds, by which a call chooses its kernel (fitted to 60 shapes, 10 to 15 % off at the median).
// Many tokens, codes and weights on the 16-byte grid: tensor cores, tiles of 256 tokens (q8_linear_umma.cu).
double linear_umma_us(const LinearArgs& a);
int launch_linear_umma(const LinearArgs& a);
// Token counts below that: weights on the side of 128 rows, the reduction split over a cluster (q8_linear_split.cu).
double linear_split_us(const LinearArgs& a);
int launch_linear_split(const LinearArgs& a);
// Few tokens, any alignment: weights streamed through shared memory (q8_linear_stream.cu).
bool linear_stream_fits(const LinearArgs& a);
double linear_stream_us(const LinearArgs& a);
int launch_linear_stream(const LinearArgs& a);
// Everything, without scratch (q8_linear_rows.cu).
int launch_linear_rows(const LinearArgs& a);
int launch_quantize_tokens(const void* x, int x_type, size_t tokens, size_t C, size_t ldx, int8_t* z, size_t ldz, float* scale, cudaStream_t s);

}  // namespace q8
