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

// Many tokens, codes on the 16-byte grid: tensor cores fed by TMA (q8_linear_umma.cu).
int launch_linear_umma(const LinearArgs& a);
// Few tokens: weights streamed through shared memory (q8_linear_stream.cu).
constexpr int kStreamTokens = 32;
bool linear_stream_fits(const LinearArgs& a);
int launch_linear_stream(const LinearArgs& a);
// Everything else, without scratch (q8_linear_rows.cu).
int launch_linear_rows(const LinearArgs& a);
int launch_quantize_tokens(const void* x, int x_type, size_t tokens, size_t C, size_t ldx, int8_t* z, size_t ldz, float* scale, cudaStream_t s);

}  // namespace q8
