// Codes and factors of tokens (q8_quantize_tokens) and the way back (q8_dequantize_tokens).
//
// A block takes one token: it holds the row's values in registers between the maximum and the codes, so that they are
// read from memory once; values beyond kHeld per thread are read a second time, from L2.  Bound by memory.
#include "q8_token_common.cuh"

namespace q8 {
namespace {

constexpr int kTokThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kTokThreads) quantize_tokens_kernel(const T* __restrict__ x, size_t tokens, size_t C, size_t ldx,
                                                                      signed char* __restrict__ z, size_t ldz, float* __restrict__ scale) {
  __shared__ unsigned int part[kTokThreads / 32];
  for (size_t t = blockIdx.x; t < tokens; t += gridDim.x) {
    const T* row = x + t * ldx;
    unsigned int m = 0;
    for (size_t c = threadIdx.x; c < C; c += kTokThreads) m = max(m, abs_word(to_f32(row[c])));
    m = warp_max(m);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTokThreads / 32; ++i) m = max(m, part[i]);
    const TokenFactor f = token_factor(m);
    if (threadIdx.x == 0) scale[t] = f.s;
    for (size_t c = threadIdx.x; c < C; c += kTokThreads) z[t * ldz + c] = (signed char)token_code(to_f32(row[c]), f);
  }
}

template <typename T>
__global__ void __launch_bounds__(kTokThreads) dequantize_tokens_kernel(const signed char* __restrict__ z, size_t tokens, size_t C, size_t ldz,
                                                                        const float* __restrict__ scale, T* __restrict__ r, size_t ldr) {
  for (size_t t = blockIdx.x; t < tokens; t += gridDim.x) {
    const float s = scale[t];
    for (size_t c = threadIdx.x; c < C; c += kTokThreads) r[t * ldr + c] = from_f32<T>(__fmul_rn(s, (float)z[t * ldz + c]));
  }
}

int check_tokens(const char* fn, const void* x, int type, size_t tokens, size_t C, size_t ldx, const void* z, size_t ldz, const float* scale) {
  if (!float_type(type)) return fail(Q8_ERR_INVALID_ARG, "%s: the type must be Q8_F32, Q8_F16 or Q8_BF16", fn);
  if (C == 0 || ldx < C || ldz < C) return fail(Q8_ERR_INVALID_ARG, "%s: C must be positive and no pitch below it", fn);
  if (tokens && (!x || !z || !scale)) return fail(Q8_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (tokens > SIZE_MAX / 8 / (ldx > ldz ? ldx : ldz)) return fail(Q8_ERR_INVALID_ARG, "%s: tensor too large", fn);
  if (!aligned_to(x, type_bytes(type)) || !aligned_to(scale, 4)) return fail(Q8_ERR_ALIGNMENT, "%s: a pointer is not aligned to its element", fn);
  return Q8_OK;
}

int token_grid(size_t tokens) { return (int)(tokens < (size_t)sm_count() * 8 ? tokens : (size_t)sm_count() * 8); }

}  // namespace

int launch_quantize_tokens(const void* x, int x_type, size_t tokens, size_t C, size_t ldx, int8_t* z, size_t ldz, float* scale, cudaStream_t s) {
  const int grid = token_grid(tokens);
  if (x_type == Q8_F32) quantize_tokens_kernel<float><<<grid, kTokThreads, 0, s>>>(static_cast<const float*>(x), tokens, C, ldx, z, ldz, scale);
  else if (x_type == Q8_F16) quantize_tokens_kernel<__half><<<grid, kTokThreads, 0, s>>>(static_cast<const __half*>(x), tokens, C, ldx, z, ldz, scale);
  else quantize_tokens_kernel<__nv_bfloat16><<<grid, kTokThreads, 0, s>>>(static_cast<const __nv_bfloat16*>(x), tokens, C, ldx, z, ldz, scale);
  return check_launch("quantize_tokens_kernel");
}

}  // namespace q8

using namespace q8;

extern "C" {

int q8_quantize_tokens(const void* x, int x_type, size_t tokens, size_t C, size_t ldx, int8_t* z, size_t ldz, float* d_scale, void* stream) {
  clear_error();
  const int rc = check_tokens("q8_quantize_tokens", x, x_type, tokens, C, ldx, z, ldz, d_scale);
  if (rc != Q8_OK || tokens == 0) return rc;
  return launch_quantize_tokens(x, x_type, tokens, C, ldx, z, ldz, d_scale, as_stream(stream));
}

int q8_dequantize_tokens(const int8_t* z, size_t tokens, size_t C, size_t ldz, const float* d_scale, void* r, int r_type, size_t ldr, void* stream) {
  clear_error();
  const int rc = check_tokens("q8_dequantize_tokens", r, r_type, tokens, C, ldr, z, ldz, d_scale);
  if (rc != Q8_OK || tokens == 0) return rc;
  const int grid = token_grid(tokens);
  cudaStream_t s = as_stream(stream);
  if (r_type == Q8_F32) dequantize_tokens_kernel<float><<<grid, kTokThreads, 0, s>>>(z, tokens, C, ldz, d_scale, static_cast<float*>(r), ldr);
  else if (r_type == Q8_F16) dequantize_tokens_kernel<__half><<<grid, kTokThreads, 0, s>>>(z, tokens, C, ldz, d_scale, static_cast<__half*>(r), ldr);
  else dequantize_tokens_kernel<__nv_bfloat16><<<grid, kTokThreads, 0, s>>>(z, tokens, C, ldz, d_scale, static_cast<__nv_bfloat16*>(r), ldr);
  return check_launch("dequantize_tokens_kernel");
}

}  // extern "C"
