// Shared by the token operators (q8_tokens.cu, q8_linear*.cu, q8_moe.cu): 16- and 32-bit floats, unaligned 16-byte loads and
// the factor and codes of a token.  Everything here has internal linkage.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "q8_internal.h"

namespace q8 {
namespace {

inline bool float_type(int t) { return t == Q8_F32 || t == Q8_F16 || t == Q8_BF16; }
inline size_t type_bytes(int t) { return t == Q8_F32 || t == Q8_S32 ? 4 : (t == Q8_F16 || t == Q8_BF16 ? 2 : 1); }
inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ unsigned int abs_word(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Factor of a token from the bits of its maximum, and the divisor of its values: RN(1/s) with two correction steps gives
// the correctly rounded quotient (Markstein, IBM J. Res. Dev. 34(1), 1990) where nothing underflows, which s >= 2^-60
// ensures for quotients that matter (|x / s| >= 0.4); other factors take the division.  |x| <= 128 s throughout.
struct TokenFactor {
  float s, r;
  int general;  // 1: divide
  int finite;   // 0: codes are 0
};
__device__ __forceinline__ TokenFactor token_factor(unsigned int max_bits) {
  TokenFactor f;
  f.finite = max_bits < 0x7f800000u;
  f.s = max_bits == 0u ? 1.0f : fmaxf(__fdiv_rn(__uint_as_float(max_bits), 127.0f), 0x1p-126f);
  f.general = !(f.s >= 0x1p-60f && f.s <= 0x1p100f);
  f.r = __frcp_rn(f.s);
  if (!f.finite) f.s = __uint_as_float(0x7fc00000u);
  return f;
}
__device__ __forceinline__ int token_code(float x, const TokenFactor& f) {
  if (!f.finite) return 0;
  float y;
  if (f.general) {
    y = __fdiv_rn(x, f.s);
  } else {
    y = __fmul_rn(x, f.r);
    y = __fmaf_rn(__fmaf_rn(-y, f.s, x), f.r, y);
    y = __fmaf_rn(__fmaf_rn(-y, f.s, x), f.r, y);
  }
  return min(max(__float2int_rn(y), -128), 127);
}

// Bytes pos .. pos + 15 of a row of `len` bytes, zero from len on; no byte outside the row is read.  kAligned: the row
// starts on the 16-byte grid and so does pos.
template <bool kAligned>
__device__ __forceinline__ uint4 load_16(const signed char* row, int pos, int len) {
  if (kAligned && pos + 16 <= len) return __ldg(reinterpret_cast<const uint4*>(row + pos));
  unsigned int w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (pos + j < len) w[j >> 2] |= (unsigned int)(unsigned char)row[pos + j] << (8 * (j & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// D (16 x 8, int32) += A (16 x 32) B (32 x 8), 8-bit integers.  Lane 4g + i holds bytes 4i..4i+3 and 16+4i.. of the rows g and
// g + 8 of A (a0, a2 and a1, a3) and of column g of B (b0, b1), and the results of row g (d0, d1) and g + 8 (d2, d3) in the
// columns 2i and 2i + 1.  The order of the 32 products is free as long as A and B share it.
__device__ __forceinline__ void mma_16x8x32(int (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ unsigned int warp_max(unsigned int m) { return __reduce_max_sync(0xffffffffu, m); }

}  // namespace
}  // namespace q8
