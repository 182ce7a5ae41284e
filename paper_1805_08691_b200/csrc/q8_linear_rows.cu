// The product with a factor per token without scratch, for any operands.
//
//   D[16 output channels, 8 NT tokens] (int32, registers) = W[16, C] (from global memory) x Z[8 NT, C]^T (shared memory)
//
// A block takes 16 output channels and 8 NT tokens; its eight warps share the channels of the reduction, 64 at a time each.
// The order of the products inside mma.sync is free as long as both operands share it, so a lane's 16 contiguous bytes of a
// weight row are its operands of two instructions as they come, without shared memory or shuffles, and 16 bytes of a token's
// codes are the other operand.  The partial sums of the warps meet in shared memory (integers: any order, same result).
// Floating-point activations become codes while they are staged.
//
// It is there for calls without scratch, whose activations every block quantizes for itself: 64 tokens of bf16, 4096 -> 4096
// 195 us (8.6 with scratch); 300 tokens of codes off the grid, 1001 -> 130 12.9 us (8.3).
#include "q8_linear.h"
#include <atomic>

#include "q8_token_common.cuh"

namespace q8 {
namespace {

constexpr int kRowWarps = 8, kRowThreads = 32 * kRowWarps;

struct RowsParams {
  int M, C, K;
  long long ldx, ldw, ldy;
  int x_type, y_type;
  int x_vec;     // rows of x on the 16-byte grid
  int chunk;     // channels staged at a time, a multiple of 64
  int pitch;     // bytes of a staged row
  const void* x;
  const float* x_scale;
  const signed char* w;
  const float* w_scale;
  const float* bias;
  void* y;
};

// Sixteen activations from channel c on, those from C on zero.
template <typename T>
__device__ __forceinline__ uint4 codes_16(const T* row, int c, int C, const TokenFactor& f) {
  unsigned int w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (c + j < C) w[j >> 2] |= ((unsigned int)token_code(to_f32(row[c + j]), f) & 0xffu) << (8 * (j & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ unsigned int row_max(const T* row, int C, int lane) {
  unsigned int m = 0;
  for (int c = lane; c < C; c += 32) m = max(m, abs_word(to_f32(row[c])));
  return warp_max(m);
}

template <int NT, bool kAligned>
__global__ void __launch_bounds__(kRowThreads) linear_rows_kernel(const __grid_constant__ RowsParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ TokenFactor s_fac[8 * NT];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, i = lane & 3;
  const int n0 = blockIdx.x * 16, t0 = blockIdx.y * 8 * NT, toks = min(8 * NT, p.M - t0);
  if (p.x_type != Q8_S8) {
    for (int t = warp; t < toks; t += kRowWarps) {
      const long long o = (long long)(t0 + t) * p.ldx;
      unsigned int m;
      if (p.x_type == Q8_F32) m = row_max(static_cast<const float*>(p.x) + o, p.C, lane);
      else if (p.x_type == Q8_F16) m = row_max(static_cast<const __half*>(p.x) + o, p.C, lane);
      else m = row_max(static_cast<const __nv_bfloat16*>(p.x) + o, p.C, lane);
      if (lane == 0) s_fac[t] = token_factor(m);
    }
    __syncthreads();
  }
  int acc[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0;
  const signed char* wa = p.w + (long long)min(n0 + g, p.K - 1) * p.ldw;
  const signed char* wb = p.w + (long long)min(n0 + g + 8, p.K - 1) * p.ldw;
  for (int k0 = 0; k0 < p.C; k0 += p.chunk) {
    const int len = min(p.chunk, (p.C - k0 + 63) & ~63);
    const int units = toks * (len >> 4);
    for (int u = threadIdx.x; u < units; u += kRowThreads) {
      const int t = u / (len >> 4), c = (u - t * (len >> 4)) * 16;
      const long long o = (long long)(t0 + t) * p.ldx;
      uint4 v;
      if (p.x_type == Q8_S8) {
        const signed char* row = static_cast<const signed char*>(p.x) + o;
        v = p.x_vec ? load_16<true>(row, k0 + c, p.C) : load_16<false>(row, k0 + c, p.C);
      } else if (p.x_type == Q8_F32) {
        v = codes_16(static_cast<const float*>(p.x) + o, k0 + c, p.C, s_fac[t]);
      } else if (p.x_type == Q8_F16) {
        v = codes_16(static_cast<const __half*>(p.x) + o, k0 + c, p.C, s_fac[t]);
      } else {
        v = codes_16(static_cast<const __nv_bfloat16*>(p.x) + o, k0 + c, p.C, s_fac[t]);
      }
      *reinterpret_cast<uint4*>(smem + t * p.pitch + c) = v;
    }
    __syncthreads();
    for (int c = warp * 64; c < len; c += 64 * kRowWarps) {
      const uint4 a = load_16<kAligned>(wa, k0 + c + 16 * i, p.C), b = load_16<kAligned>(wb, k0 + c + 16 * i, p.C);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint4 z = *reinterpret_cast<const uint4*>(smem + min(8 * t + g, toks - 1) * p.pitch + c + 16 * i);
        mma_16x8x32(acc[t], a.x, b.x, a.y, b.y, z.x, z.y);
        mma_16x8x32(acc[t], a.z, b.z, a.w, b.w, z.z, z.w);
      }
    }
    __syncthreads();
  }
  // partial sums [warp][token][16 channels] over the staged codes
  int* red = reinterpret_cast<int*>(smem);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) red[(warp * 8 * NT + 8 * t + 2 * i + (j & 1)) * 16 + g + 8 * (j >> 1)] = acc[t][j];
  __syncthreads();
  for (int o = threadIdx.x; o < toks * 16; o += kRowThreads) {
    const int t = o >> 4, n = n0 + (o & 15);
    if (n >= p.K) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) sum += red[w * 8 * NT * 16 + o];
    const float s = p.x_type == Q8_S8 ? p.x_scale[t0 + t] : s_fac[t].s;
    float v = __fmul_rn(__fmul_rn(__int2float_rn(sum), s), p.w_scale[n]);
    if (p.bias) v = __fadd_rn(v, p.bias[n]);
    const long long at = (long long)(t0 + t) * p.ldy + n;
    if (p.y_type == Q8_F32) static_cast<float*>(p.y)[at] = v;
    else if (p.y_type == Q8_F16) static_cast<__half*>(p.y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(v);
  }
}

template <int NT, bool kAligned>
int launch_rows(const RowsParams& p, cudaStream_t s) {
  const size_t staged = (size_t)(p.M < 8 * NT ? p.M : 8 * NT) * p.pitch, red = (size_t)kRowWarps * 8 * NT * 16 * 4;
  const size_t dyn = staged > red ? staged : red;
  static std::atomic<bool> set[kMaxDevices];
  const int dev = current_device();
  if (dev < 0 || !set[dev].load(std::memory_order_relaxed)) {
    const int rc = check_cuda(cudaFuncSetAttribute(linear_rows_kernel<NT, kAligned>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024), "linear_rows_kernel");
    if (rc != Q8_OK) return rc;
    if (dev >= 0) set[dev].store(true, std::memory_order_relaxed);
  }
  const dim3 grid((unsigned)((p.K + 15) / 16), (unsigned)((p.M + 8 * NT - 1) / (8 * NT)));
  linear_rows_kernel<NT, kAligned><<<grid, kRowThreads, dyn, s>>>(p);
  return check_launch("linear_rows_kernel");
}

}  // namespace

int launch_linear_rows(const LinearArgs& a) {
  RowsParams p;
  p.C = a.C; p.K = a.K; p.ldx = a.ldx; p.ldw = a.ldw; p.ldy = a.ldy; p.x_type = a.x_type; p.y_type = a.y_type;
  p.w = a.w; p.w_scale = a.w_scale; p.bias = a.bias;
  const size_t xe = type_bytes(a.x_type), ye = type_bytes(a.y_type);
  p.x_vec = aligned16(a.x) && a.ldx * xe % 16 == 0;
  const bool w16 = aligned16(a.w) && a.ldw % 16 == 0;
  // a grid has at most 65535 rows of blocks: longer inputs in parts
  for (int m0 = 0; m0 < a.M;) {
    const int left = a.M - m0, nt = left <= 8 ? 1 : (left <= 16 ? 2 : (left <= 32 ? 4 : 8));
    p.M = left < 65535 * 64 ? left : 65535 * 64;
    p.x = static_cast<const char*>(a.x) + (size_t)m0 * a.ldx * xe;
    p.x_scale = a.x_scale ? a.x_scale + m0 : nullptr;
    p.y = static_cast<char*>(a.y) + (size_t)m0 * a.ldy * ye;
    const int toks = p.M < 8 * nt ? p.M : 8 * nt;
    int chunk = (a.C + 63) & ~63;
    const int most = (96 * 1024 / toks - 64) & ~63;
    if (chunk > most) chunk = most;
    p.chunk = chunk;
    p.pitch = chunk % 128 == 64 ? chunk : chunk + 64;  // rows of neighbouring tokens in different halves of the banks
    int rc;
    switch (nt) {
      case 1: rc = w16 ? launch_rows<1, true>(p, a.stream) : launch_rows<1, false>(p, a.stream); break;
      case 2: rc = w16 ? launch_rows<2, true>(p, a.stream) : launch_rows<2, false>(p, a.stream); break;
      case 4: rc = w16 ? launch_rows<4, true>(p, a.stream) : launch_rows<4, false>(p, a.stream); break;
      default: rc = w16 ? launch_rows<8, true>(p, a.stream) : launch_rows<8, false>(p, a.stream); break;
    }
    if (rc != Q8_OK) return rc;
    m0 += p.M;
  }
  return Q8_OK;
}

}  // namespace q8
