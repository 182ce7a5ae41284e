// Codes and factors of tokens (q8_quantize_tokens) and the way back (q8_dequantize_tokens).
//
// Bound by memory.  A team of threads (a warp, or a block of 128, 256 or 512) takes a token and holds its values in registers
// between the maximum and the codes, so that they are read from memory once; what a team cannot hold is read a second time,
// from L2.  Teams are as large as leaves a thread about four pieces of 16 bytes (64 bytes in flight each), and with fewer tokens
// than that occupies the GPU large enough for one each: one token of 4096 values is then 1.5 us of latency and nothing else.
// Registers are held to what five blocks of 256 threads leave (8192 x 4096 f32: 31 us, with 512 threads a row 45).
// Rows off the 16-byte grid: four 16-bit values that adjoin, or four fp32 values as far apart as the team is large, so that a
// warp's addresses adjoin (1000 x 2051 f32: 5.0 us against 5.6; 8192 x 2678 f16: 32 us against 34 the other way round), and so
// on the way back for all types (8192 x 2678 f16: 21 us against 26).
// 8192 x 4096 bf16: 21 us to codes (4.7 TB/s of 6.5 measured; half of the rest is instructions: a scheduler issues in 70 % of
// its cycles), 19 us back (5.2 TB/s); the first form here, a block a token that
// read its row twice, value by value, 73 us for both.
#include "q8_token_common.cuh"

namespace q8 {
namespace {

constexpr int kHeld = 4;  // chunks a thread holds

// Sixteen bytes of a row (V values), or four values: from `at` on, where `left` values of the row remain; those
// behind them are zero.
template <typename T, bool kVec, int kTeam>
struct Chunk {
  static constexpr int V = kVec ? 16 / (int)sizeof(T) : 4;
  static constexpr int kStep = kVec || sizeof(T) == 2 ? 1 : kTeam;  // from value to value
  unsigned w[V * sizeof(T) / 4];
  __device__ __forceinline__ void load(const T* at, int left) {
    if (kVec && V <= left) {
      *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(at);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const bool live = j * kStep < left;
        if constexpr (sizeof(T) == 4) {
          w[j] = live ? reinterpret_cast<const unsigned*>(at)[j * kStep] : 0u;
        } else {
          const unsigned h = live ? reinterpret_cast<const unsigned short*>(at)[j * kStep] : 0u;
          w[j / 2] = j & 1 ? w[j / 2] | h << 16 : h;
        }
      }
    }
  }
  // running maximum of magnitudes: of words, or of the halves of words
  __device__ __forceinline__ void max_into(unsigned& m) const {
#pragma unroll
    for (int j = 0; j < (int)(V * sizeof(T) / 4); ++j) {
      if constexpr (sizeof(T) == 4) m = max(m, w[j] & 0x7fffffffu);
      else m = max_two(m, w[j]);
    }
  }
  // z: the codes' place
  __device__ __forceinline__ void store(signed char* z, int left, const TokenFactor& f) const {
    unsigned o[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      float v[4];
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = __uint_as_float(w[4 * j + q]);
      } else {
        unpack_two<T>(w[2 * j], v[0], v[1]);
        unpack_two<T>(w[2 * j + 1], v[2], v[3]);
      }
      o[j] = f.finite ? codes_4(v, f) : 0u;
    }
    if (kVec && V <= left) {
      if constexpr (V == 8) *reinterpret_cast<uint2*>(z) = make_uint2(o[0], o[1]);
      else *reinterpret_cast<unsigned*>(z) = o[0];
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j * kStep < left) z[j * kStep] = (signed char)(o[j / 4] >> (8 * (j & 3)));
    }
  }
};
template <typename T>
__device__ __forceinline__ unsigned as_fp32_bits(unsigned m) {  // of a maximum of halves
  if constexpr (sizeof(T) == 4) {
    return m;
  } else {
    float a, b;
    unpack_two<T>(max(m & 0xffffu, m >> 16), a, b);
    return __float_as_uint(a);
  }
}

// Teams of kTeam threads, a token each.  kTeam 32: eight tokens a block.
template <typename T, bool kVec, int kTeam>
__global__ void __launch_bounds__(kTeam == 32 ? 256 : kTeam, kTeam == 512 ? 2 : (kTeam == 128 ? 10 : 5)) quantize_tokens_kernel(const T* x, size_t tokens, size_t C, size_t ldx,
                                                                                    signed char* z, size_t ldz, float* scale) {
  using Part = Chunk<T, kVec, kTeam>;
  __shared__ unsigned part[kTeam / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = kTeam == 32 ? threadIdx.x & 31 : threadIdx.x;
  const size_t t = kTeam == 32 ? (size_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
  if (kTeam == 32 && t >= tokens) return;
  const T* row = x + t * ldx;
  signed char* out = z + t * ldz;
  constexpr int kTurn = kTeam * Part::V;
  const size_t c0 = (size_t)tid * (Part::kStep == 1 ? Part::V : 1);
  if (C <= c0) C = c0;
  const int left = (int)min(C - c0, (size_t)1 << 30);  // (more than is held)
  row += c0;
  out += c0;
  Part held[kHeld];
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (j * kTurn < left) held[j].load(row + j * kTurn, left - j * kTurn);
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (j * kTurn < left) held[j].max_into(m);
  for (size_t c = kHeld * kTurn; c < C - c0; c += kTurn) {
    Part again;
    again.load(row + c, (int)min(C - c0 - c, (size_t)1 << 30));
    again.max_into(m);
  }
  m = warp_max(as_fp32_bits<T>(m));
  if (kTeam > 32) {
    if ((tid & 31) == 0) part[tid >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTeam / 32; ++i) m = max(m, part[i]);
  }
  const TokenFactor f = token_factor(m);
  if (tid == 0) scale[t] = f.s;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (j * kTurn < left) held[j].store(out + j * kTurn, left - j * kTurn, f);
  for (size_t c = kHeld * kTurn; c < C - c0; c += kTurn) {
    Part again;
    again.load(row + c, (int)min(C - c0 - c, (size_t)1 << 30));
    again.store(out + c, (int)min(C - c0 - c, (size_t)1 << 30), f);
  }
}

// Sixteen codes a thread and turn where rows lie on the 16-byte grid, else four kTeam apart.
template <typename T, bool kVec, int kTeam>
__global__ void __launch_bounds__(256) dequantize_tokens_kernel(const signed char* z, size_t tokens, size_t C, size_t ldz,
                                                                const float* scale, T* r, size_t ldr) {
  constexpr int V = kVec ? 16 : 4;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const size_t t = (size_t)blockIdx.x * (256 / kTeam) + threadIdx.x / kTeam;
  if (t >= tokens) return;
  const float s = scale[t];
  const signed char* in = z + t * ldz;
  T* out = r + t * ldr;
  constexpr int kStep = kVec ? 1 : kTeam;
  for (size_t c = (size_t)(threadIdx.x % kTeam) * (kVec ? V : 1); c < C; c += (size_t)kTeam * V) {
    if (kVec && c + V <= C) {
      const uint4 w = *reinterpret_cast<const uint4*>(in + c);
      const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; j += sizeof(T) == 4 ? 1 : 2) {
        float v[4], x[4];
        values_4(u[j], s, v);
        if constexpr (sizeof(T) == 4) {
          reinterpret_cast<float4*>(out + c)[j] = make_float4(v[0], v[1], v[2], v[3]);
        } else {
          values_4(u[j + 1], s, x);
          reinterpret_cast<uint4*>(out + c)[j / 2] = make_uint4(pack_two<T>(v[0], v[1]), pack_two<T>(v[2], v[3]), pack_two<T>(x[0], x[1]), pack_two<T>(x[2], x[3]));
        }
      }
    } else if (kVec) {
      for (int j = 0; c + j < C; ++j) out[c + j] = from_f32<T>(__fmul_rn(s, (float)in[c + j]));
    } else {
      signed char v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = c + j * kStep < C ? in[c + j * kStep] : (signed char)0;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (c + j * kStep < C) out[c + j * kStep] = from_f32<T>(__fmul_rn(s, (float)v[j]));
    }
  }
}

template <typename... Params, typename... Args>
int launch_dependent(const char* name, void (*kernel)(Params...), size_t grid, int threads, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return check_cuda(cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...), name);
}

constexpr size_t kMostTokens = 0x7fffffff;  // of a launch

template <typename T, bool kVec>
int quantize_as(const T* x, size_t tokens, size_t C, size_t ldx, signed char* z, size_t ldz, float* scale, cudaStream_t s) {
  constexpr int V = Chunk<T, kVec, 32>::V;
  const size_t chunks = (C + V - 1) / V;
  // chunks a thread: about four, one where that leaves fewer than two blocks an SM
  const size_t want = tokens < (size_t)2 * sm_count() ? chunks : (chunks + 3) / 4;
  for (size_t t0 = 0; t0 < tokens; t0 += kMostTokens) {
    const size_t n = tokens - t0 < kMostTokens ? tokens - t0 : kMostTokens;
    const T* xt = x + t0 * ldx;
    signed char* zt = z + t0 * ldz;
    int rc;
    if (want <= 32) rc = launch_dependent("quantize_tokens_kernel", quantize_tokens_kernel<T, kVec, 32>, (n + 7) / 8, 256, s, xt, n, C, ldx, zt, ldz, scale + t0);
    else if (want <= 192) rc = launch_dependent("quantize_tokens_kernel", quantize_tokens_kernel<T, kVec, 128>, n, 128, s, xt, n, C, ldx, zt, ldz, scale + t0);
    else if (want <= 320) rc = launch_dependent("quantize_tokens_kernel", quantize_tokens_kernel<T, kVec, 256>, n, 256, s, xt, n, C, ldx, zt, ldz, scale + t0);
    else rc = launch_dependent("quantize_tokens_kernel", quantize_tokens_kernel<T, kVec, 512>, n, 512, s, xt, n, C, ldx, zt, ldz, scale + t0);
    if (rc != Q8_OK) return rc;
  }
  return Q8_OK;
}
template <typename T>
int quantize_any(const void* x, size_t tokens, size_t C, size_t ldx, signed char* z, size_t ldz, float* scale, cudaStream_t s) {
  const T* p = static_cast<const T*>(x);
  constexpr size_t V = Chunk<T, true, 32>::V;
  if (aligned16(x) && ldx % V == 0 && aligned_to(z, V) && ldz % V == 0) return quantize_as<T, true>(p, tokens, C, ldx, z, ldz, scale, s);
  return quantize_as<T, false>(p, tokens, C, ldx, z, ldz, scale, s);
}

template <typename T, bool kVec>
int dequantize_as(const signed char* z, size_t tokens, size_t C, size_t ldz, const float* scale, T* r, size_t ldr, cudaStream_t s) {
  const size_t chunks = (C + (kVec ? 15 : 3)) / (kVec ? 16 : 4);
  for (size_t t0 = 0; t0 < tokens; t0 += kMostTokens) {
    const size_t n = tokens - t0 < kMostTokens ? tokens - t0 : kMostTokens;
    const signed char* zt = z + t0 * ldz;
    T* rt = r + t0 * ldr;
    const int rc = chunks <= 96 ? launch_dependent("dequantize_tokens_kernel", dequantize_tokens_kernel<T, kVec, 32>, (n + 7) / 8, 256, s, zt, n, C, ldz, scale + t0, rt, ldr)
                                : launch_dependent("dequantize_tokens_kernel", dequantize_tokens_kernel<T, kVec, 256>, n, 256, s, zt, n, C, ldz, scale + t0, rt, ldr);
    if (rc != Q8_OK) return rc;
  }
  return Q8_OK;
}
template <typename T>
int dequantize_any(const signed char* z, size_t tokens, size_t C, size_t ldz, const float* scale, void* r, size_t ldr, cudaStream_t s) {
  T* p = static_cast<T*>(r);
  if (aligned16(z) && ldz % 16 == 0 && aligned16(r) && ldr * sizeof(T) % 16 == 0) return dequantize_as<T, true>(z, tokens, C, ldz, scale, p, ldr, s);
  return dequantize_as<T, false>(z, tokens, C, ldz, scale, p, ldr, s);
}

int check_tokens(const char* fn, const void* x, int type, size_t tokens, size_t C, size_t ldx, const void* z, size_t ldz, const float* scale) {
  if (!float_type(type)) return fail(Q8_ERR_INVALID_ARG, "%s: the type must be Q8_F32, Q8_F16 or Q8_BF16", fn);
  if (C == 0 || ldx < C || ldz < C) return fail(Q8_ERR_INVALID_ARG, "%s: C must be positive and no pitch below it", fn);
  if (tokens && (!x || !z || !scale)) return fail(Q8_ERR_INVALID_ARG, "%s: null pointer", fn);
  if (tokens > SIZE_MAX / 8 / (ldx > ldz ? ldx : ldz)) return fail(Q8_ERR_INVALID_ARG, "%s: tensor too large", fn);
  if (!aligned_to(x, type_bytes(type)) || !aligned_to(scale, 4)) return fail(Q8_ERR_ALIGNMENT, "%s: a pointer is not aligned to its element", fn);
  return Q8_OK;
}

}  // namespace

int launch_quantize_tokens(const void* x, int x_type, size_t tokens, size_t C, size_t ldx, int8_t* z, size_t ldz, float* scale, cudaStream_t s) {
  if (x_type == Q8_F32) return quantize_any<float>(x, tokens, C, ldx, z, ldz, scale, s);
  if (x_type == Q8_F16) return quantize_any<__half>(x, tokens, C, ldx, z, ldz, scale, s);
  return quantize_any<__nv_bfloat16>(x, tokens, C, ldx, z, ldz, scale, s);
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
  cudaStream_t s = as_stream(stream);
  if (r_type == Q8_F32) return dequantize_any<float>(z, tokens, C, ldz, d_scale, r, ldr, s);
  if (r_type == Q8_F16) return dequantize_any<__half>(z, tokens, C, ldz, d_scale, r, ldr, s);
  return dequantize_any<__nv_bfloat16>(z, tokens, C, ldz, d_scale, r, ldr, s);
}

}  // extern "C"
