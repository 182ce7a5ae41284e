// Mixture-of-experts layer for a few tokens: router, choice of experts, gated layers with 8-bit weights, weighted sum.
//
// Few tokens read each chosen expert's weights once and do little else: the layer is bound by the bytes of the weights, and
// everything between two streams of them is latency.  Two kernels:
//
//   moe_route_kernel    logits in 64 bits, a warp per (token, expert); the tokens as integer digits, a block per token;
//   moe_experts_kernel  all the rest.  Every block finds the chosen experts itself.  Then blocks draw work by tickets: first
//                       items of eight inner units (their eight gate and eight up rows are the sixteen rows of an
//                       instruction), then items of sixteen output channels over all chosen experts.
//
// A value of a token is held as a 24-bit integer relative to the row's largest, in three digits to the base 256 of -128 ..
// 127: the digits are three more "tokens" of an 8-bit product, which the eight columns of mma.sync.m16n8k32 have to spare
// (T tokens fill 3 T of 8 ceil(3T/8)).  Weights enter the tensor cores as the bytes they are, no conversion; all sums are
// exact integers, so neither the split of a reduction over warps nor the order of their additions changes a bit.
//
// What phase two reads of phase one: the block that completes an expert's last item turns the expert's inner activations
// into digits and raises its flag.  A block waits for the flags only with its first down weights already on their way.
// Blocks that wait hold a ticket of phase two, so that all items of phase one are in the hands of running blocks: progress
// needs no co-residency.  Waits are bounded all the same.
#include <atomic>
#include <type_traits>

#include "q8_token_common.cuh"

namespace q8 {
namespace {

constexpr int kMoeGroup = 16;    // tokens of a pass
constexpr int kMoeWarps = 16, kMoeThreads = 32 * kMoeWarps;
constexpr int kMaxTopK = 32;      // a lane each
constexpr int kMaxExperts = 1024; // a bit of a lane's word each
constexpr int kAccPitch = 20;    // ints between two columns of accumulators: lanes of a warp meet no bank twice
constexpr float kDigitMax = 8355711.0f;  // 127 (256^2 + 256 + 1)
constexpr unsigned kTimeoutMoe = 32u;
constexpr unsigned long long kMoeWaitNs = 2000000000ull;

struct MoeParams {
  int T, C, I, E, k, renormalize, x_type;
  long long ldx, ldy;
  const void* x;
  const float* router;
  const signed char* wgu;
  const float* sgu;
  const signed char* wd;
  const float* sd;
  void* y;
  int* ids;
  float* probs;
  // workspace
  double* logits;        // [T][E]
  float* x_factor;       // [T]
  float* h_factor;       // [T k]
  unsigned* sync;        // two tickets, then per chosen expert the finished items and the flag
  signed char* xd;       // digits of the tokens [T][3][x_pitch]
  signed char* hd;       // digits of the inner activations [T k][3][h_pitch]
  float* h;              // inner activations [T k][I]
  int x_pitch, h_pitch;  // multiples of 128
  int unit_blocks, tiles;
  int x_vec, r_vec;
  unsigned* status;
};

__device__ __forceinline__ float load_x(const MoeParams& p, int t, int c) {
  const long long o = (long long)t * p.ldx + c;
  if (p.x_type == Q8_F32) return static_cast<const float*>(p.x)[o];
  if (p.x_type == Q8_F16) return __half2float(static_cast<const __half*>(p.x)[o]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(p.x)[o]);
}
// Four values from c on, c a multiple of four and row and pitch aligned accordingly.
__device__ __forceinline__ float4 load_x4(const MoeParams& p, int t, int c) {
  const long long o = (long long)t * p.ldx + c;
  if (p.x_type == Q8_F32) return *reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + o);
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const unsigned short*>(p.x) + o);
  if (p.x_type == Q8_F16) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&w.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
    return make_float4(a.x, a.y, b.x, b.y);
  }
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}

// Factor of a row's digits and its reciprocal.  Maxima below 2^-104 take a power of two, whose reciprocal is finite; a row
// with a NaN or an infinity has factor NaN and digits zero.
struct DigitScale { float factor, inverse; };
__device__ __forceinline__ DigitScale digit_scale(unsigned max_bits) {
  DigitScale d;
  if (max_bits >= 0x7f800000u) { d.factor = __uint_as_float(0x7fc00000u); d.inverse = 0.0f; return d; }
  const float m = __uint_as_float(max_bits);
  if (m < 0x1p-104f) { d.factor = 0x1p-126f; d.inverse = 0x1p126f; return d; }
  d.factor = __fdiv_rn(m, kDigitMax);
  d.inverse = __fdiv_rn(kDigitMax, m);
  return d;
}
// Digits of v, most significant first.  |code| <= 8355711, so each digit fits eight bits.
__device__ __forceinline__ void digits_of(float v, const DigitScale& s, int& a, int& b, int& c) {
  const float q = fminf(fmaxf(__fmul_rn(v, s.inverse), -kDigitMax), kDigitMax);
  const int code = s.inverse == 0.0f ? 0 : __float2int_rn(q);
  c = (int)(signed char)code;
  const int r = (code - c) >> 8;
  b = (int)(signed char)r;
  a = (r - b) >> 8;
}
// Four values as one word of each digit.
__device__ __forceinline__ void digits_4(const float4 v, const DigitScale& s, unsigned& a, unsigned& b, unsigned& c) {
  int d[4][3];
  digits_of(v.x, s, d[0][0], d[0][1], d[0][2]);
  digits_of(v.y, s, d[1][0], d[1][1], d[1][2]);
  digits_of(v.z, s, d[2][0], d[2][1], d[2][2]);
  digits_of(v.w, s, d[3][0], d[3][1], d[3][2]);
  unsigned w[3];
#pragma unroll
  for (int k = 0; k < 3; ++k)
    w[k] = (unsigned)(d[0][k] & 255) | (unsigned)(d[1][k] & 255) << 8 | (unsigned)(d[2][k] & 255) << 16 | (unsigned)(d[3][k] & 255) << 24;
  a = w[0]; b = w[1]; c = w[2];
}
// The sum that three digits' accumulators stand for, rounded once.
__device__ __forceinline__ float digits_sum(int a, int b, int c) {
  return __ll2float_rn(((long long)a << 16) + ((long long)b << 8) + (long long)c);
}

// ------------------------------------------------------------------------------------------ router
__global__ void __launch_bounds__(256) moe_route_kernel(const __grid_constant__ MoeParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if ((int)blockIdx.x < p.T) {  // digits of a token
    const int t = blockIdx.x;
    if (t == 0) for (int i = threadIdx.x; i < 2 + 2 * min(p.E, p.T * p.k); i += 256) p.sync[i] = 0u;
    __shared__ unsigned part[8];
    unsigned m = 0;
    if (p.x_vec) {
      for (int c = 4 * threadIdx.x; c < p.C; c += 1024) {
        const float4 v = load_x4(p, t, c);
        m = max(m, max(max(abs_word(v.x), abs_word(v.y)), max(abs_word(v.z), abs_word(v.w))));
      }
    } else {
      for (int c = threadIdx.x; c < p.C; c += 256) m = max(m, abs_word(load_x(p, t, c)));
    }
    m = warp_max(m);
    if (lane == 0) part[warp] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, part[i]);
    const DigitScale s = digit_scale(m);
    if (threadIdx.x == 0) p.x_factor[t] = s.factor;
    signed char* out = p.xd + (size_t)t * 3 * p.x_pitch;
    for (int c = 4 * threadIdx.x; c < p.x_pitch; c += 1024) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p.x_vec) {
        if (c < p.C) v = load_x4(p, t, c);
      } else {
        if (c < p.C) v.x = load_x(p, t, c);
        if (c + 1 < p.C) v.y = load_x(p, t, c + 1);
        if (c + 2 < p.C) v.z = load_x(p, t, c + 2);
        if (c + 3 < p.C) v.w = load_x(p, t, c + 3);
      }
      unsigned a, b, d;
      digits_4(v, s, a, b, d);
      *reinterpret_cast<unsigned*>(out + c) = a;
      *reinterpret_cast<unsigned*>(out + p.x_pitch + c) = b;
      *reinterpret_cast<unsigned*>(out + 2 * (size_t)p.x_pitch + c) = d;
    }
    return;
  }
  const int pair = ((int)blockIdx.x - p.T) * 8 + warp;
  if (pair >= p.T * p.E) return;
  const int e = pair / p.T, t = pair - e * p.T;
  const float* r = p.router + (size_t)e * p.C;
  double s0 = 0.0, s1 = 0.0;
  if (p.x_vec && p.r_vec) {
#pragma unroll 4
    for (int c = 4 * lane; c < p.C; c += 128) {
      const float4 v = load_x4(p, t, c), w = __ldg(reinterpret_cast<const float4*>(r + c));
      s0 = __fma_rn((double)v.x, (double)w.x, s0);
      s1 = __fma_rn((double)v.y, (double)w.y, s1);
      s0 = __fma_rn((double)v.z, (double)w.z, s0);
      s1 = __fma_rn((double)v.w, (double)w.w, s1);
    }
  } else {
    for (int c = lane; c < p.C; c += 32) s0 = __fma_rn((double)load_x(p, t, c), (double)r[c], s0);
  }
  s0 += s1;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
  if (lane == 0) p.logits[(size_t)t * p.E + e] = s0;
}

// ------------------------------------------------------------------------------------------ experts
// A logit as an integer of the same order; a NaN below everything.
__device__ __forceinline__ unsigned long long order_key(double v) {
  if (isnan(v)) return 0ull;
  const long long b = __double_as_longlong(v == 0.0 ? 0.0 : v);
  return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}

// What a block knows of the choice of experts; rows: (token, chosen expert) pairs by expert, then token.
struct MoeChoice {
  int* expert;          // [rows] experts some token has chosen, ascending
  unsigned* tokens;     // [rows] ... their tokens as bits
  int* first;           // [rows] ... their first row
  float* prob;          // [rows] by row
  int* row_of;          // [T][k] rows of a token, ascending
  int* row_expert;      // [rows]
};

__device__ __forceinline__ int load_acquire(const unsigned* p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return (int)v;
}
__device__ __forceinline__ void store_release(unsigned* p, unsigned v) {
  asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}

// Whether `*flag` was raised in time.  All lanes of a warp call it.
__device__ __noinline__ bool wait_raised(const unsigned* flag, volatile int* gave_up, unsigned* status) {
  unsigned long long t0 = 0;
  for (unsigned spins = 1;; ++spins) {
    if (__all_sync(0xffffffffu, load_acquire(flag) != 0)) return true;
    if ((spins & 255u) == 0) {
      unsigned long long now;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (t0 == 0) t0 = now;
      int over = *gave_up;
      if (now - t0 > kMoeWaitNs) over = 1;
      if (__any_sync(0xffffffffu, over)) {
        if ((threadIdx.x & 31) == 0) { *gave_up = 1; atomicOr(status, kTimeoutMoe); }
        return false;
      }
    }
  }
}

// Sixteen bytes pos .. of a weight row, for the row's alignment kGrid (16, 8 or 1 bytes), zero from `len` on.  Rows off the
// grid are read in aligned words, each of which holds a byte of the row.
template <int kGrid>
__device__ __forceinline__ uint4 load_weights(const signed char* row, int pos, int len) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (kGrid == 16) {
    if (pos < len)
      asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + pos));
  } else if (kGrid == 8) {
    if (pos < len) { const uint2 a = __ldg(reinterpret_cast<const uint2*>(row + pos)); v.x = a.x; v.y = a.y; }
    if (pos + 8 < len) { const uint2 a = __ldg(reinterpret_cast<const uint2*>(row + pos + 8)); v.z = a.x; v.w = a.y; }
  } else {
    const unsigned long long at = (unsigned long long)(row + pos);
    const unsigned* w = reinterpret_cast<const unsigned*>(at & ~3ull);
    const int m = (int)(at & 3ull);
    unsigned u[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) u[k] = pos + 4 * k - m < len && (k < 4 || m > 0) ? __ldg(w + k) : 0u;
    v.x = __funnelshift_r(u[0], u[1], 8 * m);
    v.y = __funnelshift_r(u[1], u[2], 8 * m);
    v.z = __funnelshift_r(u[2], u[3], 8 * m);
    v.w = __funnelshift_r(u[3], u[4], 8 * m);
  }
  return v;
}

// Columns of the digits of an expert's tokens for this lane: byte offsets of the rows it reads.
template <int NT>
__device__ __forceinline__ void column_offsets(unsigned tokens, int count, int first_row, int pitch, bool by_row, int lane, unsigned (&off)[NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int col = 8 * t + (lane >> 2), r = min(col / 3, count - 1), d = col - col / 3 * 3;
    const int row = by_row ? first_row + r : (int)__fns(tokens, 0, r + 1);
    off[t] = (unsigned)(row * 3 + d) * (unsigned)pitch + 16u * (lane & 3);
  }
}

// Partial products of 16 weight rows (this lane's are wa and wb) with 8 NT columns over the steps [s0, s1) of 64 bytes,
// added to acc[column][16] in shared memory.  `wait`: called once, with the first weights on their way.
template <int NT, int kGrid, typename Wait>
__device__ __forceinline__ void stream_rows(const signed char* wa, const signed char* wb, int len, const signed char* cols, const unsigned (&off)[NT],
                                            int s0, int s1, int columns, int* acc, int lane, Wait wait) {
  constexpr int U = NT <= 2 ? 4 : 2;
  const int i = lane & 3, g = lane >> 2;
  int d[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t) d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0;
  uint4 a[U], b[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int pos = (s0 + u) * 64 + 16 * i, end = s0 + u < s1 ? len : 0;
    a[u] = load_weights<kGrid>(wa, pos, end);
    b[u] = load_weights<kGrid>(wb, pos, end);
  }
  if (!wait()) return;
  for (int s = s0; s < s1; s += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u < s1) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint4 z = *reinterpret_cast<const uint4*>(cols + off[t] + (size_t)(s + u) * 64);
          mma_16x8x32(d[t], a[u].x, b[u].x, a[u].y, b[u].y, z.x, z.y);
          mma_16x8x32(d[t], a[u].z, b[u].z, a[u].w, b[u].w, z.z, z.w);
        }
      }
      const int n = s + u + U, pos = n * 64 + 16 * i, end = n < s1 ? len : 0;
      a[u] = load_weights<kGrid>(wa, pos, end);
      b[u] = load_weights<kGrid>(wb, pos, end);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = 8 * t + 2 * i + (j & 1);
      if (col < columns) atomicAdd(acc + col * kAccPitch + g + 8 * (j >> 1), d[t][j]);
    }
}

// The digits of one row of inner activations, by a warp.
__device__ __forceinline__ void make_digits(const MoeParams& p, int row, int lane) {
  const float* h = p.h + (size_t)row * p.I;
  unsigned m = 0;
  for (int i = lane; i < p.I; i += 32) m = max(m, abs_word(__ldcg(h + i)));
  m = warp_max(m);
  const DigitScale s = digit_scale(m);
  if (lane == 0) p.h_factor[row] = s.factor;
  signed char* out = p.hd + (size_t)row * 3 * p.h_pitch;
  for (int i = 4 * lane; i < p.h_pitch; i += 128) {
    float4 v;
    v.x = i < p.I ? __ldcg(h + i) : 0.0f;
    v.y = i + 1 < p.I ? __ldcg(h + i + 1) : 0.0f;
    v.z = i + 2 < p.I ? __ldcg(h + i + 2) : 0.0f;
    v.w = i + 3 < p.I ? __ldcg(h + i + 3) : 0.0f;
    unsigned a, b, c;
    digits_4(v, s, a, b, c);
    *reinterpret_cast<unsigned*>(out + i) = a;
    *reinterpret_cast<unsigned*>(out + p.h_pitch + i) = b;
    *reinterpret_cast<unsigned*>(out + 2 * (size_t)p.h_pitch + i) = c;
  }
}

// Shared memory of a block, in bytes: lists of rows, masks by expert, accumulators of either phase.
struct MoeShared {
  int rows, acc_ints, chosen, total;
  __host__ __device__ MoeShared(int T, int k, int E) {
    rows = T * k;
    const int one = kMoeWarps * 3 * T * kAccPitch, two = 3 * rows * kAccPitch;  // every warp an item; every row
    acc_ints = one > two ? one : two;
    chosen = rows < E ? rows : E;
    total = 4 * (acc_ints + 6 * rows + 16 * rows + 2 * E) + 64;
  }
};

template <int kGridC, int kGridI>
__global__ void __launch_bounds__(kMoeThreads, 1) moe_experts_kernel(const __grid_constant__ MoeParams p, const int kw) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int s_active, s_ticket[2], s_last[kMoeWarps], gave_up;
  const MoeShared lay(p.T, p.k, p.E);
  int* const acc = reinterpret_cast<int*>(smem);
  float* const sums = reinterpret_cast<float*>(acc + lay.acc_ints);  // [rows][16]
  MoeChoice ch;
  ch.expert = reinterpret_cast<int*>(sums + 16 * lay.rows);
  ch.tokens = reinterpret_cast<unsigned*>(ch.expert + lay.rows);
  ch.first = reinterpret_cast<int*>(ch.tokens + lay.rows);
  ch.prob = reinterpret_cast<float*>(ch.first + lay.rows);
  ch.row_of = reinterpret_cast<int*>(ch.prob + lay.rows);
  ch.row_expert = ch.row_of + lay.rows;
  unsigned* const mask = reinterpret_cast<unsigned*>(ch.row_expert + lay.rows);  // [E] tokens that chose an expert
  int* const index = reinterpret_cast<int*>(mask + p.E);                          // [E] its place among the chosen
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int e = tid; e < p.E; e += kMoeThreads) mask[e] = 0u;
  if (tid == 0) gave_up = 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  // ---- choice: a warp per token
  int mine = -1;        // lane j: the j-th chosen expert
  float weight = 0.0f;  // ... its probability
  if (warp < p.T) {
    const double* l = p.logits + (size_t)warp * p.E;
    double best0 = 0.0, v_mine = 0.0;
    unsigned long long taken = 0ull;  // bit q: expert lane + 32 q (up to 1024 experts: 32 bits)
    for (int j = 0; j < p.k; ++j) {
      unsigned long long key = 0ull;
      int at = 0x7fffffff;
      for (int q = 0, e = lane; e < p.E; ++q, e += 32) {
        if (taken >> q & 1ull) continue;
        const unsigned long long o = order_key(__ldcg(l + e));
        if (at == 0x7fffffff || o > key) { key = o; at = e; }
      }
      // among lanes that have a candidate, the largest key, then the lowest expert
      const unsigned have = at != 0x7fffffff;
      const unsigned hi = have ? (unsigned)(key >> 32) : 0u;
      const unsigned top_hi = __reduce_max_sync(0xffffffffu, hi);
      const bool in = have && hi == top_hi;
      const unsigned top_lo = __reduce_max_sync(0xffffffffu, in ? (unsigned)key : 0u);
      const int e = (int)__reduce_min_sync(0xffffffffu, in && (unsigned)key == top_lo ? (unsigned)at : 0x7fffffffu);
      if ((e & 31) == lane) taken |= 1ull << (e >> 5);
      const double v = __ldcg(l + e);
      if (j == 0) best0 = v;
      if (lane == j) { mine = e; v_mine = v; }
    }
    float total = 0.0f;
    const float ex = lane < p.k ? expf((float)(v_mine - best0)) : 0.0f;
    if (p.renormalize) total = ex;
    else for (int e = lane; e < p.E; e += 32) total += expf((float)(__ldcg(l + e) - best0));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    weight = __fdiv_rn(ex, total);
    if (lane < p.k) {
      atomicOr(&mask[mine], 1u << warp);
      if (blockIdx.x == 0) {
        if (p.ids) p.ids[warp * p.k + lane] = mine;
        if (p.probs) p.probs[warp * p.k + lane] = weight;
      }
    }
  }
  __syncthreads();
  if (warp == 0) {  // chosen experts in order, their first rows
    int n = 0, rows = 0;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
      const unsigned m = e0 + lane < p.E ? mask[e0 + lane] : 0u;
      const unsigned some = __ballot_sync(0xffffffffu, m != 0u);
      int before = __popc(m);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int u = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += u; }
      if (m) {
        const int at = n + __popc(some & ((1u << lane) - 1u));
        ch.expert[at] = e0 + lane; ch.tokens[at] = m; ch.first[at] = rows + before - __popc(m);
        index[e0 + lane] = at;
      }
      n += __popc(some);
      rows += __shfl_sync(0xffffffffu, before, 31);
    }
    if (lane == 0) s_active = n;
  }
  if (tid == 32) s_ticket[0] = (int)atomicAdd(&p.sync[0], 1u);
  __syncthreads();
  if (warp < p.T && lane < p.k) {
    const int at = index[mine], row = ch.first[at] + __popc(ch.tokens[at] & ((1u << warp) - 1u));
    int place = 0;
    for (int j = 0; j < p.k; ++j) place += __shfl_sync((p.k == 32 ? 0xffffffffu : (1u << p.k) - 1u), mine, j) < mine;
    ch.prob[row] = weight;
    ch.row_of[warp * p.k + place] = row;
    ch.row_expert[row] = mine;
  }
  const int active = s_active;
  unsigned* const done = p.sync + 2;
  unsigned* const ready = done + lay.chosen;

  // ---- phase one: kw warps an item
  const int groups = kMoeWarps / kw, group = warp / kw, part = warp - group * kw;
  const int items = active * p.unit_blocks, bundles = (items + groups - 1) / groups;
  const int steps = (p.C + 63) >> 6, per = (steps + kw - 1) / kw;
  int* const my_acc = acc + group * 3 * p.T * kAccPitch;
  int parity = 0;
  for (;;) {
    const int bundle = s_ticket[parity];
    if (bundle >= bundles) break;
    const int item = bundle * groups + group;
    const bool live = item < items;
    const int a = live ? item / p.unit_blocks : 0, i0 = (item - a * p.unit_blocks) * 8;
    const int e = ch.expert[a], count = __popc(ch.tokens[a]);
    for (int i = tid; i < groups * 3 * p.T * kAccPitch; i += kMoeThreads) acc[i] = 0;
    __syncthreads();
    unsigned next = 0;
    if (tid == 0) next = atomicAdd(&p.sync[0], 1u);
    if (live) {
      const int s0 = part * per, s1 = min(steps, s0 + per);
      const int unit = min(i0 + (lane >> 2), p.I - 1);
      const signed char* wa = p.wgu + ((size_t)e * 2 * p.I + unit) * p.C;
      const signed char* wb = wa + (size_t)p.I * p.C;
      auto go = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        unsigned off[NT];
        column_offsets<NT>(ch.tokens[a], count, 0, p.x_pitch, false, lane, off);
        stream_rows<NT, kGridC>(wa, wb, p.C, p.xd, off, s0, s1, 3 * count, my_acc, lane, [] { return true; });
      };
      if (s0 < s1) {
        if (count <= 2) go(std::integral_constant<int, 1>{});
        else if (count <= 5) go(std::integral_constant<int, 2>{});
        else go(std::integral_constant<int, 6>{});
      }
    }
    __syncthreads();
    if (live) {
      for (int o = part * 32 + lane; o < 8 * count; o += 32 * kw) {
        const int r = o >> 3, u = o & 7, i = i0 + u;
        if (i >= p.I) continue;
        const int* q = my_acc + 3 * r * kAccPitch + u;
        const float f = p.x_factor[__fns(ch.tokens[a], 0, r + 1)];
        const size_t at = (size_t)e * 2 * p.I + i;
        const float g = __fmul_rn(__fmul_rn(digits_sum(q[0], q[kAccPitch], q[2 * kAccPitch]), f), p.sgu[at]);
        const float v = __fmul_rn(__fmul_rn(digits_sum(q[8], q[kAccPitch + 8], q[2 * kAccPitch + 8]), f), p.sgu[at + p.I]);
        p.h[(size_t)(ch.first[a] + r) * p.I + i] = __fmul_rn(__fdiv_rn(g, __fadd_rn(1.0f, expf(-g))), v);
      }
    }
    if (tid == 0) s_ticket[parity ^ 1] = (int)next;
    __syncthreads();
    if (part == 0 && lane == 0) {
      int last = 0;
      if (live) {
        __threadfence();
        last = atomicAdd(&done[a], 1u) == (unsigned)p.unit_blocks - 1u;
        __threadfence();
      }
      s_last[group] = last;
    }
    __syncthreads();
    for (int q = 0; q < groups; ++q) {
      if (!s_last[q]) continue;  // the same for all threads
      const int qa = (bundle * groups + q) / p.unit_blocks;
      if (warp < __popc(ch.tokens[qa])) make_digits(p, ch.first[qa] + warp, lane);
      __syncthreads();
      if (tid == 0) { __threadfence(); store_release(&ready[qa], 1u); }
    }
    parity ^= 1;
  }

  // ---- phase two: sixteen output channels, all chosen experts
  const int hsteps = (p.I + 63) >> 6;
  int kd = 1;  // warps an expert
  while (2 * kd * active <= kMoeWarps && 4 * kd <= hsteps) kd *= 2;
  const int hper = (hsteps + kd - 1) / kd, tasks = active * kd, rows = p.T * p.k;
  __syncthreads();
  for (;;) {
    if (tid == 0) s_ticket[0] = (int)atomicAdd(&p.sync[1], 1u);
    for (int i = tid; i < 3 * rows * kAccPitch; i += kMoeThreads) acc[i] = 0;
    __syncthreads();
    const int tile = s_ticket[0];
    if (tile >= p.tiles) break;
    const int c0 = tile * 16;
    for (int task = warp; task < tasks; task += kMoeWarps) {
      const int a = task / kd, s0 = (task - a * kd) * hper, s1 = min(hsteps, s0 + hper);
      if (s0 >= s1) continue;
      const int e = ch.expert[a], count = __popc(ch.tokens[a]);
      const signed char* wa = p.wd + ((size_t)e * p.C + min(c0 + (lane >> 2), p.C - 1)) * p.I;
      const signed char* wb = p.wd + ((size_t)e * p.C + min(c0 + (lane >> 2) + 8, p.C - 1)) * p.I;
      auto go = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        unsigned off[NT];
        column_offsets<NT>(0u, count, ch.first[a], p.h_pitch, true, lane, off);
        stream_rows<NT, kGridI>(wa, wb, p.I, p.hd, off, s0, s1, 3 * count, acc + 3 * ch.first[a] * kAccPitch, lane,
                                [&] { return wait_raised(&ready[a], &gave_up, p.status); });
      };
      if (count <= 2) go(std::integral_constant<int, 1>{});
      else if (count <= 5) go(std::integral_constant<int, 2>{});
      else go(std::integral_constant<int, 6>{});
    }
    __syncthreads();
    for (int o = tid; o < 16 * rows; o += kMoeThreads) {
      const int r = o >> 4, c = o & 15;
      const int* q = acc + 3 * r * kAccPitch + c;
      const float s = p.sd[(size_t)ch.row_expert[r] * p.C + min(c0 + c, p.C - 1)];
      sums[o] = __fmul_rn(ch.prob[r], __fmul_rn(__fmul_rn(digits_sum(q[0], q[kAccPitch], q[2 * kAccPitch]), __ldcg(p.h_factor + r)), s));
    }
    __syncthreads();
    for (int o = tid; o < 16 * p.T; o += kMoeThreads) {
      const int t = o >> 4, c = o & 15;
      if (c0 + c >= p.C) continue;
      float y = 0.0f;
      for (int j = 0; j < p.k; ++j) y = __fadd_rn(y, sums[16 * ch.row_of[t * p.k + j] + c]);
      const long long at = (long long)t * p.ldy + c0 + c;
      if (p.x_type == Q8_F32) static_cast<float*>(p.y)[at] = y;
      else if (p.x_type == Q8_F16) static_cast<__half*>(p.y)[at] = __float2half_rn(y);
      else static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(y);
    }
    __syncthreads();
  }
}

int validate_moe(const q8_moe_desc* d) {
  if (!d) return fail(Q8_ERR_INVALID_ARG, "q8_moe: null descriptor");
  if (d->T < 0 || d->C <= 0 || d->I <= 0 || d->E <= 0) return fail(Q8_ERR_INVALID_ARG, "q8_moe: C, I and E must be positive, T non-negative");
  if (d->top_k <= 0 || d->top_k > d->E) return fail(Q8_ERR_INVALID_ARG, "q8_moe: top_k must be in 1 .. E");
  if (!float_type(d->x_type)) return fail(Q8_ERR_INVALID_ARG, "q8_moe: x_type must be Q8_F32, Q8_F16 or Q8_BF16");
  if ((d->renormalize != 0 && d->renormalize != 1) || d->reserved != 0) return fail(Q8_ERR_INVALID_ARG, "q8_moe: renormalize must be 0 or 1, reserved 0");
  const long long ldx = d->ldx == 0 ? d->C : d->ldx, ldy = d->ldy == 0 ? d->C : d->ldy, most = 1ll << 60;
  if (ldx < d->C || ldy < d->C) return fail(Q8_ERR_INVALID_ARG, "q8_moe: a pitch is below the row length");
  if (ldx > most / (d->T + 1ll) || ldy > most / (d->T + 1ll)) return fail(Q8_ERR_INVALID_ARG, "q8_moe: tensor too large");
  if (d->C > 131071 || d->I > 131071 || d->E > kMaxExperts || d->top_k > kMaxTopK)
    return fail(Q8_ERR_UNSUPPORTED, "q8_moe: limits are C, I <= 131071, E <= 1024, top_k <= 32");
  return Q8_OK;
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
int pitch128(int n) { return (n + 127) & ~127; }  // rows of digits end with their lines

// The workspace of up to kMoeGroup tokens; sets the pointers of `p` where there is one.  Returns its size.
size_t moe_space(const q8_moe_desc& d, char* ws, MoeParams* p) {
  const size_t T = d.T < kMoeGroup ? d.T : kMoeGroup, rows = T * d.top_k;
  size_t at = 0;
  auto take = [&](size_t bytes) { char* q = ws + at; at += up256(bytes); return q; };
  p->logits = reinterpret_cast<double*>(take(T * d.E * sizeof(double)));
  p->x_factor = reinterpret_cast<float*>(take(T * 4));
  p->h_factor = reinterpret_cast<float*>(take(rows * 4));
  p->sync = reinterpret_cast<unsigned*>(take((2 + 2 * rows) * 4));
  p->xd = reinterpret_cast<signed char*>(take(T * 3 * pitch128(d.C)));
  p->hd = reinterpret_cast<signed char*>(take(rows * 3 * pitch128(d.I)));
  p->h = reinterpret_cast<float*>(take(rows * d.I * 4));
  return at;
}

int row_grid(const void* w, int len) { return aligned16(w) && len % 16 == 0 ? 16 : (aligned_to(w, 8) && len % 8 == 0 ? 8 : 1); }

template <int kGridC, int kGridI>
int launch_experts(const MoeParams& p, int kw, cudaStream_t s) {
  const int smem = MoeShared(p.T, p.k, p.E).total;
  static std::atomic<bool> set[kMaxDevices];
  const int dev = current_device();
  if (dev < 0 || !set[dev].load(std::memory_order_relaxed)) {
    const int rc = check_cuda(cudaFuncSetAttribute(moe_experts_kernel<kGridC, kGridI>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024), "moe_experts_kernel");
    if (rc != Q8_OK) return rc;
    if (dev >= 0) set[dev].store(true, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(sm_count()));
  cfg.blockDim = dim3(kMoeThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return check_cuda(cudaLaunchKernelEx(&cfg, moe_experts_kernel<kGridC, kGridI>, p, kw), "moe_experts_kernel");
}

template <int kGridC>
int launch_experts(const MoeParams& p, int grid_i, int kw, cudaStream_t s) {
  if (grid_i == 16) return launch_experts<kGridC, 16>(p, kw, s);
  if (grid_i == 8) return launch_experts<kGridC, 8>(p, kw, s);
  return launch_experts<kGridC, 1>(p, kw, s);
}

int launch_route(const MoeParams& p, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(p.T + (p.T * p.E + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return check_cuda(cudaLaunchKernelEx(&cfg, moe_route_kernel, p), "moe_route_kernel");
}

}  // namespace
}  // namespace q8

using namespace q8;

extern "C" {

int q8_moe_workspace_bytes(const q8_moe_desc* d, size_t* bytes) {
  clear_error();
  const int rc = validate_moe(d);
  if (rc != Q8_OK) return rc;
  if (!bytes) return fail(Q8_ERR_INVALID_ARG, "q8_moe_workspace_bytes: null pointer");
  MoeParams p{};
  *bytes = d->T ? moe_space(*d, nullptr, &p) : 0;
  return Q8_OK;
}

int q8_moe(const q8_moe_desc* d, const void* x, const float* router, const int8_t* w_gate_up, const float* s_gate_up, const int8_t* w_down,
           const float* s_down, void* y, int32_t* ids, float* probs, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  int rc = validate_moe(d);
  if (rc != Q8_OK) return rc;
  if (!router || !w_gate_up || !s_gate_up || !w_down || !s_down || (d->T && (!x || !y))) return fail(Q8_ERR_INVALID_ARG, "q8_moe: null pointer");
  const size_t e = type_bytes(d->x_type);
  if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(router, 4) || !aligned_to(s_gate_up, 4) || !aligned_to(s_down, 4) ||
      !aligned_to(ids, 4) || !aligned_to(probs, 4))
    return fail(Q8_ERR_ALIGNMENT, "q8_moe: a pointer is not aligned to its element");
  if (!aligned_to(workspace, 256)) return fail(Q8_ERR_ALIGNMENT, "q8_moe: workspace not 256-byte aligned");
  if (d->T == 0) return Q8_OK;
  MoeParams p{};
  const size_t need = moe_space(*d, static_cast<char*>(workspace), &p);
  if (!workspace || workspace_bytes < need) return fail(Q8_ERR_WORKSPACE, "q8_moe: %zu bytes of workspace needed", need);
  p.C = d->C; p.I = d->I; p.E = d->E; p.k = d->top_k; p.renormalize = d->renormalize; p.x_type = d->x_type;
  p.ldx = d->ldx == 0 ? d->C : d->ldx;
  p.ldy = d->ldy == 0 ? d->C : d->ldy;
  p.router = router; p.wgu = w_gate_up; p.sgu = s_gate_up; p.wd = w_down; p.sd = s_down;
  p.x_pitch = pitch128(p.C); p.h_pitch = pitch128(p.I);
  p.unit_blocks = (p.I + 7) / 8; p.tiles = (p.C + 15) / 16;
  p.x_vec = aligned_to(x, 4 * e) && p.ldx % 4 == 0 && p.C % 4 == 0;
  p.r_vec = aligned16(router) && p.C % 4 == 0;
  p.status = status_word_device_ptr();
  if (!p.status) return fail(Q8_ERR_CUDA, "q8_moe: status word not available");
  cudaStream_t s = as_stream(stream);
  for (int t0 = 0; t0 < d->T; t0 += kMoeGroup) {
    p.T = d->T - t0 < kMoeGroup ? d->T - t0 : kMoeGroup;
    p.x = static_cast<const char*>(x) + (size_t)t0 * p.ldx * e;
    p.y = static_cast<char*>(y) + (size_t)t0 * p.ldy * e;
    p.ids = ids ? ids + (size_t)t0 * p.k : nullptr;
    p.probs = probs ? probs + (size_t)t0 * p.k : nullptr;
    if ((rc = launch_route(p, s)) != Q8_OK) return rc;
    const int kw = 2, gi = row_grid(w_down, p.I);
    switch (row_grid(w_gate_up, p.C)) {
      case 16: rc = launch_experts<16>(p, gi, kw, s); break;
      case 8: rc = launch_experts<8>(p, gi, kw, s); break;
      default: rc = launch_experts<1>(p, gi, kw, s); break;
    }
    if (rc != Q8_OK) return rc;
  }
  return Q8_OK;
}

}  // extern "C"
