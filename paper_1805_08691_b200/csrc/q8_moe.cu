// Mixture-of-experts layer for a few tokens: router, choice of experts, gated layers with 8-bit weights, weighted sum.
#include "q8_token_common.cuh"

namespace q8 {
namespace {

constexpr int kMoeGroup = 16;  // tokens of a pass

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
  int* w_ids;      // workspace: chosen experts [T][k]
  float* w_probs;  // ... their probabilities [T][k]
  float* h;        // ... inner activations [T][k][I]
};

__device__ __forceinline__ float load_x(const MoeParams& p, int t, int c) {
  const long long o = (long long)t * p.ldx + c;
  if (p.x_type == Q8_F32) return static_cast<const float*>(p.x)[o];
  if (p.x_type == Q8_F16) return __half2float(static_cast<const __half*>(p.x)[o]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(p.x)[o]);
}

// Whether logit a of expert i ranks before logit b of expert j.
__device__ __forceinline__ bool ranks_before(double a, int i, double b, int j) {
  const bool na = isnan(a), nb = isnan(b);
  if (na || nb) return na && nb ? i < j : nb;
  return a > b || (a == b && i < j);
}

__global__ void __launch_bounds__(256) moe_route_kernel(const __grid_constant__ MoeParams p) {
  extern __shared__ double logits[];
  const int t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int e = warp; e < p.E; e += 8) {
    double s = 0.0;
    for (int c = lane; c < p.C; c += 32) s += (double)load_x(p, t, c) * (double)p.router[(size_t)e * p.C + c];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) logits[e] = s;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  int chosen[32];
  for (int j = 0; j < p.k; ++j) {
    int best = -1;
    for (int e = 0; e < p.E; ++e) {
      bool taken = false;
      for (int q = 0; q < j; ++q) taken |= chosen[q] == e;
      if (!taken && (best < 0 || ranks_before(logits[e], e, logits[best], best))) best = e;
    }
    chosen[j] = best;
  }
  const double top = logits[chosen[0]];
  float total = 0.0f;
  if (p.renormalize) for (int j = 0; j < p.k; ++j) total += expf((float)(logits[chosen[j]] - top));
  else for (int e = 0; e < p.E; ++e) total += expf((float)(logits[e] - top));
  for (int j = 0; j < p.k; ++j) {
    const float w = __fdiv_rn(expf((float)(logits[chosen[j]] - top)), total);
    p.w_ids[t * p.k + j] = chosen[j];
    p.w_probs[t * p.k + j] = w;
    if (p.ids) p.ids[t * p.k + j] = chosen[j];
    if (p.probs) p.probs[t * p.k + j] = w;
  }
}

__device__ __forceinline__ float warp_sum(float s) {
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

__global__ void __launch_bounds__(256) moe_gate_up_kernel(const __grid_constant__ MoeParams p) {
  const int lane = threadIdx.x & 31, i = blockIdx.x * 8 + (threadIdx.x >> 5), slot = blockIdx.y;
  if (i >= p.I) return;
  const int t = slot / p.k, e = p.w_ids[slot];
  const signed char* wg = p.wgu + ((size_t)e * 2 * p.I + i) * p.C;
  const signed char* wu = wg + (size_t)p.I * p.C;
  float g = 0.0f, u = 0.0f;
  for (int c = lane; c < p.C; c += 32) {
    const float v = load_x(p, t, c);
    g = __fmaf_rn(v, (float)wg[c], g);
    u = __fmaf_rn(v, (float)wu[c], u);
  }
  g = warp_sum(g) * p.sgu[(size_t)e * 2 * p.I + i];
  u = warp_sum(u) * p.sgu[(size_t)e * 2 * p.I + p.I + i];
  if (lane == 0) p.h[(size_t)slot * p.I + i] = __fdiv_rn(g, 1.0f + expf(-g)) * u;
}

__global__ void __launch_bounds__(256) moe_down_kernel(const __grid_constant__ MoeParams p) {
  const int lane = threadIdx.x & 31, c = blockIdx.x * 8 + (threadIdx.x >> 5), t = blockIdx.y;
  if (c >= p.C) return;
  float y = 0.0f;
  for (int j = 0; j < p.k; ++j) {
    const int slot = t * p.k + j, e = p.w_ids[slot];
    const signed char* w = p.wd + ((size_t)e * p.C + c) * p.I;
    float s = 0.0f;
    for (int i = lane; i < p.I; i += 32) s = __fmaf_rn(p.h[(size_t)slot * p.I + i], (float)w[i], s);
    y += p.w_probs[slot] * (warp_sum(s) * p.sd[(size_t)e * p.C + c]);
  }
  if (lane != 0) return;
  const long long o = (long long)t * p.ldy + c;
  if (p.x_type == Q8_F32) static_cast<float*>(p.y)[o] = y;
  else if (p.x_type == Q8_F16) static_cast<__half*>(p.y)[o] = __float2half_rn(y);
  else static_cast<__nv_bfloat16*>(p.y)[o] = __float2bfloat16_rn(y);
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
  if (d->C > 131071 || d->I > 131071 || d->E > 1024 || d->top_k > 32)
    return fail(Q8_ERR_UNSUPPORTED, "q8_moe: limits are C, I <= 131071, E <= 1024, top_k <= 32");
  return Q8_OK;
}

struct MoeSpace { size_t ids, probs, h, bytes; };
MoeSpace moe_space(const q8_moe_desc& d) {
  const size_t slots = (size_t)(d.T < kMoeGroup ? d.T : kMoeGroup) * d.top_k;
  auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  MoeSpace s;
  s.ids = 0;
  s.probs = s.ids + up(slots * 4);
  s.h = s.probs + up(slots * 4);
  s.bytes = s.h + up(slots * d.I * 4);
  return s;
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
  *bytes = d->T ? moe_space(*d).bytes : 0;
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
  const MoeSpace sp = moe_space(*d);
  if (!workspace || workspace_bytes < sp.bytes) return fail(Q8_ERR_WORKSPACE, "q8_moe: %zu bytes of workspace needed", sp.bytes);
  MoeParams p{};
  p.C = d->C; p.I = d->I; p.E = d->E; p.k = d->top_k; p.renormalize = d->renormalize; p.x_type = d->x_type;
  p.ldx = d->ldx == 0 ? d->C : d->ldx;
  p.ldy = d->ldy == 0 ? d->C : d->ldy;
  p.router = router; p.wgu = w_gate_up; p.sgu = s_gate_up; p.wd = w_down; p.sd = s_down;
  char* ws = static_cast<char*>(workspace);
  p.w_ids = reinterpret_cast<int*>(ws + sp.ids);
  p.w_probs = reinterpret_cast<float*>(ws + sp.probs);
  p.h = reinterpret_cast<float*>(ws + sp.h);
  cudaStream_t s = as_stream(stream);
  for (int t0 = 0; t0 < d->T; t0 += kMoeGroup) {
    p.T = d->T - t0 < kMoeGroup ? d->T - t0 : kMoeGroup;
    p.x = static_cast<const char*>(x) + (size_t)t0 * p.ldx * e;
    p.y = static_cast<char*>(y) + (size_t)t0 * p.ldy * e;
    p.ids = ids ? ids + (size_t)t0 * p.k : nullptr;
    p.probs = probs ? probs + (size_t)t0 * p.k : nullptr;
    moe_route_kernel<<<p.T, 256, p.E * sizeof(double), s>>>(p);
    if ((rc = check_launch("moe_route_kernel")) != Q8_OK) return rc;
    moe_gate_up_kernel<<<dim3((p.I + 7) / 8, p.T * p.k), 256, 0, s>>>(p);
    if ((rc = check_launch("moe_gate_up_kernel")) != Q8_OK) return rc;
    moe_down_kernel<<<dim3((p.C + 7) / 8, p.T), 256, 0, s>>>(p);
    if ((rc = check_launch("moe_down_kernel")) != Q8_OK) return rc;
  }
  return Q8_OK;
}

}  // extern "C"
