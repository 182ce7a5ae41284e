// Entry point of the product with a factor per token and per output channel: checks and choice of the kernel.
#include "q8_linear.h"
#include "q8_token_common.cuh"

namespace q8 {
namespace {

int validate_linear(const q8_linear_desc* d, LinearArgs* a) {
  if (!d) return fail(Q8_ERR_INVALID_ARG, "q8_linear: null descriptor");
  if (d->M < 0 || d->C <= 0 || d->K <= 0) return fail(Q8_ERR_INVALID_ARG, "q8_linear: C and K must be positive, M non-negative");
  if (d->x_type != Q8_S8 && !float_type(d->x_type)) return fail(Q8_ERR_INVALID_ARG, "q8_linear: x_type must be Q8_S8, Q8_F32, Q8_F16 or Q8_BF16");
  if (!float_type(d->y_type)) return fail(Q8_ERR_INVALID_ARG, "q8_linear: y_type must be Q8_F32, Q8_F16 or Q8_BF16");
  // |z|, |w| <= 128: C products stay inside int32 below 2^31 / 2^14
  if (d->C > 131071) return fail(Q8_ERR_INVALID_ARG, "q8_linear: C > 131071 could overflow the int32 accumulator");
  if (d->reserved != 0) return fail(Q8_ERR_INVALID_ARG, "q8_linear: reserved must be 0");
  a->M = d->M; a->C = d->C; a->K = d->K;
  a->ldx = d->ldx == 0 ? d->C : d->ldx;
  a->ldw = d->ldw == 0 ? d->C : d->ldw;
  a->ldy = d->ldy == 0 ? d->K : d->ldy;
  if (a->ldx < d->C || a->ldw < d->C || a->ldy < d->K) return fail(Q8_ERR_INVALID_ARG, "q8_linear: a pitch is below the row length");
  const long long most = 1ll << 60;
  if (a->ldx > most / (d->M + 1) || a->ldw > most / d->K || a->ldy > most / (d->M + 1)) return fail(Q8_ERR_INVALID_ARG, "q8_linear: tensor too large");
  a->x_type = d->x_type; a->y_type = d->y_type;
  return Q8_OK;
}

// Rows of bytes onto the 16-byte grid: thread = 16 bytes.
__global__ void __launch_bounds__(256) regrid_kernel(const signed char* __restrict__ in, long long rows, int C, long long ld, signed char* __restrict__ out,
                                                     int pitch) {
  const int chunks = pitch >> 4;
  const long long n = rows * chunks;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long r = i / chunks;
    const int c = (int)(i - r * chunks) * 16;
    *reinterpret_cast<uint4*>(out + r * pitch + c) = load_16<false>(in + r * ld, c, C);
  }
}
int regrid(const int8_t* in, long long rows, int C, long long ld, int8_t* out, int pitch, cudaStream_t s) {
  const long long blocks = (rows * (pitch >> 4) + 255) / 256, most = (long long)sm_count() * 32;
  regrid_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, s>>>(in, rows, C, ld, out, pitch);
  return check_launch("regrid_kernel");
}

bool on_grid(const void* p, long long ld) { return aligned16(p) && ld % 16 == 0 && ld < (1ll << 40); }
bool few_tokens(const LinearArgs& a) { return linear_stream_fits(a); }
// Floating-point activations of so few tokens are quantized by every block of the streaming kernel.
constexpr int kStagedTokens = 4;
size_t up16(size_t v) { return (v + 15) & ~(size_t)15; }

// Parts of the workspace: codes and factors of x, weights on the grid; a part of zero bytes is not needed.
struct LinearSpace { size_t codes, factors, weights; size_t bytes() const { return codes + factors + weights; } };
LinearSpace linear_space(const LinearArgs& a, bool x_on_grid, bool w_on_grid) {
  LinearSpace s{0, 0, 0};
  const bool few = few_tokens(a);
  if (a.M == 0 || (few && (a.x_type == Q8_S8 || a.M <= kStagedTokens))) return s;
  if (a.x_type != Q8_S8) s.factors = up16((size_t)a.M * 4);
  if (a.x_type != Q8_S8 || !x_on_grid) s.codes = (size_t)a.M * up16(a.C);
  if (!w_on_grid && !few) s.weights = (size_t)a.K * up16(a.C);
  return s;
}

}  // namespace
}  // namespace q8

using namespace q8;

extern "C" {

int q8_linear_workspace_bytes(const q8_linear_desc* d, size_t* bytes) {
  clear_error();
  LinearArgs a{};
  const int rc = validate_linear(d, &a);
  if (rc != Q8_OK) return rc;
  if (!bytes) return fail(Q8_ERR_INVALID_ARG, "q8_linear_workspace_bytes: null pointer");
  *bytes = linear_space(a, on_grid(nullptr, a.ldx), on_grid(nullptr, a.ldw)).bytes();
  return Q8_OK;
}

int q8_linear(const q8_linear_desc* d, const void* x, const float* x_scale, const int8_t* w, const float* w_scale, const float* bias,
              void* y, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  LinearArgs a{};
  int rc = validate_linear(d, &a);
  if (rc != Q8_OK) return rc;
  if (!w || !w_scale || (a.M && (!x || !y))) return fail(Q8_ERR_INVALID_ARG, "q8_linear: null x, w, w_scale or y");
  if (a.M && (a.x_type == Q8_S8) != (x_scale != nullptr))
    return fail(Q8_ERR_INVALID_ARG, "q8_linear: x_scale belongs to codes, and floating-point activations have none");
  if (!aligned_to(x, type_bytes(a.x_type)) || !aligned_to(y, type_bytes(a.y_type)) || !aligned_to(x_scale, 4) || !aligned_to(w_scale, 4) || !aligned_to(bias, 4))
    return fail(Q8_ERR_ALIGNMENT, "q8_linear: a pointer is not aligned to its element");
  if (workspace && !aligned16(workspace)) return fail(Q8_ERR_ALIGNMENT, "q8_linear: workspace not 16-byte aligned");
  if (a.M == 0) return Q8_OK;
  a.x = x; a.x_scale = x_scale; a.w = w; a.w_scale = w_scale; a.bias = bias; a.y = y;
  a.stream = as_stream(stream);
  const LinearSpace sp = linear_space(a, on_grid(x, a.ldx), on_grid(w, a.ldw));
  const bool few = few_tokens(a);
  if (sp.bytes() > (workspace ? workspace_bytes : 0) || (few && sp.bytes() == 0)) return few ? launch_linear_stream(a) : launch_linear_rows(a);
  int8_t* const codes = static_cast<int8_t*>(workspace);
  float* const factors = reinterpret_cast<float*>(codes + sp.codes);
  const int pitch = (int)up16(a.C);
  if (a.x_type != Q8_S8) {
    rc = launch_quantize_tokens(x, a.x_type, (size_t)a.M, (size_t)a.C, (size_t)a.ldx, codes, (size_t)pitch, factors, a.stream);
    a.x_type = Q8_S8; a.x_scale = factors;
  } else if (sp.codes) {
    rc = regrid(static_cast<const int8_t*>(x), a.M, a.C, a.ldx, codes, pitch, a.stream);
  }
  if (rc != Q8_OK) return rc;
  if (sp.codes) { a.x = codes; a.ldx = pitch; }
  if (sp.weights) {
    int8_t* const weights = codes + sp.codes + sp.factors;
    rc = regrid(w, a.K, a.C, a.ldw, weights, pitch, a.stream);
    if (rc != Q8_OK) return rc;
    a.w = weights; a.ldw = pitch;
  }
  return few ? launch_linear_stream(a) : launch_linear_umma(a);
}

}  // extern "C"
