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
  *bytes = 0;
  return Q8_OK;
}

int q8_linear(const q8_linear_desc* d, const void* x, const float* x_scale, const int8_t* w, const float* w_scale, const float* bias,
              void* y, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  LinearArgs a{};
  const int rc = validate_linear(d, &a);
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
  return launch_linear_rows(a);
}

}  // extern "C"
