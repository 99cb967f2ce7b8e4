// C ABI of the token layers: short causal convolution, selective scan, norm.
// Stateless host side: every call checks its arguments, picks a kernel and
// enqueues it; a negative status means nothing ran.
#include <cmath>
#include <initializer_list>

#include "launch.hpp"
#include "token_check.hpp"

using namespace coinf;

namespace {

bool shortconv_ok(const co_shortconv_desc* d) {
  return d && d->batch > 0 && d->channels > 0 && d->kernel > 0 &&
         d->kernel <= CO_SHORTCONV_MAX_TAPS && dtype_ok(d->dtype) &&
         (d->act == CO_ACT_NONE || d->act == CO_ACT_RELU || d->act == CO_ACT_SILU) &&
         mul_to(mul_to(d->batch, d->channels, kMaxValues), d->kernel, kMaxValues) >= 0;
}

bool scan_ok(const co_scan_desc* d) {
  if (!d || d->batch <= 0 || d->heads <= 0 || d->head_dim <= 0 || d->state_size <= 0 ||
      d->groups <= 0 || d->heads % d->groups || !dtype_ok(d->dtype) || !dtype_ok(d->dt_dtype))
    return false;
  if (d->state_size > CO_SCAN_MAX_STATE) return false;
  const int64_t inner = mul_to(d->heads, d->head_dim, INT32_MAX);
  if (inner < 0 || mul_to(d->groups, d->state_size, INT32_MAX) < 0) return false;
  return mul_to(mul_to(d->batch, inner, kMaxValues), d->state_size, kMaxValues) >= 0;
}

}  // namespace

extern "C" {

co_status co_shortconv_query(const co_shortconv_desc* desc, int64_t* state_bytes) {
  if (!shortconv_ok(desc) || !state_bytes) return CO_EINVAL;
  *state_bytes =
      int64_t(desc->batch) * desc->channels * (desc->kernel - 1) * elem(desc->dtype);
  return CO_OK;
}

co_status co_shortconv_forward_steps(const co_shortconv_desc* desc, const co_shortconv_call* call,
                                     void* stream) {
  if (!shortconv_ok(desc) || !call || call->T < 0 || !call->weight) return CO_EINVAL;
  if (desc->has_bias && !call->bias) return CO_EINVAL;
  const int32_t T = call->T, dt = desc->dtype;
  if (T == 0) return CO_OK;
  if (!tokens_ok(call->x, desc->batch, T, dt) ||
      !out_ok(call->y, desc->batch, T, desc->channels, dt) || call->x.data == call->y.data)
    return CO_EINVAL;
  if (!aligned(call->weight, elem(dt)) || !aligned(call->bias, elem(dt)) ||
      !aligned(call->state, elem(dt)) || !aligned(call->lengths, 4))
    return CO_EINVAL;
  if (mul_to(mul_to(desc->batch, desc->channels, kMaxValues), T, kMaxValues) < 0)
    return CO_EINVAL;
  return done(launch_shortconv(*desc, *call, as_stream(stream)));
}

co_status co_scan_query(const co_scan_desc* desc, int64_t* state_bytes) {
  if (!scan_ok(desc) || !state_bytes) return CO_EINVAL;
  *state_bytes = int64_t(desc->batch) * desc->heads * desc->head_dim * desc->state_size * 4;
  return CO_OK;
}

co_status co_scan_workspace_bytes(const co_scan_desc* desc, int32_t T, int64_t* bytes) {
  if (!scan_ok(desc) || T < 0 || !bytes) return CO_EINVAL;
  *bytes = scan_chunk_takes(*desc, T) ? scan_chunk_workspace(*desc, T) : 0;
  return CO_OK;
}

co_status co_scan_forward_steps(const co_scan_desc* desc, const co_scan_call* call, void* stream) {
  if (!scan_ok(desc) || !call || call->T < 0 || !call->A || call->workspace_bytes < 0)
    return CO_EINVAL;
  const int32_t B = desc->batch, T = call->T, dt = desc->dtype;
  if (T == 0) return CO_OK;
  const int32_t inner = desc->heads * desc->head_dim;
  if (!tokens_ok(call->x, B, T, dt) || !tokens_ok(call->b, B, T, dt) ||
      !tokens_ok(call->c, B, T, dt) || !tokens_ok(call->dt, B, T, desc->dt_dtype) ||
      !out_ok(call->y, B, T, inner, dt))
    return CO_EINVAL;
  const void* y = call->y.data;
  if (y == call->x.data || y == call->b.data || y == call->c.data || y == call->dt.data)
    return CO_EINVAL;
  if (!aligned(call->A, 4) || !aligned(call->D, 4) || !aligned(call->dt_bias, 4) ||
      !aligned(call->state, 4) || !aligned(call->lengths, 4) || !aligned(call->workspace, 16))
    return CO_EINVAL;
  if (mul_to(mul_to(B, inner, kMaxValues), T, kMaxValues) < 0) return CO_EINVAL;
  const ScanCall c{*desc, *call};
  if (scan_chunk_takes(*desc, T) && call->workspace &&
      call->workspace_bytes >= scan_chunk_workspace(*desc, T))
    return done(launch_scan_chunk(c, as_stream(stream)));
  return done(launch_scan_seq(c, as_stream(stream)));
}

co_status co_norm_forward(const co_norm_desc* desc, const co_norm_call* call, void* stream) {
  return co_norm_forward_lengths(desc, call, nullptr, stream);
}

co_status co_norm_forward_lengths(const co_norm_desc* desc, const co_norm_call* call,
                                  const int32_t* lengths, void* stream) {
  if (!desc || desc->batch < 0 || desc->tokens < 0 || desc->dim <= 0 || desc->groups <= 0 ||
      desc->dim % desc->groups || !dtype_ok(desc->dtype) || !dtype_ok(desc->residual_dtype))
    return CO_EINVAL;
  if (desc->gate < CO_NORM_NONE || desc->gate > CO_NORM_AFTER || desc->residual < CO_NORM_NONE ||
      desc->residual > CO_NORM_AFTER || !(desc->eps >= 0.f) || !std::isfinite(desc->eps))
    return CO_EINVAL;
  if (desc->dim / desc->groups > CO_NORM_MAX_WIDTH) return CO_ENOTSUP;
  const int32_t B = desc->batch, T = desc->tokens, dt = desc->dtype, rt = desc->residual_dtype;
  if (mul_to(int64_t(B) * T, desc->groups, INT32_MAX) < 0) return CO_ENOTSUP;
  if (B == 0 || T == 0) return CO_OK;
  if (!call || !tokens_ok(call->x, B, T, dt)) return CO_EINVAL;
  if (desc->gate && !tokens_ok(call->gate, B, T, dt)) return CO_EINVAL;
  if (desc->residual &&
      (!tokens_ok(call->residual, B, T, rt) || !out_ok(call->residual_out, B, T, desc->dim, rt)))
    return CO_EINVAL;
  if (desc->residual != CO_NORM_AFTER && !out_ok(call->y, B, T, desc->dim, dt)) return CO_EINVAL;
  if (!aligned(call->weight, 4) || !aligned(call->scale, 4) || !aligned(lengths, 4))
    return CO_EINVAL;
  // what the form does not have takes no part in the choice of a kernel
  co_norm_call c = *call;
  const co_tokens none{nullptr, 0, 0};
  if (!desc->gate) c.gate = none;
  if (!desc->residual) c.residual = c.residual_out = none;
  if (desc->residual == CO_NORM_AFTER) c.y = none;
  for (const co_tokens* out : {&c.y, &c.residual_out}) {
    const int32_t ot = out == &c.y ? dt : rt;
    if (!out->data) continue;
    if (!in_place_ok(*out, ot, c.x, dt, B, T) || !in_place_ok(*out, ot, c.gate, dt, B, T) ||
        !in_place_ok(*out, ot, c.residual, rt, B, T))
      return CO_EINVAL;
  }
  if (c.y.data && c.y.data == c.residual_out.data) return CO_EINVAL;
  return done(launch_norm(*desc, c, lengths, as_stream(stream)));
}

}  // extern "C"
