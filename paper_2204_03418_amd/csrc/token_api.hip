// C ABI of the token layers: short causal convolution, selective scan, norm.
// Stateless host side: every call checks its arguments, picks a kernel and
// enqueues it; a negative status means nothing ran.
#include <cmath>

#include "device.hpp"
#include "launch.hpp"

using namespace coinf;

namespace {

// Values of one tensor in a call.
constexpr int64_t kMaxValues = int64_t(1) << 38;

bool dtype_ok(int32_t t) { return t == CO_F32 || t == CO_BF16; }
int elem(int32_t t) { return t == CO_BF16 ? 2 : 4; }

bool aligned(const void* p, int a) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(a) == 0; }

// a * b, or -1 where it would pass the bound (a, b >= 0).
int64_t mul_to(int64_t a, int64_t b, int64_t bound) {
  if (a < 0 || b < 0) return -1;
  if (a && b > bound / a) return -1;
  return a * b;
}

constexpr int64_t kMaxOffset = int64_t(1) << 58;  // elements; byte offsets stay below 2^61

// Whether the last value of a (B, T, width) tensor has an offset that fits.
bool tokens_ok(const co_tokens& t, int32_t B, int32_t T, int32_t dtype) {
  return t.data && aligned(t.data, elem(dtype)) &&
         mul_to(t.batch_stride, B, kMaxOffset) >= 0 && mul_to(t.token_stride, T, kMaxOffset) >= 0;
}

// The same for an output, whose values must lie apart.
bool out_ok(const co_tokens& t, int32_t B, int32_t T, int64_t width, int32_t dtype) {
  if (!tokens_ok(t, B, T, dtype)) return false;
  if (T > 1 && t.token_stride < width) return false;
  if (B > 1 && t.batch_stride < width) return false;
  if (T == 1 || B == 1) return true;
  return t.batch_stride >= (T - 1) * t.token_stride + width ||
         t.token_stride >= (B - 1) * t.batch_stride + width;
}

// A call too large for one launch is refused by its launcher.
co_status done(hipError_t e) {
  if (e == hipErrorInvalidConfiguration) return CO_ENOTSUP;
  return e == hipSuccess ? CO_OK : CO_EHIP;
}
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

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

co_status co_shortconv_forward_steps(const co_shortconv_desc* desc, const void* weight,
                                     const void* bias, const co_tokens* x, int32_t T,
                                     const int32_t* lengths, void* state, const co_tokens* y,
                                     int32_t update_state, void* stream) {
  if (!shortconv_ok(desc) || T < 0 || !x || !y || !weight) return CO_EINVAL;
  if (desc->has_bias && !bias) return CO_EINVAL;
  if (T == 0) return CO_OK;
  const int32_t dt = desc->dtype;
  if (!tokens_ok(*x, desc->batch, T, dt) || !out_ok(*y, desc->batch, T, desc->channels, dt))
    return CO_EINVAL;
  if (x->data == y->data) return CO_EINVAL;
  if (!aligned(weight, elem(dt)) || !aligned(bias, elem(dt)) || !aligned(state, elem(dt)) ||
      !aligned(lengths, 4))
    return CO_EINVAL;
  if (mul_to(mul_to(desc->batch, desc->channels, kMaxValues), T, kMaxValues) < 0)
    return CO_EINVAL;
  return done(launch_shortconv(*desc, weight, desc->has_bias ? bias : nullptr, *x, T, lengths,
                               state, *y, update_state != 0, as_stream(stream)));
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

co_status co_scan_forward_steps(const co_scan_desc* desc, const float* A, const float* D,
                                const float* dt_bias, const co_scan_io* io, int32_t T,
                                const int32_t* lengths, float* state, int32_t update_state,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  if (!scan_ok(desc) || T < 0 || !io || !A || workspace_bytes < 0) return CO_EINVAL;
  if (T == 0) return CO_OK;
  const int32_t B = desc->batch, dt = desc->dtype;
  const int32_t inner = desc->heads * desc->head_dim;
  if (!tokens_ok(io->x, B, T, dt) || !tokens_ok(io->b, B, T, dt) || !tokens_ok(io->c, B, T, dt) ||
      !tokens_ok(io->dt, B, T, desc->dt_dtype) || !out_ok(io->y, B, T, inner, dt))
    return CO_EINVAL;
  if (io->y.data == io->x.data || io->y.data == io->b.data || io->y.data == io->c.data ||
      io->y.data == io->dt.data)
    return CO_EINVAL;
  if (!aligned(A, 4) || !aligned(D, 4) || !aligned(dt_bias, 4) || !aligned(state, 4) ||
      !aligned(lengths, 4) || !aligned(workspace, 16))
    return CO_EINVAL;
  if (mul_to(mul_to(B, inner, kMaxValues), T, kMaxValues) < 0) return CO_EINVAL;
  ScanCall c{*desc, *io, A, D, dt_bias, lengths, state, T, update_state && state ? 1 : 0};
  if (scan_chunk_takes(*desc, T) && workspace &&
      workspace_bytes >= scan_chunk_workspace(*desc, T))
    return done(launch_scan_chunk(c, workspace, as_stream(stream)));
  return done(launch_scan_seq(c, as_stream(stream)));
}

co_status co_norm_forward(const co_norm_desc* desc, const co_tokens* x, const co_tokens* gate,
                          const co_tokens* residual, const float* weight, const float* scale,
                          const co_tokens* y, const co_tokens* residual_out, void* stream) {
  if (!desc || desc->batch < 0 || desc->tokens < 0 || desc->dim <= 0 || desc->groups <= 0 ||
      desc->dim % desc->groups || !dtype_ok(desc->dtype) || !dtype_ok(desc->residual_dtype))
    return CO_EINVAL;
  if (desc->gate < CO_NORM_NONE || desc->gate > CO_NORM_AFTER || desc->residual < CO_NORM_NONE ||
      desc->residual > CO_NORM_AFTER || !(desc->eps >= 0.f) || !std::isfinite(desc->eps))
    return CO_EINVAL;
  if (desc->dim / desc->groups > CO_NORM_MAX_WIDTH) return CO_ENOTSUP;
  const int64_t rows = int64_t(desc->batch) * desc->tokens;
  if (mul_to(rows, desc->groups, INT32_MAX) < 0) return CO_ENOTSUP;
  if (rows == 0) return CO_OK;
  const auto in_ok = [&](const co_tokens* t, int32_t dtype) {
    return t && tokens_ok(*t, desc->batch, desc->tokens, dtype);
  };
  const auto result_ok = [&](const co_tokens* t, int32_t dtype) {
    return t && out_ok(*t, desc->batch, desc->tokens, desc->dim, dtype);
  };
  const int32_t dt = desc->dtype, rt = desc->residual_dtype;
  if (!in_ok(x, dt)) return CO_EINVAL;
  if (desc->gate && !in_ok(gate, dt)) return CO_EINVAL;
  if (desc->residual && (!in_ok(residual, rt) || !result_ok(residual_out, rt))) return CO_EINVAL;
  if (desc->residual != CO_NORM_AFTER && !result_ok(y, dt)) return CO_EINVAL;
  if (!aligned(weight, 4) || !aligned(scale, 4)) return CO_EINVAL;
  const co_tokens none{nullptr, 0, 0};
  return done(launch_norm(*desc, *x, desc->gate ? *gate : none, desc->residual ? *residual : none,
                          weight, scale, desc->residual != CO_NORM_AFTER ? *y : none,
                          desc->residual ? *residual_out : none, as_stream(stream)));
}

}  // extern "C"
