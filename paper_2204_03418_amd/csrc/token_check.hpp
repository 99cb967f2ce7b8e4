// Argument checks that the C ABI of the token layers and of attention share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "coinf.h"

namespace coinf {

// Values of one tensor in a call.
constexpr int64_t kMaxValues = int64_t(1) << 38;

inline bool dtype_ok(int32_t t) { return t == CO_F32 || t == CO_BF16; }
inline int elem(int32_t t) { return t == CO_BF16 ? 2 : 4; }

inline bool aligned(const void* p, int a) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(a) == 0; }

// a * b, or -1 where it would pass the bound (a, b >= 0).
inline int64_t mul_to(int64_t a, int64_t b, int64_t bound) {
  if (a < 0 || b < 0) return -1;
  if (a && b > bound / a) return -1;
  return a * b;
}

constexpr int64_t kMaxOffset = int64_t(1) << 58;  // elements; byte offsets stay below 2^61

// Whether the last value of a (B, T, width) tensor has an offset that fits.
inline bool tokens_ok(const co_tokens& t, int32_t B, int32_t T, int32_t dtype) {
  return t.data && aligned(t.data, elem(dtype)) &&
         mul_to(t.batch_stride, B, kMaxOffset) >= 0 && mul_to(t.token_stride, T, kMaxOffset) >= 0;
}

// The same for an output, whose values must lie apart.
inline bool out_ok(const co_tokens& t, int32_t B, int32_t T, int64_t width, int32_t dtype) {
  if (!tokens_ok(t, B, T, dtype)) return false;
  if (T > 1 && t.token_stride < width) return false;
  if (B > 1 && t.batch_stride < width) return false;
  if (T == 1 || B == 1) return true;
  return t.batch_stride >= (T - 1) * t.token_stride + width ||
         t.token_stride >= (B - 1) * t.batch_stride + width;
}

// Whether an output may be written while workgroups still read an input: they are apart, or it is
// in place, every value where the input has it.
inline bool in_place_ok(const co_tokens& out, int32_t out_dtype, const co_tokens& in, int32_t in_dtype,
                 int32_t B, int32_t T) {
  return out.data != in.data ||
         (elem(out_dtype) == elem(in_dtype) && (B == 1 || out.batch_stride == in.batch_stride) &&
          (T == 1 || out.token_stride == in.token_stride));
}

// A call too large for one launch is refused by its launcher.
inline co_status done(hipError_t e) {
  if (e == hipErrorInvalidConfiguration) return CO_ENOTSUP;
  return e == hipSuccess ? CO_OK : CO_EHIP;
}
inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

}  // namespace coinf
