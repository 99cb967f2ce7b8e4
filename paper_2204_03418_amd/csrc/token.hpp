// Device helpers of the token layers.
#pragma once

#include "device.hpp"

namespace coinf {

// 16 bytes of T: 8 bfloat16 or 4 float32 values.
template <typename T>
constexpr int kWide = 16 / int(sizeof(T));

// V contiguous values from memory aligned to all of them.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
  T v[V];
};

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  return *reinterpret_cast<const Pack<T, V>*>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& v) {
  *reinterpret_cast<Pack<T, V>*>(p) = v;
}

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// v / (1 + exp(-v)); 0 for very negative v.
__device__ __forceinline__ float silu(float v) {
  return v * __builtin_amdgcn_rcpf(1.f + exp2_fast(-v * kLog2e));
}

// log(1 + exp(v)) = max(v, 0) + log(1 + u), u = exp(-|v|), to 4e-7 of its value also where it is
// small: a state sums it over many tokens.  exp takes what the product with log2(e) rounds off as
// a factor; with w = 1 + u rounded, log(w) u / (w - 1) is log(1 + u) without w's rounding (Kahan).
// 20 instructions where log1pf(expf(v)) has 137.
__device__ __forceinline__ float softplus(float v) {
  const float a = fmaxf(-fabsf(v), -128.f);
  const float h = a * kLog2e;
  const float low = fmaf(a, kLog2e, -h) + a * 1.925963033500e-8f;  // of log2(e)
  float u = exp2_fast(h);
  u = fmaf(u, low * 0.69314718055994530942f, u);
  const float w = 1.f + u, d = w - 1.f;
  const float log_w = __builtin_amdgcn_logf(w) * 0.69314718055994530942f;
  const float l = d > 0.f ? log_w * (u * __builtin_amdgcn_rcpf(d)) : u;
  return (v < 0.f ? 0.f : v) + l;  // NaN stays
}

// Tokens of stream b in a call over T.
__device__ __forceinline__ int stream_tokens(const int32_t* lengths, int b, int T) {
  return lengths ? min(max(lengths[b], 0), T) : T;
}

// Whether a launch of so many workgroups has a size the hardware takes (fewer
// than 2^32 threads).
inline bool grid_fits(int64_t grid, int block = kBlock) {
  return grid > 0 && grid < (int64_t(1) << 32) / block;
}

}  // namespace coinf
