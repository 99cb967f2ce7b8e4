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

// log(1 + exp(v)): log1p keeps the relative accuracy of small results, which a
// state sums over many tokens.
__device__ __forceinline__ float softplus(float v) { return v > 20.f ? v : log1pf(expf(v)); }

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
