// Layout of the cache's pages (include/coinf.h), host and device.
#pragma once

#include <cstdint>

namespace coinf {

constexpr int kCacheBlock = 32;  // channels that share a scale
constexpr int kCacheTile = 16;   // tokens side by side

// Bytes of one kv head in a page of P tokens, and where its parts lie.
struct PageHead {
  int32_t P, NB;
  __host__ __device__ int32_t tile_bytes() const { return NB * kCacheTile * 16; }
  __host__ __device__ int32_t codes_bytes() const { return P / kCacheTile * tile_bytes(); }
  __host__ __device__ int32_t scales_bytes() const { return P * NB; }
  __host__ __device__ int32_t bytes() const { return 2 * (codes_bytes() + scales_bytes()); }
  // which 0: K, 1: V
  __host__ __device__ int32_t codes(int which) const { return which * codes_bytes(); }
  __host__ __device__ int32_t scales(int which) const {
    return 2 * codes_bytes() + which * scales_bytes();
  }
};

inline int32_t cache_blocks(int32_t head_dim) {
  return (head_dim + kCacheBlock - 1) / kCacheBlock;
}

}  // namespace coinf
