// Attention over the cache: a wave a row of queries, keys across its lanes.
#include <algorithm>

#include "cache.hpp"
#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

struct AttendArgs {
  co_attn_desc d;
  co_attn_cache c;
  co_tokens q, y;
  int32_t T;
  PageHead lay;
  int64_t page_bytes;
  float scale_log2;
};

__device__ __forceinline__ float code_value(int c) {
  const int m = c & 7;
  const float v = m < 2 ? 0.5f * m
                        : __uint_as_float(uint32_t(126 + (m >> 1)) << 23 | uint32_t(m & 1) << 22);
  return c & 8 ? -v : v;
}
__device__ __forceinline__ float value_at(const char* head, const PageHead& lay, int which, int in,
                                          int c) {
  const int tile = in / kCacheTile, at = c / kCacheBlock * kCacheTile + in % kCacheTile;
  const int s = uint8_t(head[lay.scales(which) + tile * lay.NB * kCacheTile + at]);
  const int two = uint8_t(head[lay.codes(which) + tile * lay.tile_bytes() + at * 16 + c % 32 / 2]);
  return code_value(c & 1 ? two >> 4 : two) *
         (s == 255 ? __builtin_nanf("") : __uint_as_float(uint32_t(s) << 23));
}

template <typename T>
__global__ __launch_bounds__(64) void attend_row_kernel(AttendArgs a) {
  const int lane = threadIdx.x, H = a.d.heads, D = a.d.head_dim;
  __shared__ float q[CO_ATTN_MAX_HEAD];
  __shared__ float p[64];
  __shared__ const char* at[64];
  const int64_t rows = int64_t(a.d.batch) * a.T * H;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int h = int(row % H), t = int(row / H % a.T), b = int(row / H / a.T);
    const int n = stream_tokens(a.c.granted, b, a.T);
    const int64_t pos = int64_t(a.c.base[b]) + t;
    int64_t lo = a.c.first ? max(a.c.first[b], 0) : 0;
    if (a.d.window) lo = max(lo, pos - a.d.window + 1);
    const T* src = static_cast<const T*>(a.q.data) + b * a.q.batch_stride +
                   t * a.q.token_stride + int64_t(h) * D;
    T* dst = static_cast<T*>(a.y.data) + b * a.y.batch_stride + t * a.y.token_stride +
             int64_t(h) * D;
    float o[4] = {}, m = -__builtin_inff(), l = 0.f;
    __syncthreads();
    if (t < n) {
      for (int c = lane; c < D; c += 64) q[c] = to_f32<T>(src[c]);
      __syncthreads();
      for (int64_t j0 = lo; j0 <= pos; j0 += 64) {
        const int64_t j = j0 + lane;
        int page = -1;
        if (j <= pos)
          page = a.c.table[int64_t(b) * a.d.stream_pages + j / a.lay.P % a.d.stream_pages];
        const bool on = page >= 0 && page < a.d.pages;
        const char* head = static_cast<const char*>(a.c.pool) + (on ? page : 0) * a.page_bytes +
                           int64_t(h / (H / a.d.kv_heads)) * a.lay.bytes();
        float s = 0.f;
        if (on)
          for (int c = 0; c < D; ++c) s = fmaf(q[c], value_at(head, a.lay, 0, int(j % a.lay.P), c), s);
        s = on ? s * a.scale_log2 : -__builtin_inff();
        float top = s;
        for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
        const float m2 = fmaxf(m, top);
        const float w = on ? exp2_fast(s - m2) : 0.f;
        float sum = w;
        for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
        const float keep = m2 == m ? 1.f : exp2_fast(m - m2);
        l = l * keep + sum;
        m = m2;
        p[lane] = w;
        at[lane] = on ? head : nullptr;
        __syncthreads();
        for (int i = 0; i < 4; ++i) {
          const int c = lane + 64 * i;
          if (c >= D) break;
          o[i] *= keep;
          for (int k = 0; k < 64; ++k)
            if (at[k]) o[i] = fmaf(p[k], value_at(at[k], a.lay, 1, int((j0 + k) % a.lay.P), c), o[i]);
        }
        __syncthreads();
      }
    }
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < D) dst[lane + 64 * i] = from_f32<T>(l != 0.f ? o[i] / l : 0.f);
  }
}

}  // namespace

int64_t attend_workspace(const co_attn_desc&, int32_t) { return 0; }

hipError_t launch_attend(const co_attn_desc& d, const co_attn_cache& c, const co_tokens& q,
                         const co_tokens& y, int32_t T, void*, hipStream_t stream) {
  AttendArgs a{d, c, q, y, T};
  a.lay = {d.page_tokens, cache_blocks(d.head_dim)};
  a.page_bytes = int64_t(a.lay.bytes()) * d.kv_heads;
  a.scale_log2 = d.scale * kLog2e;
  const unsigned grid = unsigned(std::min<int64_t>(int64_t(d.batch) * T * d.heads, 1 << 20));
  if (d.dtype == CO_BF16)
    attend_row_kernel<bf16_t><<<grid, 64, 0, stream>>>(a);
  else
    attend_row_kernel<float><<<grid, 64, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace coinf
