// Keys and values into the cache's pages, 4 bits a value, and back.
// Bound by memory.  Four lanes hold a block of 32 channels, 8 values each, so that a
// token is read in whole 16-byte pieces; the block's largest magnitude is two
// exchanges away.  A workgroup writes a tile of 16 tokens of one kv head: all its
// codes lie side by side, so no line of the pool is written by two workgroups but at
// the ends of a call.  16384 tokens of 8 heads of 128, bfloat16: 16 to 19 us into the cache
// and 16 us back, 85 MB each at 4.5 to 5.2 TB/s; 64 single tokens 3.6 and 3.4 us.
#include <algorithm>

#include "cache.hpp"
#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

struct CacheArgs {
  co_attn_desc d;
  co_attn_cache c;
  co_tokens kv[2];
  const int32_t* from;
  int32_t T;
  PageHead lay;
  int64_t page_bytes;
  int32_t page_shift;
  FastDiv by_W, by_row;  // a row: the quarter blocks of a token
};

// The scale byte of a block whose largest magnitude has the float32 bits `most`; codes follow it:
// 255 where that is not finite, 0 where all codes are (up to 2^-122, half of the least one).
__device__ __forceinline__ int scale_byte(uint32_t most) {
  if (most >= 0x7f800000u) return 255;
  if (most <= 0x02800000u) return 0;
  // 2^k m, 1 <= m < 2: the least e with 2^k m <= 7 2^e
  const int e = int(most >> 23) - 127 - 2 + ((most & 0x7fffffu) > 0x600000u);
  return min(max(e, -120), 125) + 127;
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float(uint32_t(byte) << 23); }

// Eight values of channels c.. of a row, 0 past D.
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* row, int c, int D, float (&v)[8]) {
  if constexpr (WIDE) {
    constexpr int V = kWide<T>;
#pragma unroll
    for (int w = 0; w < 8 / V; ++w) {
      Pack<T, V> p{};
      if (c < D) p = load_pack<T, V>(row + c + w * V);
#pragma unroll
      for (int i = 0; i < V; ++i) v[w * V + i] = to_f32<T>(p.v[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < D ? to_f32<T>(row[c + i]) : 0.f;
  }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T* row, int c, int D, const float (&v)[8]) {
  if constexpr (WIDE) {
    constexpr int V = kWide<T>;
    if (c >= D) return;
#pragma unroll
    for (int w = 0; w < 8 / V; ++w) {
      Pack<T, V> p;
#pragma unroll
      for (int i = 0; i < V; ++i) p.v[i] = from_f32<T>(v[w * V + i]);
      store_pack<T, V>(row + c + w * V, p);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < D) row[c + i] = from_f32<T>(v[i]);
  }
}

// blockIdx: tile of the call's positions, kv head, stream.
template <typename T, bool WIDE>
__global__ __launch_bounds__(kBlock) void append_kernel(CacheArgs a) {
  const int b = blockIdx.z, h = blockIdx.y;
  const int P = a.lay.P, NB = a.lay.NB, D = a.d.head_dim;
  const int n = stream_tokens(a.c.granted, b, a.T);
  const int64_t base = a.c.base[b];
  const int64_t pos0 = (base / kCacheTile + blockIdx.x) * kCacheTile;
  if (base < 0 || pos0 >= base + n) return;
  const int lp = int(pos0 >> a.page_shift);
  const int page = a.c.table[int64_t(b) * a.d.stream_pages + lp - fdiv(lp, a.by_W) * a.d.stream_pages];
  if (page < 0 || page >= a.d.pages) return;
  char* head = static_cast<char*>(a.c.pool) + page * a.page_bytes + int64_t(h) * a.lay.bytes();
  const int tile = int(pos0 & (P - 1)) / kCacheTile;
  const int first = int(base - pos0), end = int(min(base + n - pos0, int64_t(kCacheTile)));
  const T* x[2];
#pragma unroll
  for (int w = 0; w < 2; ++w)
    x[w] = static_cast<const T*>(a.kv[w].data) + b * a.kv[w].batch_stride + int64_t(h) * D -
           first * a.kv[w].token_stride;
  for (int i = threadIdx.x; i < kCacheTile * NB * 4; i += kBlock) {
    const int tok = fdiv(i, a.by_row), rest = i - tok * NB * 4, block = rest / 4, quad = rest % 4;
    if (tok < first || tok >= end) continue;  // the four lanes of a block alike
    float v[2][8];
#pragma unroll
    for (int w = 0; w < 2; ++w)
      load8<T, WIDE>(x[w] + tok * a.kv[w].token_stride, block * kCacheBlock + quad * 8, D, v[w]);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint32_t most = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(v[w][k]) & 0x7fffffffu);
      most = max(most, uint32_t(__shfl_xor(int(most), 1)));
      most = max(most, uint32_t(__shfl_xor(int(most), 2)));
      const int s = scale_byte(most);
      uint32_t code = 0;
      if (s != 255 && s != 0) {
        const float scale = scale_of(s);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[w][0], v[w][1], scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[w][2], v[w][3], scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[w][4], v[w][5], scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[w][6], v[w][7], scale, 3);
      }
      const int at = block * kCacheTile + tok;
      *reinterpret_cast<uint32_t*>(head + a.lay.codes(w) + tile * a.lay.tile_bytes() + at * 16 +
                                   quad * 4) = code;
      if (quad == 0) head[a.lay.scales(w) + tile * NB * kCacheTile + at] = char(s);
    }
  }
}

// 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, times the scale: exact in float32.
__device__ __forceinline__ void decode8(uint32_t code, float scale, float (&v)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
  v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}

// blockIdx: 16 of the call's tokens, kv head, stream.
template <typename T, bool WIDE>
__global__ __launch_bounds__(kBlock) void read_kernel(CacheArgs a) {
  const int b = blockIdx.z, h = blockIdx.y;
  const int P = a.lay.P, NB = a.lay.NB, D = a.d.head_dim;
  const int64_t lowest = a.c.first ? max(a.c.first[b], 0) : 0;
  const int64_t end = int64_t(a.c.base[b]) + max(a.c.granted[b], 0), from = a.from[b];
  T* y[2];
#pragma unroll
  for (int w = 0; w < 2; ++w)
    y[w] = static_cast<T*>(a.kv[w].data) + b * a.kv[w].batch_stride + int64_t(h) * D;
  for (int i = threadIdx.x; i < kCacheTile * NB * 4; i += kBlock) {
    const int tok = fdiv(i, a.by_row), rest = i - tok * NB * 4, block = rest / 4, quad = rest % 4;
    const int64_t t = int64_t(blockIdx.x) * kCacheTile + tok, pos = from + t;
    if (t >= a.T) continue;
    int page = -1;
    if (pos >= lowest && pos < end && pos <= INT32_MAX) {
      const int lp = int(pos) >> a.page_shift;
      page = a.c.table[int64_t(b) * a.d.stream_pages + lp - fdiv(lp, a.by_W) * a.d.stream_pages];
    }
    float v[2][8] = {};
    if (page >= 0 && page < a.d.pages) {
      const char* head =
          static_cast<const char*>(a.c.pool) + page * a.page_bytes + int64_t(h) * a.lay.bytes();
      const int in = int(pos) & (P - 1), tile = in / kCacheTile;
      const int at = block * kCacheTile + in % kCacheTile;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t code = *reinterpret_cast<const uint32_t*>(
            head + a.lay.codes(w) + tile * a.lay.tile_bytes() + at * 16 + quad * 4);
        const int s = uint8_t(head[a.lay.scales(w) + tile * NB * kCacheTile + at]);
        decode8(code, s == 255 ? __builtin_nanf("") : scale_of(s), v[w]);
        if (s == 255)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[w][k] = __builtin_nanf("");
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w)
      store8<T, WIDE>(y[w] + t * a.kv[w].token_stride, block * kCacheBlock + quad * 8, D, v[w]);
  }
}

CacheArgs args(const co_attn_desc& d, const co_attn_cache& c, const co_tokens& k,
               const co_tokens& v, int32_t T) {
  CacheArgs a{d, c, {k, v}, nullptr, T};
  a.lay = {d.page_tokens, cache_blocks(d.head_dim)};
  a.page_bytes = int64_t(a.lay.bytes()) * d.kv_heads;
  while ((1 << a.page_shift) < d.page_tokens) ++a.page_shift;
  a.by_W = make_fastdiv(d.stream_pages);
  a.by_row = make_fastdiv(a.lay.NB * 4);
  return a;
}

// Whether pieces of 16 bytes lie on their alignment everywhere.
bool wide(const CacheArgs& a) {
  const int V = a.d.dtype == CO_BF16 ? 8 : 4, es = 16 / V;
  int64_t all = a.d.head_dim % 8 ? 1 : 0;
  for (const co_tokens& t : a.kv)
    all |= t.batch_stride | t.token_stride | int64_t(reinterpret_cast<uintptr_t>(t.data) / es);
  return all % V == 0;
}

}  // namespace

hipError_t launch_attn_append(const co_attn_desc& d, const co_attn_cache& c, const co_tokens& k,
                              const co_tokens& v, int32_t T, hipStream_t stream) {
  const CacheArgs a = args(d, c, k, v, T);
  const dim3 grid(unsigned((int64_t(T) + kCacheTile - 2) / kCacheTile + 1), unsigned(d.kv_heads),
                  unsigned(d.batch));
  if (d.dtype == CO_BF16) {
    if (wide(a)) append_kernel<bf16_t, true><<<grid, kBlock, 0, stream>>>(a);
    else append_kernel<bf16_t, false><<<grid, kBlock, 0, stream>>>(a);
  } else {
    if (wide(a)) append_kernel<float, true><<<grid, kBlock, 0, stream>>>(a);
    else append_kernel<float, false><<<grid, kBlock, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_attn_read(const co_attn_desc& d, const co_attn_cache& c, const int32_t* from,
                            const co_tokens& k, const co_tokens& v, int32_t T, hipStream_t stream) {
  CacheArgs a = args(d, c, k, v, T);
  a.from = from;
  const dim3 grid(unsigned((int64_t(T) + kCacheTile - 1) / kCacheTile), unsigned(d.kv_heads),
                  unsigned(d.batch));
  if (d.dtype == CO_BF16) {
    if (wide(a)) read_kernel<bf16_t, true><<<grid, kBlock, 0, stream>>>(a);
    else read_kernel<bf16_t, false><<<grid, kBlock, 0, stream>>>(a);
  } else {
    if (wide(a)) read_kernel<float, true><<<grid, kBlock, 0, stream>>>(a);
    else read_kernel<float, false><<<grid, kBlock, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace coinf
