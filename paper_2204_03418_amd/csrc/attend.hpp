// What the attention kernels share.
#pragma once

#include <type_traits>

#include "cache.hpp"
#include "launch.hpp"
#include "token.hpp"

namespace coinf {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct AttendArgs {
  co_attn_desc d;
  co_attn_cache c;
  co_tokens q, y;
  int32_t T;
  PageHead lay;
  int64_t page_bytes;
  float scale_log2;    // > 0
  float slack;         // of scores: kSlack
  float q_sign;        // -1, 0 or 1: the scale's
  int32_t group;       // query heads a kv head
  FastDiv by_group, by_W;
  int32_t page_shift;  // log2 of a page's tokens
  int32_t row_tiles;   // of a stream's tokens * group
  FastDiv by_row_tiles, by_splits, by_kv;
  int32_t pairs;       // streams * kv heads
  int32_t splits;      // parts of a unit's keys at most
  int32_t keys;        // of a tile
  int32_t part_tiles;  // of a part at least
  int32_t wide;        // q and y four values at a time
  float* part;         // (units, splits, rows, NB * 32) values, then (.., rows) reference score and sum
  float2* part_stat;
};

constexpr int kMostKeys = 128;  // of a tile

// Weights are 2^{x + kLift}, x <= kSlack over the row's reference: 2^15, below 16-bit floats' highest.
// Their least step is 2^-24, 2^-35 of the row's reference.
constexpr float kLift = 11.f, kSlack = 4.f;
// Values are 16-bit floats c 2^{s - E + kValueLift}, s <= E: below 6 2^12, and taken as that down to
// s = E - kSpan, c = 0.5: exact for bfloat16 calls; normal (2^-14 and more) for float32, since matrix
// instructions sum denormal ones with fewer bits (45 rows that see only values 2^20 below others moved by
// 1 bit, 2^24 by 6e-8, 2^28 by 6.6e-7).  E, one for all channels and keys of a pass (those too that a row does
// not see), only rises.  A pass that meets values further below it, or in which it rises by more than
// kMostRise (sums under the first one are 2^-13 and more, and keep 24 bits above 2^-126), is lost.
// It is taken again with values as bfloat16, c 2^{s - E + kFarLift} under the last E, which are exact
// down to s = E - 204, and weights in bfloat16 terms: sums over 2^31 keys stay below 2^127, and those
// of values down to s = E - 170 keep 24 bits.
constexpr int kValueLift = 12, kValueSlack = 4;
template <typename T>
constexpr int kSpan = sizeof(T) == 2 ? 35 : 25;
constexpr int kMostRise = 85, kFarLift = 78;

// What a stream's rows see.
struct Span {
  int base, n;  // n: tokens of the call
  int lowest;
  __device__ Span(const AttendArgs& a, int b) : base(a.c.base[b]) {
    // positions stay below 2^31
    n = base < 0 ? 0 : min(stream_tokens(a.c.granted, b, a.T), INT32_MAX - 4 * kMostKeys - base);
    n = max(n, 0);
    lowest = a.c.first ? max(a.c.first[b], 0) : 0;
  }
  // a token's first key
  __device__ int lo(const AttendArgs& a, int t) const {
    const int w = a.d.window ? base - a.d.window + 1 + t : 0;
    return max(w, lowest);
  }
};

// Tiles first..end - 1 of a unit's part `split` of the keys lo..hi - 1; parts: of the unit.
struct Part {
  int first, end, parts;
  __device__ Part(const AttendArgs& a, int lo, int hi, int split) {
    const int t0 = lo / a.keys, t1 = lo < hi ? (hi + a.keys - 1) / a.keys : t0;
    const int each = max((t1 - t0 + a.splits - 1) / a.splits, a.part_tiles);
    parts = max((t1 - t0 + each - 1) / each, 1);
    first = min(t0 + split * each, t1);
    end = min(first + each, t1);
  }
};

// The largest of the lanes' values.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_max(int v) {
  return max(v, __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int wave_max(int v) {  // v >= 0
  v = dpp_max<0x111, 0xf>(v);  // from 1, 2, 4 and 8 lanes below, within 16
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);  // lane 15 of the 16 below
  v = dpp_max<0x143, 0xc>(v);  // lane 31
  return __builtin_amdgcn_readlane(v, 63);
}

// A kernel's only argument, read again: the compiler would keep the first pass's for the second.
__device__ __forceinline__ const AttendArgs& again(const AttendArgs&) {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttendArgs*)(p);
}

// Four values of channels c.. of a row, 0 past D.
template <typename T>
__device__ __forceinline__ void load4(const T* row, int c, int D, bool wide, float* v) {
  if (wide) {
    Pack<T, 4> p{};
    if (c < D) p = load_pack<T, 4>(row + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32<T>(p.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < D ? to_f32<T>(row[c + i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* row, int c, int D, bool wide, const float* v) {
  if (wide) {
    Pack<T, 4> p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.v[i] = from_f32<T>(v[i]);
    if (c < D) store_pack<T, 4>(row + c, p);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < D) row[c + i] = from_f32<T>(v[i]);
  }
}

__device__ __forceinline__ float exponent_to_f32(int biased) {
  return __uint_as_float(uint32_t(min(max(biased, 0), 254)) << 23);
}

// The 8-bit terms of 16 values, 2^{e - 4 k} the scale of term k: words[k] 16 bytes.  A term has 4 bits
// and steps of 2^-9 of its scale at least.  Two, where the block's largest is 2^7 of the first scale
// and more, hold a bfloat16 exactly down to 2^-13 of that largest, and leave up to 2^-21 of it
// (half of 2^-13 2^-7) below.
template <int TERMS>
__device__ __forceinline__ void to_terms(float (&v)[16], int scale_byte, i32x4 (&words)[TERMS]) {
#pragma unroll
  for (int k = 0; k < TERMS; ++k) {
    const float scale = exponent_to_f32(scale_byte - 4 * k);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      s16x2 p = {0, 0};
      p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[4 * w], v[4 * w + 1], scale, false);
      p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[4 * w + 2], v[4 * w + 3], scale, true);
      const int word = __builtin_bit_cast(int, p);
      words[k][w] = word;
      if (k + 1 < TERMS) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, scale, false);
        const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, scale, true);
        v[4 * w] -= lo[0], v[4 * w + 1] -= lo[1], v[4 * w + 2] -= hi[0], v[4 * w + 3] -= hi[1];
      }
    }
  }
}

// The scale byte of a block of queries whose largest magnitude has the bits `most`: that lies in
// 2^7..2^8 of it (below 2^-80: multiples of 2^-96).
__device__ __forceinline__ int query_scale(uint32_t most) {
  return max(int(most >> 23) - 7, 40);
}

// Scores.  bfloat16: keys as they are against queries in two 8-bit terms, whose instructions sum to about
// 2^-20 of their largest product; what the terms leave of a query adds to that.  float32: those sums would be its error (4e-6 to 1e-5 measured), so
// its keys become bfloat16 (exactly) and its queries three bfloat16 terms (24 bits).
template <typename T>
constexpr int kQueryTerms = sizeof(T) == 2 ? 2 : 3;
template <typename T>
constexpr int kWeightTerms = sizeof(T) == 2 ? 1 : 2;
template <typename T>
constexpr int kFarTerms = sizeof(T) == 2 ? 2 : 3;  // bfloat16: 16 or 24 bits

// Eight codes as 16-bit floats, times the scale.
__device__ __forceinline__ f16x8 decode8(uint32_t w, float scale) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight codes as bfloat16, times 2^{byte - 127}; NaN for 255.
__device__ __forceinline__ bf16x8 decode8_bf16(uint32_t w, int byte) {
  const float scale = __uint_as_float(byte == 255 ? 0x7fc00000u : uint32_t(byte) << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Whether values of scale s lie too far below E; those of scale 0 are 0.
template <typename T>
__device__ __forceinline__ bool lost_values(int s, int E) {
  return uint32_t(s - 1) < uint32_t(max(E - kSpan<T> - 1, 0));
}
// The exponent of the pass for far values: outputs' factor 2^{E - kFarLift - 127} is in float32's range.
__device__ __forceinline__ int far_exponent(int E) { return max(E, kFarLift + 1); }
// Eight of them for the pass of far values.
__device__ __forceinline__ bf16x8 decode8_far(uint32_t w, int s, int E) {
  const int byte = 127 + kFarLift + s - E;
  const bool some = s != 0 && s != 255 && byte > 0;
  return decode8_bf16(some ? w : 0, some ? byte : 127);
}

// Eight values as bfloat16 terms.
template <int TERMS>
__device__ __forceinline__ void to_bf16_terms(float (&v)[8], bf16x8 (&terms)[TERMS]) {
#pragma unroll
  for (int k = 0; k < TERMS; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      terms[k][i] = __bf16(v[i]);
      v[i] -= float(terms[k][i]);
    }
}

// Four rows of 16 columns of an LDS tile of 16-bit values, turned: lane j of 16 gets column j.
// p: this lane's row j / 4 and columns 4 (j % 4).
__device__ __forceinline__ s16x4 turned4(const _Float16* p) {
  using Lds = __attribute__((address_space(3))) s16x4;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(p));
}


// Calls of at most kFewTiles * 16 rows, in column tiles of 16.
constexpr int kFewTiles = 2, kFewKeys = 64;
void launch_attend_few(const AttendArgs& a, int NB, int tiles, hipStream_t stream);
// The others, 128 or 256 rows a workgroup: 256 for heads of at most so many blocks (whose queries and
// sums leave registers for two waves a SIMD).
template <typename T>
constexpr int kWideBlocks = sizeof(T) == 2 ? 4 : 2;
void launch_attend_rows(const AttendArgs& a, int NB, int rows, hipStream_t stream);

}  // namespace coinf
