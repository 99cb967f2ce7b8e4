// Rotary positions: pairs of a head's values turn by an angle that grows with the
// position.  Bound by memory: queries and keys are read and written once, in one
// launch.  A workgroup makes the sines and cosines of its tokens' pairs once, one
// a thread, in LDS, and all heads use them (computed for each head they would cost
// about as much as the memory).  16384 tokens of 40 heads of 128, bfloat16: 65 to 70 us,
// 336 MB at 4.8 to 5.2 TB/s; 24 single tokens 3.6 us, the launch.
//
// The angle in turns is position * f / (2 pi) modulo 1, an exact 64-bit product of
// the position and the frequency in units of 2^-64 turns; what is left of the nearest
// quarter turn is rounded to float32 once, and sine and cosine are their Taylor
// series there.
#include <algorithm>

#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

// Tokens of a workgroup at most.
constexpr int kMaxTokens = 8;
constexpr int kMaxPairs = CO_ATTN_MAX_HEAD / 2;

struct RotaryArgs {
  co_rotary_desc d;
  co_rotary_call c;
  FastDiv by_T, by_heads, by_units;
  int32_t tokens;      // of all streams
  int32_t groups;      // of group_tokens tokens
  int32_t group_tokens;
  int32_t turn_units;  // of V pairs a head
  int32_t units;       // a head: and of V values that stay
  int32_t in_place;    // bit i: y[i] is x[i]
};

// Sine and cosine of 2^-64 turns * frac.  |x| <= pi / 4: the series' next terms are below
// 2^-29 and 2^-29.
__device__ __forceinline__ float2 sincos_turns(uint64_t frac) {
  const uint64_t quarter = (frac + (uint64_t(1) << 61)) >> 62;
  const int64_t rest = int64_t(frac - (quarter << 62));
  const float x = float(rest) * 3.40612158008655459e-19f;  // 2 pi 2^-64
  const float z = x * x;
  float s = fmaf(z, 2.7557319223985893e-6f, -1.9841269841269841e-4f);
  s = fmaf(z, s, 8.3333333333333333e-3f);
  s = fmaf(z, s, -1.6666666666666667e-1f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -2.7557319223985888e-7f, 2.4801587301587302e-5f);
  c = fmaf(z, c, -1.3888888888888889e-3f);
  c = fmaf(z, c, 4.1666666666666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const bool swap = quarter & 1;
  const float a = swap ? c : s, b = swap ? s : c;
  return {quarter & 2 ? -a : a, (quarter + 1) & 2 ? -b : b};
}

// Where a pair's sine and cosine lie: of units of eight, which are 64 bytes, every other four have
// their 16-byte parts in another order, so that eight units' first parts lie in all banks (a call 71.8 -> 69.4 us).
template <int V>
__device__ __forceinline__ int place(int pair) {
  return V == 8 ? pair ^ (pair / 32 % 2 * 2) : pair;
}

// V pairs, or V values that stay, a unit.
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kBlock) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 turn[kMaxTokens * kMaxPairs];  // cosine, sine
  __shared__ int32_t stream[kMaxTokens], token[kMaxTokens];  // token -1: past the length
  const int R = a.d.rotary_dim, pairs = R / 2, D = a.d.head_dim;
  for (int group = blockIdx.x; group < a.groups; group += gridDim.x) {
    const int n0 = group * a.group_tokens;
    const int count = min(a.group_tokens, a.tokens - n0);
    if (group != int(blockIdx.x)) __syncthreads();
    for (int i = threadIdx.x; i < count * pairs; i += kBlock) {
      const int k = i / pairs, pair = i - k * pairs;
      const int b = fdiv(n0 + k, a.by_T), t = n0 + k - b * a.c.T;
      const int64_t p =
          a.c.positions ? a.c.positions[b * a.c.position_batch_stride +
                                        t * a.c.position_token_stride] +
                              int64_t(a.c.position_each ? 0 : t)
                        : t;
      const float2 v = sincos_turns(uint64_t(p) * a.c.turns[pair]);
      turn[k * pairs + place<V>(pair)] = {v.y * a.d.magnitude, v.x * a.d.magnitude};
      if (pair == 0) {
        stream[k] = b;
        token[k] = t < stream_tokens(a.c.lengths, b, a.c.T) ? t : ~t;
      }
    }
    __syncthreads();
    const int heads = a.d.heads[0] + a.d.heads[1];
    for (int u = threadIdx.x; u < count * heads * a.units; u += kBlock) {
      const int row = fdiv(u, a.by_units), unit = u - row * a.units;
      const int k = fdiv(row, a.by_heads);
      int h = row - k * heads;
      const int which = h >= a.d.heads[0];
      h -= which ? a.d.heads[0] : 0;
      const int b = stream[k];
      const bool live = token[k] >= 0;
      const int t = live ? token[k] : ~token[k];
      const co_tokens& in = a.c.x[which];
      const co_tokens& out = a.c.y[which];
      const T* x = static_cast<const T*>(in.data) + b * in.batch_stride + t * in.token_stride +
                   int64_t(h) * D;
      T* y = static_cast<T*>(out.data) + b * out.batch_stride + t * out.token_stride +
             int64_t(h) * D;
      if (unit >= a.turn_units) {  // values that stay
        const int at = R + (unit - a.turn_units) * V;
        Pack<T, V> v{};
        if (live) {
          if (a.in_place >> which & 1) continue;
          v = load_pack<T, V>(x + at);
        }
        store_pack<T, V>(y + at, v);
        continue;
      }
      const int pair = unit * V;
      const int at0 = HALF ? pair : 2 * pair, at1 = HALF ? pairs + pair : 2 * pair + V;
      Pack<T, V> v0{}, v1{};
      if (live) {
        v0 = load_pack<T, V>(x + at0);
        v1 = load_pack<T, V>(x + at1);
        const float2* cs = turn + k * pairs + pair;
        const int moved = place<V>(pair) - pair;  // of the unit's first
#pragma unroll
        for (int i = 0; i < V; ++i) {
          // the pair's places: i of either pack, or neighbours
          T& lo = HALF ? v0.v[i] : 2 * i < V ? v0.v[2 * i % V] : v1.v[2 * i % V];
          T& hi = HALF ? v1.v[i] : 2 * i + 1 < V ? v0.v[(2 * i + 1) % V] : v1.v[(2 * i + 1) % V];
          const float p = to_f32<T>(lo), q = to_f32<T>(hi);
          const float2 r = cs[i ^ moved];
          lo = from_f32<T>(fmaf(p, r.x, -(q * r.y)));
          hi = from_f32<T>(fmaf(q, r.x, p * r.y));
        }
      }
      store_pack<T, V>(y + at0, v0);
      store_pack<T, V>(y + at1, v1);
    }
  }
}

template <typename T, int V>
void run(const RotaryArgs& a, unsigned grid, hipStream_t s) {
  if (a.d.layout == CO_ROTARY_HALF)
    rotary_kernel<T, V, true><<<grid, kBlock, 0, s>>>(a);
  else
    rotary_kernel<T, V, false><<<grid, kBlock, 0, s>>>(a);
}

}  // namespace

hipError_t launch_rotary(const co_rotary_desc& d, const co_rotary_call& c, hipStream_t stream) {
  RotaryArgs a;
  a.d = d;
  a.c = c;
  const int es = d.dtype == CO_BF16 ? 2 : 4, pairs = d.rotary_dim / 2;
  const int64_t tokens = int64_t(d.batch) * c.T;
  const int heads = d.heads[0] + d.heads[1];
  // a workgroup's units have 31-bit indexes
  if (tokens >= INT32_MAX || int64_t(heads) * kMaxTokens * d.head_dim >= INT32_MAX)
    return hipErrorInvalidConfiguration;
  // values of a pack: as many as every pointer, stride and part of a head is a multiple of
  int64_t all = pairs | (d.head_dim - d.rotary_dim) | d.head_dim;
  for (int i = 0; i < (d.heads[1] ? 2 : 1); ++i)
    for (const co_tokens* v : {&c.x[i], &c.y[i]})
      all |= v->batch_stride | v->token_stride | int64_t(reinterpret_cast<uintptr_t>(v->data) / es);
  int V = 16 / es;
  while (all % V) V /= 2;
  a.tokens = int32_t(tokens);
  // sines for all threads, but a workgroup for each of 1024 tokens first
  a.group_tokens = int32_t(std::max<int64_t>(
      1, std::min<int64_t>({kMaxTokens, std::max(1, kBlock / pairs), tokens / 1024})));
  a.groups = int32_t((tokens + a.group_tokens - 1) / a.group_tokens);
  a.turn_units = pairs / V;
  a.units = a.turn_units + (d.head_dim - d.rotary_dim) / V;
  a.by_T = make_fastdiv(c.T);
  a.by_heads = make_fastdiv(heads);
  a.by_units = make_fastdiv(a.units);
  a.in_place = (c.x[0].data == c.y[0].data) | (c.x[1].data == c.y[1].data) << 1;
  const unsigned grid = unsigned(std::min(a.groups, 1 << 20));
  if (d.dtype == CO_BF16) {
    if (V == 8) run<bf16_t, 8>(a, grid, stream);
    else if (V == 4) run<bf16_t, 4>(a, grid, stream);
    else if (V == 2) run<bf16_t, 2>(a, grid, stream);
    else run<bf16_t, 1>(a, grid, stream);
  } else {
    if (V == 4) run<float, 4>(a, grid, stream);
    else if (V == 2) run<float, 2>(a, grid, stream);
    else run<float, 1>(a, grid, stream);
  }
  return hipGetLastError();
}

}  // namespace coinf
