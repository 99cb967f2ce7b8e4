// Root-mean-square norm of rows with a gate and a residual sum.
// Bound by memory: every input read once, every output written once.  A part
// (dim / groups values) stays in the registers of L lanes, at most 32 values
// each, all loaded before the first is used (but for a post-norm's residual, which
// is loaded after the sum); its sum of squares is reduced once.  16384 rows of 4096
// in bfloat16: gated 403 MB in 75 us (5.4 TB/s, a little over a large copy), with a
// float32 residual before 805 MB in 150 us (5.4 TB/s), after 671 MB in 141 us (4.8);
// a pre-norm of 64 rows of 2048 3.4 us, which is a launch.
#include <algorithm>
#include <type_traits>

#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

struct NormArgs {
  co_tokens x, z, r, y, o;  // o: the new residual
  const int32_t* lengths;
  const float* weight;
  const float* scale;
  uint32_t parts;  // tokens of all streams * groups
  uint32_t groups, tokens;
  int32_t width;
  float eps;
};

// Where a tensor has token t of stream b.
__device__ __forceinline__ int64_t place(const co_tokens& v, uint32_t b, uint32_t t) {
  return b * v.batch_stride + t * v.token_stride;
}

// V neighbouring values as float32.
template <typename T, int V>
__device__ __forceinline__ void load_f32(const void* p, int64_t at, float (&o)[V]) {
  const Pack<T, V> v = load_pack<T, V>(static_cast<const T*>(p) + at);
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = to_f32<T>(v.v[i]);
}
template <typename T, int V>
__device__ __forceinline__ void store_f32(void* p, int64_t at, const float* v) {
  Pack<T, V> o;
#pragma unroll
  for (int i = 0; i < V; ++i) o.v[i] = from_f32<T>(v[i]);
  store_pack<T, V>(static_cast<T*>(p) + at, o);
}
// V float32 values, in 16-byte pieces (V = 8 needs two), or `one` where there is no array.
template <int V>
__device__ __forceinline__ void load_vec(const float* p, int64_t at, float (&o)[V]) {
  constexpr int W = V < 4 ? V : 4;
#pragma unroll
  for (int i = 0; i < V; i += W) {
    Pack<float, W> v;
#pragma unroll
    for (int k = 0; k < W; ++k) v.v[k] = 1.f;
    if (p) v = load_pack<float, W>(p + at + i);
#pragma unroll
    for (int k = 0; k < W; ++k) o[i + k] = v.v[k];
  }
}

// T: x, z, y.  R: the residual.  L lanes a part, NV packs of V values a lane.
template <typename T, typename R, int GATE, int RES, int L, int V, int NV>
__device__ __forceinline__ void norm_parts(const NormArgs& a, uint32_t part0) {
  constexpr int WAVES = L / 64;
  // a residual of 4 bytes beside values of 2 comes in two 16-byte pieces
  constexpr int RV = V * int(sizeof(R)) > 16 ? V / 2 : V;
  const int lane = threadIdx.x % L;
  const uint32_t part = part0 + __builtin_amdgcn_readfirstlane(threadIdx.x / L);
  if (part >= a.parts) return;
  const uint32_t row = part / a.groups, b = row / a.tokens, t = row % a.tokens;
  const int base = int(part % a.groups) * a.width;
  const int64_t x0 = place(a.x, b, t) + base, z0 = GATE ? place(a.z, b, t) + base : 0;
  const int64_t r0 = RES ? place(a.r, b, t) + base : 0, o0 = RES ? place(a.o, b, t) + base : 0;
  if (a.lengths && int32_t(t) >= a.lengths[b]) {  // not read; the same in all waves of the part
    const float zero[V] = {};
    for (int e = lane * V; e < a.width; e += L * V) {
      if (RES != CO_NORM_AFTER) store_f32<T, V>(a.y.data, place(a.y, b, t) + base + e, zero);
      if (RES)
#pragma unroll
        for (int j = 0; j < V; j += RV) store_f32<R, RV>(a.o.data, o0 + e + j, zero);
    }
    return;
  }
  float v[NV][V], gate[GATE ? NV : 1][V];
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (i * L + lane) * V;
    const bool in = e < a.width;
#pragma unroll
    for (int k = 0; k < V; ++k) v[i][k] = 0.f;
    if (in) {
      load_f32<T, V>(a.x.data, x0 + e, v[i]);
      if (GATE) {
        load_f32<T, V>(a.z.data, z0 + e, gate[i]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          gate[i][k] = silu(gate[i][k]);
          if (GATE == CO_NORM_BEFORE) v[i][k] *= gate[i][k];
        }
      }
      if (RES == CO_NORM_BEFORE) {
        float s[V];
        load_vec<V>(a.scale, base + e, s);
#pragma unroll
        for (int j = 0; j < V; j += RV) {
          float r[RV];
          load_f32<R, RV>(a.r.data, r0 + e + j, r);
#pragma unroll
          for (int k = 0; k < RV; ++k) v[i][j + k] = fmaf(s[j + k], v[i][j + k], r[k]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) sum = fmaf(v[i][k], v[i][k], sum);
  }
  // stored after all loads, which a store in between would hold up
  if (RES == CO_NORM_BEFORE) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = (i * L + lane) * V;
      if (e >= a.width) break;
#pragma unroll
      for (int j = 0; j < V; j += RV)
        store_f32<R, RV>(a.o.data, o0 + e + j, v[i] + j);
    }
  }
#pragma unroll
  for (int m = 32; m > 0; m /= 2) sum += __shfl_xor(sum, m);
  if constexpr (WAVES > 1) {
    __shared__ float part_sum[WAVES];
    if (threadIdx.x % 64 == 0) part_sum[threadIdx.x / 64] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part_sum[w];
  }
  const float inv = 1.f / sqrtf(sum / float(a.width) + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (i * L + lane) * V;
    if (e >= a.width) break;
    float w[V];
    load_vec<V>(a.weight, base + e, w);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      v[i][k] = v[i][k] * inv * w[k];
      if (GATE == CO_NORM_AFTER) v[i][k] *= gate[i][k];
    }
    if (RES == CO_NORM_AFTER) {
      float s[V];
      load_vec<V>(a.scale, base + e, s);
#pragma unroll
      for (int j = 0; j < V; j += RV) {
        float r[RV];
        load_f32<R, RV>(a.r.data, r0 + e + j, r);
#pragma unroll
        for (int k = 0; k < RV; ++k) r[k] = fmaf(s[j + k], v[i][j + k], r[k]);
        store_f32<R, RV>(a.o.data, o0 + e + j, r);
      }
    } else {
      store_f32<T, V>(a.y.data, place(a.y, b, t) + base + e, v[i]);
    }
  }
}

template <typename T, typename R, int GATE, int RES, int L, int V, int NV>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_kernel(NormArgs a) {
  constexpr int PER = L < 256 ? 256 / L : 1;  // parts a workgroup
  const uint32_t by = gridDim.x * PER;  // at most 2^23: no sum here passes 32 bits
  for (uint32_t part = blockIdx.x * PER; part < a.parts; part += by) {
    norm_parts<T, R, GATE, RES, L, V, NV>(a, part);
    if (L > 64 && part + by < a.parts) __syncthreads();  // the waves' sums are read
  }
}

template <typename T, typename R, int GATE, int RES, int V>
hipError_t launch_width(const NormArgs& a, hipStream_t s) {
  // lanes by the part's width: a wave up to 512 values, 256 lanes up to 8192, then
  // 1024; a lane keeps at most 32 values
  const auto go = [&](auto kernel, int L) {
    const int per = L < 256 ? 256 / L : 1;
    const int64_t most = int64_t(1) << 21;  // then a workgroup takes several
    const int64_t grid = std::min((int64_t(a.parts) + per - 1) / per, most);
    hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(L < 256 ? 256 : L), 0, s, a);
    return hipGetLastError();
  };
  if (a.width <= 512) return go(norm_kernel<T, R, GATE, RES, 64, V, 8 / V>, 64);
  if (a.width <= 2048) return go(norm_kernel<T, R, GATE, RES, 256, V, 8 / V>, 256);
  if (a.width <= 4096) return go(norm_kernel<T, R, GATE, RES, 256, V, 16 / V>, 256);
  if (a.width <= 8192) return go(norm_kernel<T, R, GATE, RES, 256, V, 32 / V>, 256);
  return go(norm_kernel<T, R, GATE, RES, 1024, V, 32 / V>, 1024);
}

template <typename T, typename R, int V>
hipError_t launch_kind(const NormArgs& a, int gate, int res, hipStream_t s) {
  if constexpr (std::is_same_v<R, float>) {  // no residual: no type of one either
    if (res == 0 && gate == 0) return launch_width<T, R, 0, 0, V>(a, s);
    if (res == 0 && gate == 1) return launch_width<T, R, 1, 0, V>(a, s);
    if (res == 0 && gate == 2) return launch_width<T, R, 2, 0, V>(a, s);
  }
  switch (gate * 3 + res) {
    case 1: return launch_width<T, R, 0, 1, V>(a, s);
    case 2: return launch_width<T, R, 0, 2, V>(a, s);
    case 4: return launch_width<T, R, 1, 1, V>(a, s);
    case 5: return launch_width<T, R, 1, 2, V>(a, s);
    case 7: return launch_width<T, R, 2, 1, V>(a, s);
    case 8: return launch_width<T, R, 2, 2, V>(a, s);
  }
  return hipErrorInvalidValue;
}

template <typename T, typename R>
hipError_t launch_t(const NormArgs& a, int gate, int res, hipStream_t s) {
  constexpr int V = kWide<T>;
  const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const auto wide = [&](const co_tokens& t) {
    return at(t.data) && t.batch_stride % V == 0 && t.token_stride % V == 0;
  };
  // 16-byte accesses where every one of them is aligned, values otherwise
  const bool fits = a.width % V == 0 && wide(a.x) && wide(a.z) && wide(a.r) && wide(a.y) &&
                    wide(a.o) && at(a.weight) && at(a.scale);
  return fits ? launch_kind<T, R, V>(a, gate, res, s) : launch_kind<T, R, 1>(a, gate, res, s);
}

}  // namespace

hipError_t launch_norm(const co_norm_desc& d, const co_norm_call& c, const int32_t* lengths,
                       hipStream_t stream) {
  const NormArgs a{c.x, c.gate, c.residual, c.y, c.residual_out, lengths, c.weight, c.scale,
                   uint32_t(int64_t(d.batch) * d.tokens * d.groups), uint32_t(d.groups),
                   uint32_t(d.tokens), d.dim / d.groups, d.eps};
  const bool r16 = d.residual && d.residual_dtype == CO_BF16;
  if (d.dtype == CO_BF16)
    return r16 ? launch_t<bf16_t, bf16_t>(a, d.gate, d.residual, stream)
               : launch_t<bf16_t, float>(a, d.gate, d.residual, stream);
  return r16 ? launch_t<float, bf16_t>(a, d.gate, d.residual, stream)
             : launch_t<float, float>(a, d.gate, d.residual, stream);
}

}  // namespace coinf
