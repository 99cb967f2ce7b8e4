// Short causal convolution over tokens with its activation:
//   y[t,c] = act(bias[c] + sum_k w[c,k] x[t-K+1+k,c]).
// Bound by memory: x read once, y written once, 2K flops a value.  A thread
// takes 16 bytes of channels and runs of kRun tokens, whose loads are in flight
// together and over the run before; the K - 1 tokens before its first run it
// loads again.  4 x 4096 tokens of 4352 channels in bfloat16: 285 MB, 313 with what
// is loaded twice, in 58 us (5.4 TB/s); six tokens of 32 streams 6.0 us, one token
// of 64 streams 4.3 us.
#include "launch.hpp"
#include "short_conv.hpp"
#include "token.hpp"

namespace coinf {

namespace {

static_assert(kBlock == kConvThreads);

struct ConvCall {
  const void* weight;
  const void* bias;
  const void* x;
  void* y;
  void* state;
  const int32_t* lengths;
  int64_t x_batch, x_token, y_batch, y_token;
  int32_t C, T, act, update;
  int32_t c_blocks, t_blocks;  // workgroups across the channels and along the tokens
  int32_t runs;                // of a thread
};

__device__ __forceinline__ float activate(float v, int act) {
  if (act == CO_ACT_SILU) return silu(v);
  return act == CO_ACT_RELU ? fmaxf(v, 0.f) : v;
}

// V channels a thread, a.runs runs of RUN tokens a thread; LANES threads across the
// channels, 256 / LANES threads along the tokens.
template <typename T, int K, int V, int RUN, int LANES>
__global__ __launch_bounds__(kBlock) void shortconv_kernel(ConvCall a) {
  constexpr int ROWS = kBlock / LANES;
  const int lane = threadIdx.x % LANES, seg = threadIdx.x / LANES;
  const int cb = int(blockIdx.x % uint32_t(a.c_blocks));
  const int rest = int(blockIdx.x / uint32_t(a.c_blocks));
  const int tb = rest % a.t_blocks, b = rest / a.t_blocks;
  const int64_t c = (int64_t(cb) * LANES + lane) * V;
  const int64_t t0 = (int64_t(tb) * ROWS + seg) * RUN * a.runs;
  if (c >= a.C || t0 >= a.T) return;
  const int len = stream_tokens(a.lengths, b, a.T);
  const T* x = static_cast<const T*>(a.x) + b * a.x_batch + c;
  T* y = static_cast<T*>(a.y) + b * a.y_batch + c;
  T* state = a.state ? static_cast<T*>(a.state) + int64_t(b) * (K - 1) * a.C + c : nullptr;

  const auto load_run = [&](Pack<T, V>(&to)[RUN], int64_t t) {
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      to[i] = Pack<T, V>{};
      if (t + i < len) to[i] = load_pack<T, V>(x + (t + i) * a.x_token);
    }
  };
  // the K - 1 tokens before the run, from x, or the state before token 0
  Pack<T, V> old[K > 1 ? K - 1 : 1], first[K > 1 ? K - 1 : 1], run[RUN];
#pragma unroll
  for (int i = 0; i < K - 1; ++i) {
    const int64_t t = t0 + i - (K - 1);
    old[i] = Pack<T, V>{};
    if (t >= 0) {
      if (t < len) old[i] = load_pack<T, V>(x + t * a.x_token);
    } else if (state) {
      old[i] = load_pack<T, V>(state + (t + K - 1) * a.C);
    }
    first[i] = old[i];
  }
  load_run(run, t0);
  float w[V][K], bias[V];
  {
    Pack<T, V> raw[K];
    const T* wp = static_cast<const T*>(a.weight) + c * K;
#pragma unroll
    for (int k = 0; k < K; ++k) raw[k] = load_pack<T, V>(wp + k * V);
#pragma unroll
    for (int i = 0; i < V * K; ++i) w[i / K][i % K] = to_f32<T>(raw[i / V].v[i % V]);
    Pack<T, V> rb{};
    if (a.bias) rb = load_pack<T, V>(static_cast<const T*>(a.bias) + c);
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = to_f32<T>(rb.v[v]);
  }
  for (int r = 0; r < a.runs; ++r) {
    const int64_t t1 = t0 + int64_t(r) * RUN;
    if (t1 >= a.T) break;
    Pack<T, V> next[RUN];
    if (r + 1 < a.runs) load_run(next, t1 + RUN);  // in flight over this run's sums
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      const int64_t t = t1 + i;
      Pack<T, V> out{};
      if (t < len) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float s = bias[v];
#pragma unroll
          for (int k = 0; k < K; ++k) {
            const int at = i + k - (K - 1);
            s = fmaf(w[v][k], to_f32<T>(at < 0 ? old[at + K - 1 < 0 ? 0 : at + K - 1].v[v]
                                               : run[at < 0 ? 0 : at].v[v]), s);
          }
          out.v[v] = from_f32<T>(activate(s, a.act));
        }
      }
      if (t < a.T) store_pack<T, V>(y + t * a.y_token, out);
    }
    if (r + 1 < a.runs) {
#pragma unroll
      for (int i = 0; i < K - 1; ++i) {
        const int at = RUN + i - (K - 1);  // of old and run together, RUN tokens on
        old[i] = at < 0 ? old[at + K - 1 < 0 ? 0 : at + K - 1] : run[at < 0 ? 0 : at];
      }
#pragma unroll
      for (int i = 0; i < RUN; ++i) run[i] = next[i];
    }
  }
  // The state is read by the threads of token 0 alone (shortconv_cut), and they write
  // it: its j-th token is number len - (K - 1) + j of the call, or what the old state has.
  if (K > 1 && t0 == 0 && a.update && len > 0) {
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
      Pack<T, V> v{};
      if (RUN == 1) {
        v = j + 1 < K - 1 ? first[j + 1 < K - 1 ? j + 1 : 0] : run[0];  // the old ones move up
      } else if (len + j >= K - 1) {
        v = load_pack<T, V>(x + (len + j - (K - 1)) * a.x_token);
      } else {
#pragma unroll
        for (int i = j + 1; i < K - 1; ++i)
          if (i == len + j) v = first[i];
      }
      store_pack<T, V>(state + int64_t(j) * a.C, v);
    }
  }
}

template <typename T, int K, int V>
hipError_t launch_k(ConvCall a, int32_t B, hipStream_t s) {
  const int64_t packs = (int64_t(a.C) + V - 1) / V;
  const ShortConvCut cut = shortconv_cut(B, packs, a.T, K);
  const auto go = [&](auto kernel) {
    a.c_blocks = int32_t((packs + cut.lanes - 1) / cut.lanes);
    a.t_blocks = cut.t_blocks;
    a.runs = cut.runs;
    const int64_t grid = int64_t(a.c_blocks) * a.t_blocks * B;
    if (!grid_fits(grid)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(kBlock), 0, s, a);
    return hipGetLastError();
  };
  if (cut.run == 1) return go(shortconv_kernel<T, K, V, 1, kBlock>);
  return cut.lanes == 64 ? go(shortconv_kernel<T, K, V, kRun, 64>)
                         : go(shortconv_kernel<T, K, V, kRun, 32>);
}

template <typename T, int V>
hipError_t launch_v(const ConvCall& a, int32_t B, int32_t K, hipStream_t s) {
  switch (K) {
    case 1: return launch_k<T, 1, V>(a, B, s);
    case 2: return launch_k<T, 2, V>(a, B, s);
    case 3: return launch_k<T, 3, V>(a, B, s);
    case 4: return launch_k<T, 4, V>(a, B, s);
    case 5: return launch_k<T, 5, V>(a, B, s);
    case 6: return launch_k<T, 6, V>(a, B, s);
    case 7: return launch_k<T, 7, V>(a, B, s);
    case 8: return launch_k<T, 8, V>(a, B, s);
  }
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_t(const ConvCall& a, int32_t B, int32_t K, hipStream_t s) {
  constexpr int V = kWide<T>;
  const auto wide = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  // 16-byte accesses where every one of them is aligned, values otherwise
  const bool fits = a.C % V == 0 && a.x_batch % V == 0 && a.x_token % V == 0 &&
                    a.y_batch % V == 0 && a.y_token % V == 0 && wide(a.x) && wide(a.y) &&
                    wide(a.weight) && wide(a.bias) && wide(a.state);
  return fits ? launch_v<T, V>(a, B, K, s) : launch_v<T, 1>(a, B, K, s);
}

}  // namespace

hipError_t launch_shortconv(const co_shortconv_desc& d, const co_shortconv_call& c,
                            hipStream_t stream) {
  const ConvCall a{c.weight, d.has_bias ? c.bias : nullptr, c.x.data, c.y.data, c.state, c.lengths,
                   c.x.batch_stride, c.x.token_stride, c.y.batch_stride, c.y.token_stride,
                   d.channels, c.T, d.act, c.update_state && c.state ? 1 : 0, 0, 0, 1};
  if (d.dtype == CO_BF16) return launch_t<bf16_t>(a, d.batch, d.kernel, stream);
  return launch_t<float>(a, d.batch, d.kernel, stream);
}

}  // namespace coinf
