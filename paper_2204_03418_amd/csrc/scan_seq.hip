// Selective scan, token after token, with the state in registers:
//   S = exp(d A) S + d x (outer) B,  y = S C + D x.
// Bound by the state, read and written once: a row of it lies across NL lanes,
// four values each, and a thread keeps ROWS rows, all loaded together.  64
// streams of 64 heads of 64 x 128, one token: 268 MB of states in 55.2 us (4.9
// TB/s).  Further tokens add 0.3 us each, or 0.14 us a million state values:
// about 100 vector instructions for 32 values a lane; the next token's inputs
// are loaded over the last one's, d_t is made for 64 tokens at once, and the
// sums over a row cross lanes in registers (32 streams of 64 heads, 16 tokens:
// 113 us with LDS permutes and a softplus in every thread a token, 58 us so).
#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

struct SeqArgs {
  ScanCall c;
  int32_t p_blocks;
};

// The value of lane l ^ M, within rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int M>
__device__ __forceinline__ float xor_lane(float v) {
  static_assert(M == 1 || M == 2 || M == 4 || M == 8);
  if constexpr (M == 1) return dpp<0xb1>(v);         // 1 0 3 2 of each four
  if constexpr (M == 2) return dpp<0x4e>(v);         // 2 3 0 1
  if constexpr (M == 4) return dpp<0x1b>(dpp<0x141>(v));  // 7 - l of each eight, then 3 - l of four
  return dpp<0x128>(v);                              // 8 round in sixteen
}
// a over the lanes without bit M plus over those with it, the same of b: the lanes without bit M
// get a's sum, the others b's.
template <int M>
__device__ __forceinline__ float halves(float a, float b, bool up) {
  if constexpr (M >= 16) {  // one instruction swaps rows of 16 (or 32) between two registers
    const auto r = M == 16
        ? __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false)
        : __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    return (up ? b : a) + xor_lane<M>(up ? a : b);
  }
}
// Sums each of v[0..ROWS) over NL lanes: while there are several rows, lanes exchange halves of
// them, so lane l of the NL ends with row l / (NL / ROWS).
template <int M, int N, int ROWS>
__device__ __forceinline__ float reduce_rows(float (&v)[ROWS], int nl) {
  if constexpr (M == 0) {
    return v[0];
  } else if constexpr (N > 1) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = halves<M>(v[i], v[i + N / 2], nl & M);
    return reduce_rows<M / 2, N / 2>(v, nl);
  } else {
    v[0] = halves<M>(v[0], v[0], nl & M);
    return reduce_rows<M / 2, 1>(v, nl);
  }
}

__device__ __forceinline__ float load_dt(const co_scan_call& io, int dt_dtype, int64_t at) {
  return dt_dtype == CO_BF16 ? bf16_to_f32(static_cast<const bf16_t*>(io.dt.data)[at])
                             : static_cast<const float*>(io.dt.data)[at];
}

// A lane's values of B or C: 4 neighbours where WIDE, else NL apart.
template <typename T, int NL, bool WIDE>
__device__ __forceinline__ Pack<T, 4> load_n(const T* p, int nl, int N) {
  if (WIDE) return nl * 4 < N ? load_pack<T, 4>(p + nl * 4) : Pack<T, 4>{};
  Pack<T, 4> r{};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (nl + NL * j < N) r.v[j] = p[nl + NL * j];
  return r;
}

// One token's inputs of a thread.
template <typename T, int ROWS>
struct Token {
  Pack<T, 4> b, c;
  Pack<T, ROWS> x;
};

// ONE: a call over single tokens.
template <typename T, int NL, int ROWS, bool WIDE, bool ONE>
__global__ __launch_bounds__(kBlock) void scan_seq_kernel(SeqArgs a) {
  constexpr int GROUPS = kBlock / NL;
  const co_scan_desc& d = a.c.d;
  const co_scan_call& io = a.c.c;
  const int nl = threadIdx.x % NL, group = threadIdx.x / NL;
  const int pb = int(blockIdx.x % uint32_t(a.p_blocks));
  const int bh = int(blockIdx.x / uint32_t(a.p_blocks));
  const int h = bh % d.heads, b = bh / d.heads;
  const int g = h / (d.heads / d.groups);
  const int P = d.head_dim, N = d.state_size;
  const int p0 = (pb * GROUPS + group) * ROWS;
  const int len = stream_tokens(a.c.c.lengths, b, a.c.c.T);

  const T* xp = static_cast<const T*>(io.x.data) + b * io.x.batch_stride + int64_t(h) * P + p0;
  const T* bp = static_cast<const T*>(io.b.data) + b * io.b.batch_stride + int64_t(g) * N;
  const T* cp = static_cast<const T*>(io.c.data) + b * io.c.batch_stride + int64_t(g) * N;
  T* yp = static_cast<T*>(io.y.data) + b * io.y.batch_stride + int64_t(h) * P + p0;
  const int64_t dt0 = b * io.dt.batch_stride + h;
  float* sp = a.c.c.state ? a.c.c.state + (int64_t(bh) * P + p0) * N : nullptr;

  const auto load_token = [&](int t) {
    Token<T, ROWS> k;
    k.b = load_n<T, NL, WIDE>(bp + t * io.b.token_stride, nl, N);
    k.c = load_n<T, NL, WIDE>(cp + t * io.c.token_stride, nl, N);
    const T* x = xp + t * io.x.token_stride;
    k.x = Pack<T, ROWS>{};
    if (WIDE) {
      if (p0 < P) k.x = load_pack<T, ROWS>(x);
    } else {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
        if (p0 + r < P) k.x.v[r] = x[r];
    }
    return k;
  };
  Token<T, ROWS> now{};
  if (len > 0) now = load_token(0);
  float S[ROWS][4] = {};
  if (sp && len > 0) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (p0 + r >= P) break;
      const Pack<float, 4> v = load_n<float, NL, WIDE>(sp + int64_t(r) * N, nl, N);
#pragma unroll
      for (int j = 0; j < 4; ++j) S[r][j] = v.v[j];
    }
  }
  const float A2 = a.c.c.A[h] * kLog2e, D = a.c.c.D ? a.c.c.D[h] : 0.f;
  const float bias = a.c.c.dt_bias ? a.c.c.dt_bias[h] : 0.f;
  constexpr int STEP = NL / ROWS;  // lanes that end with the same row
  const int row = nl / STEP;
  // d_t and e^{d_t A}: of 64 tokens at once, a token a lane, in every wave
  const auto decays = [&](int t) {
    float dt = 0.f;
    if (t < len) {
      dt = load_dt(io, d.dt_dtype, dt0 + t * io.dt.token_stride) + bias;
      if (d.dt_softplus) dt = softplus(dt);
    }
    return dt;
  };
  float dts = decays(ONE ? 0 : int(threadIdx.x % 64));

  for (int t = 0; t < len; ++t) {
    Token<T, ROWS> next = now;
    if (!ONE && t + 1 < len) next = load_token(t + 1);
    if (!ONE && t > 0 && t % 64 == 0) dts = decays(t + int(threadIdx.x % 64));
    const float dt = ONE ? dts : __uint_as_float(__builtin_amdgcn_readlane(
                                     __float_as_uint(dts), t % 64));
    const float decay = exp2_fast(fmaxf(dt * A2, -160.f));
    float y[ROWS], xr = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      y[r] = 0.f;
      const float x = to_f32<T>(now.x.v[r]), u = dt * x;
      if (r == row) xr = x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        S[r][j] = fmaf(decay, S[r][j], u * to_f32<T>(now.b.v[j]));
        y[r] = fmaf(S[r][j], to_f32<T>(now.c.v[j]), y[r]);
      }
    }
    const float sum = reduce_rows<NL / 2, ROWS>(y, nl);
    if (nl % STEP == 0 && p0 + row < P)
      yp[t * io.y.token_stride + row] = from_f32<T>(fmaf(D, xr, sum));
    if (ONE) break;
    now = next;
  }
  for (int t = len; t < a.c.c.T; ++t)
    if (nl % STEP == 0 && p0 + row < P) yp[t * io.y.token_stride + row] = T{};

  if (a.c.c.state && a.c.c.update_state && len > 0) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (p0 + r >= P) break;
      float* q = sp + int64_t(r) * N;
      if (WIDE) {
        if (nl * 4 < N) store_pack<float, 4>(q + nl * 4, {S[r][0], S[r][1], S[r][2], S[r][3]});
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (nl + NL * j < N) q[nl + NL * j] = S[r][j];
      }
    }
  }
}

template <typename T, int NL, int ROWS>
hipError_t launch_rows(const ScanCall& c, bool wide, hipStream_t s) {
  const int per = kBlock / NL * ROWS;
  const int64_t p_blocks = (int64_t(c.d.head_dim) + per - 1) / per;
  if (p_blocks * per > INT32_MAX) return hipErrorInvalidConfiguration;  // rows are counted in int
  SeqArgs a{c, int32_t(p_blocks)};
  const int64_t grid = int64_t(a.p_blocks) * c.d.heads * c.d.batch;
  if (!grid_fits(grid)) return hipErrorInvalidConfiguration;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(kBlock), 0, s, a);
    return hipGetLastError();
  };
  if (c.c.T == 1)
    return wide ? go(scan_seq_kernel<T, NL, ROWS, true, true>)
                : go(scan_seq_kernel<T, NL, ROWS, false, true>);
  return wide ? go(scan_seq_kernel<T, NL, ROWS, true, false>)
              : go(scan_seq_kernel<T, NL, ROWS, false, false>);
}

template <typename T, int NL>
hipError_t launch_lanes(const ScanCall& c, bool wide, hipStream_t s) {
  // As many rows a thread as leave about four workgroups for each of 256 CUs.
  const int64_t rows = int64_t(c.d.batch) * c.d.heads * c.d.head_dim;
  const int64_t fill = rows / (int64_t(kBlock / NL) * 1024);
  const int64_t fit = int64_t(c.d.head_dim) * NL / kBlock;  // rows that one head gives a thread
  const int64_t most = fill < fit ? fill : fit;
  if constexpr (NL >= 8)
    if (most >= 8) return launch_rows<T, NL, 8>(c, wide, s);
  if (most >= 4) return launch_rows<T, NL, 4>(c, wide, s);
  if (most >= 2) return launch_rows<T, NL, 2>(c, wide, s);
  return launch_rows<T, NL, 1>(c, wide, s);
}

template <typename T>
hipError_t launch_t(const ScanCall& c, hipStream_t s) {
  const int N = c.d.state_size;
  const auto at = [](const void* p, int a) { return reinterpret_cast<uintptr_t>(p) % a == 0; };
  const auto by = [&](const co_tokens& t, int n) {
    return at(t.data, n * sizeof(T)) && t.batch_stride % n == 0 && t.token_stride % n == 0;
  };
  // a state row, and the rows that a thread has of x, in whole pieces
  const bool wide = N % 4 == 0 && c.d.head_dim % 8 == 0 && at(c.c.state, 16) && by(c.c.b, 4) &&
                    by(c.c.c, 4) && by(c.c.x, 8);
  if (N <= 16) return launch_lanes<T, 4>(c, wide, s);
  if (N <= 32) return launch_lanes<T, 8>(c, wide, s);
  if (N <= 64) return launch_lanes<T, 16>(c, wide, s);
  if (N <= 128) return launch_lanes<T, 32>(c, wide, s);
  return launch_lanes<T, 64>(c, wide, s);
}

}  // namespace

hipError_t launch_scan_seq(const ScanCall& c, hipStream_t stream) {
  if (c.d.dtype == CO_BF16) return launch_t<bf16_t>(c, stream);
  return launch_t<float>(c, stream);
}

}  // namespace coinf
