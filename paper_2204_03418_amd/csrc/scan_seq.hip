// Selective scan, token after token, with the state in registers:
//   S = exp(d A) S + d x (outer) B,  y = S C + D x.
// For single tokens and short calls it is bound by the state, read and written
// once: a row of it lies across NL lanes, four values each, and a thread keeps
// ROWS rows, all loaded together.
#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

struct SeqArgs {
  ScanCall c;
  int32_t p_blocks;
};

// Sums each of v[0..ROWS) over NL lanes: while there are several rows, lanes
// exchange halves of them, so lane l of the NL ends with row l / (NL / ROWS).
template <int NL, int ROWS>
__device__ __forceinline__ float reduce_rows(float (&v)[ROWS], int nl) {
  int n = ROWS;
#pragma unroll
  for (int m = NL / 2; m > 0; m /= 2) {
    if (n > 1) {
      n /= 2;
      const bool up = nl & m;
#pragma unroll
      for (int i = 0; i < ROWS / 2; ++i) {
        if (i >= n) break;
        const float keep = up ? v[i + n] : v[i];
        const float send = up ? v[i] : v[i + n];
        v[i] = keep + __shfl_xor(send, m);
      }
    } else {
      v[0] += __shfl_xor(v[0], m);
    }
  }
  return v[0];
}

__device__ __forceinline__ float load_dt(const co_scan_io& io, int dt_dtype, int64_t at) {
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

template <typename T, int NL, int ROWS, bool WIDE>
__global__ __launch_bounds__(kBlock) void scan_seq_kernel(SeqArgs a) {
  constexpr int GROUPS = kBlock / NL;
  const co_scan_desc& d = a.c.d;
  const co_scan_io& io = a.c.io;
  const int nl = threadIdx.x % NL, group = threadIdx.x / NL;
  const int pb = int(blockIdx.x % uint32_t(a.p_blocks));
  const int bh = int(blockIdx.x / uint32_t(a.p_blocks));
  const int h = bh % d.heads, b = bh / d.heads;
  const int g = h / (d.heads / d.groups);
  const int P = d.head_dim, N = d.state_size;
  const int p0 = (pb * GROUPS + group) * ROWS;
  const int len = stream_tokens(a.c.lengths, b, a.c.T);

  const T* xp = static_cast<const T*>(io.x.data) + b * io.x.batch_stride + int64_t(h) * P + p0;
  const T* bp = static_cast<const T*>(io.b.data) + b * io.b.batch_stride + int64_t(g) * N;
  const T* cp = static_cast<const T*>(io.c.data) + b * io.c.batch_stride + int64_t(g) * N;
  T* yp = static_cast<T*>(io.y.data) + b * io.y.batch_stride + int64_t(h) * P + p0;
  const int64_t dt0 = b * io.dt.batch_stride + h;
  float* sp = a.c.state ? a.c.state + (int64_t(bh) * P + p0) * N : nullptr;

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
  const float A2 = a.c.A[h] * kLog2e, D = a.c.D ? a.c.D[h] : 0.f;
  const float bias = a.c.dt_bias ? a.c.dt_bias[h] : 0.f;
  constexpr int STEP = NL / ROWS;  // lanes that end with the same row
  const int row = nl / STEP;

  for (int t = 0; t < len; ++t) {
    const Pack<T, 4> bv = load_n<T, NL, WIDE>(bp + t * io.b.token_stride, nl, N);
    const Pack<T, 4> cv = load_n<T, NL, WIDE>(cp + t * io.c.token_stride, nl, N);
    float x[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      x[r] = p0 + r < P ? to_f32<T>(xp[t * io.x.token_stride + r]) : 0.f;
    float dt = load_dt(io, d.dt_dtype, dt0 + t * io.dt.token_stride) + bias;
    if (d.dt_softplus) dt = softplus(dt);
    const float decay = exp2_fast(fmaxf(dt * A2, -160.f));
    float y[ROWS], xr = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      y[r] = 0.f;
      const float u = dt * x[r];
      if (r == row) xr = x[r];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        S[r][j] = fmaf(decay, S[r][j], u * to_f32<T>(bv.v[j]));
        y[r] = fmaf(S[r][j], to_f32<T>(cv.v[j]), y[r]);
      }
    }
    const float sum = reduce_rows<NL, ROWS>(y, nl);
    if (nl % STEP == 0 && p0 + row < P)
      yp[t * io.y.token_stride + row] = from_f32<T>(fmaf(D, xr, sum));
  }
  for (int t = len; t < a.c.T; ++t)
    if (nl % STEP == 0 && p0 + row < P) yp[t * io.y.token_stride + row] = T{};

  if (a.c.update && len > 0) {
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
  SeqArgs a{c, (c.d.head_dim + per - 1) / per};
  const int64_t grid = int64_t(a.p_blocks) * c.d.heads * c.d.batch;
  if (!grid_fits(grid)) return hipErrorInvalidConfiguration;
  if (wide)
    hipLaunchKernelGGL((scan_seq_kernel<T, NL, ROWS, true>), dim3(unsigned(grid)), dim3(kBlock), 0,
                       s, a);
  else
    hipLaunchKernelGGL((scan_seq_kernel<T, NL, ROWS, false>), dim3(unsigned(grid)), dim3(kBlock),
                       0, s, a);
  return hipGetLastError();
}

template <typename T, int NL>
hipError_t launch_lanes(const ScanCall& c, bool wide, hipStream_t s) {
  // As many rows a thread as leave about four workgroups for each of 256 CUs.
  const int64_t rows = int64_t(c.d.batch) * c.d.heads * c.d.head_dim;
  const int64_t fill = rows / (int64_t(kBlock / NL) * 1024);
  const int fit = c.d.head_dim * NL / kBlock;  // rows that one head gives a thread
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
  const auto four = [&](const co_tokens& t) {
    return at(t.data, 4 * sizeof(T)) && t.batch_stride % 4 == 0 && t.token_stride % 4 == 0;
  };
  const bool wide = N % 4 == 0 && at(c.state, 16) && four(c.io.b) && four(c.io.c);
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
