// Selective scan over chunks of Q tokens on the matrix cores.  With the log
// decays l_t = d_t A and cum_t their sums from the chunk's start, a chunk that
// begins in state S has
//   y_t = e^{cum_t} S C_t + sum_{s<=t} e^{cum_t - cum_s} d_s (B_s . C_t) x_s + D x_t
//   S'  = e^{cum_Q} S + sum_s (e^{cum_Q - cum_s} d_s x_s) (outer) B_s,
// four products of sizes Q, P and N.  A workgroup's four waves are four units of
// a group's heads, a unit being PT * 16 of a head's P rows; they share the
// chunk's B and C and the products B_s . C_t in LDS.  A wave keeps its state
// in the accumulators of S' all along (S^T, rows n and columns p), which are
// also the layout that the product with C takes it in: the depth index of a
// matrix instruction may be permuted freely if both operands agree, so lane
// group g holds the depths 4g..4g+3 and 16+4g..16+4g+3, exactly the rows it has
// of two 16-row result tiles.  The same holds for B_s . C_t, whose result tiles
// become the operand of the product with x without leaving their lanes.
//
// bfloat16: x, B and C are used as they are.  What is float32 and becomes an
// operand goes in bfloat16 terms: two (16 bits) of e^{...} d_s (B_s . C_t) and of
// the state in its product with C, whose sums are rounded to bfloat16 once as y, 8
// bits; three (24 bits) of the weighted x in the state's sum, which goes on being
// summed.  With one term of the first two, y was off by u times the sum of its
// terms' magnitudes, far more than its own rounding where they cancel, and
// differed as much from single tokens (16384 tokens of 64 heads: 190 us with one
// term, 200 to 215 with two).  float32 inputs use the float32 matrix instructions
// throughout.
//
// A small launch before makes what the heads of a group and the units of a head
// share: the products B_s . C_t, and of each chunk its decays.  Long sequences
// of few heads are cut into segments of whole chunks that run beside each other:
// one launch makes each segment's own sum, a small one carries the states across
// them, and the last computes everything.
//
// Chunks of 32 tokens: one depth of a matrix instruction, and the products
// within a chunk (Q P) stay small beside those with the state (2 N P).  64
// tokens took 65 registers more than two waves of a SIMD have.
//
// Measured: 16384 tokens of 64 heads of 64 x 128, one group, bfloat16: 283 MB and
// 43 GFLOP of the recurrence in 200 us; the launches take 12 us (B . C, decays),
// 71 us (segments' sums), 14 us (carry) and 151 us (outputs) when traced.  The
// last runs its matrix instructions at 626 TFLOP/s (256 without the further terms
// of the split operands); it is bound by issue and latency at two waves a SIMD
// (matrix pipes busy 38% of the cycles, vector units 68%, waves waiting 21%), not
// by memory (327 MB from and to memory in it, 2.2 TB/s).  Tried and no faster:
// three waves a SIMD (spills), eight waves a workgroup, operands read further
// ahead, matrix and vector instructions interleaved by hand, sums of finer parts than
// the segments at three and four waves a SIMD.
#include <type_traits>

#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kChunk = 32;  // Q, the depth of one matrix instruction
constexpr int kPairs = 3;   // 16 x 16 tiles of B . C at and below the diagonal: (0,0), (0,1), (1,1)

// Decays of one chunk of a head, l2 = log2 of them: what its waves read.
struct ChunkDecay {
  float total;  // of the chunk
  float reach;  // the largest magnitude of the sums
  float pad[2];
  // 2^{cum_t}, and from kChunk on 2^{-cum_t} d_t, or 2^{total - cum_t} d_t where the reach passes
  // kSpan: a value for each lane of a wave
  float factor[2 * kChunk];
  // where the reach passes kSpan: d_t, and cum_t = cum + cum_low
  float step[kChunk], cum[kChunk], cum_low[kChunk];
};
static_assert(sizeof(ChunkDecay) % 16 == 0);
static_assert(std::extent_v<decltype(ChunkDecay::factor)> == 64);

struct ChunkArgs {
  ScanCall c;
  f32x4* ws_bc;          // (B, G, chunks, kPairs, 64 lanes): tiles of B . C
  ChunkDecay* ws_decay;  // (B H, chunks)
  float* ws_state;       // (B H, segments, P, N): a segment's sum, then its first state
  float* ws_total;       // (B H, segments): a segment's log2 decay
  int32_t chunks;
  int32_t unit_blocks;   // workgroups a group of heads
  int32_t p_blocks;      // units a head
  int32_t segments;
  int32_t seg_chunks;    // chunks a segment
};

// Depth-32 operand of a 16 x 16 product: lane l holds row (or column) l % 16 and
// the depths 16 a + 4 (l / 16) + i, a < 2, i < 4, at index 4 a + i.
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
  bf16x8 v;
};
template <>
struct Frag<float> {
  float v[8];
};

__device__ __forceinline__ void mma(f32x4& acc, const Frag<bf16_t>& a, const Frag<bf16_t>& b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x4& acc, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], acc, 0, 0, 0);
}

__device__ __forceinline__ float get(const Frag<bf16_t>& f, int i) { return float(f.v[i]); }
__device__ __forceinline__ float get(const Frag<float>& f, int i) { return f.v[i]; }

// The operand nearest to v, and in v what is left of it.
__device__ __forceinline__ void take(Frag<bf16_t>& f, float (&v)[8]) {
  uint32_t pairs[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    pairs[i] = __builtin_bit_cast(
        uint32_t, __builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2));
    v[2 * i] -= __uint_as_float(pairs[i] << 16);
    v[2 * i + 1] -= __uint_as_float(pairs[i] & 0xffff0000u);
  }
  struct Four {
    uint32_t p[4];
  };
  f.v = __builtin_bit_cast(bf16x8, Four{{pairs[0], pairs[1], pairs[2], pairs[3]}});
}
__device__ __forceinline__ void take(Frag<float>& f, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = v[i], v[i] = 0.f;
}

__device__ __forceinline__ void round_to(Frag<bf16_t>& f, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = __bf16(v[i]);
}
__device__ __forceinline__ void round_to(Frag<float>& f, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = v[i];
}

// Whether one of an operand's values is not finite.
__device__ __forceinline__ bool not_finite(const Frag<bf16_t>& f) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  struct Words {
    uint32_t w[4];
  };
  const Words v = __builtin_bit_cast(Words, f.v);
  u16x2 most = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)  // both halves of a word at once
    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v.w[i] & 0x7fff7fffu));
  return max(most[0], most[1]) >= 0x7f80;
}
__device__ __forceinline__ bool not_finite(const Frag<float>& f) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(f.v[i]) & 0x7fffffffu);
  return most >= 0x7f800000u;
}

// Puts 0 in the place of the values that are not finite, and in `bad` 1 for each of them.
template <typename T>
__device__ __forceinline__ void part_finite(Frag<T>& f, Frag<T>& bad) {
  float keep[8], out[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = get(f, i);
    const bool fine = fabsf(v) < __builtin_inff();
    keep[i] = fine ? v : 0.f;
    out[i] = fine ? 0.f : 1.f;
  }
  round_to(f, keep);
  round_to(bad, out);
}

// An operand's depths 4 g..4 g + 3 and 16 + 4 g..16 + 4 g + 3.
__device__ __forceinline__ Frag<bf16_t> join(const Pack<bf16_t, 4>& lo, const Pack<bf16_t, 4>& hi) {
  struct Both {
    Pack<bf16_t, 4> lo, hi;
  };
  return {__builtin_bit_cast(bf16x8, Both{lo, hi})};
}
__device__ __forceinline__ Frag<float> join(const Pack<float, 4>& lo, const Pack<float, 4>& hi) {
  Frag<float> f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f.v[i] = lo.v[i], f.v[4 + i] = hi.v[i];
  return f;
}

// Rows row0..row0+15 of an LDS tile, depths along its columns from col0.
template <typename T>
__device__ __forceinline__ Frag<T> rows_of(const T* tile, int stride, int row0, int col0) {
  const int l = threadIdx.x % 64;
  const T* p = tile + (row0 + l % 16) * stride + col0 + 4 * (l / 16);
  return join(load_pack<T, 4>(p), load_pack<T, 4>(p + 16));
}

// Columns of an LDS tile, depths along its rows from row0.  four = the first of
// the 4 neighbouring columns that lanes 4q..4q+3 of 16 take, for q = l % 4 (the
// transposing read gathers them so); one = the column of lane l % 16.
__device__ __forceinline__ Frag<bf16_t> cols_of(const bf16_t* tile, int stride, int row0, int four,
                                                int one) {
  const int l = threadIdx.x % 64;
  const bf16_t* p = tile + (row0 + 4 * (l / 16) + l % 16 / 4) * stride + four;
  using Lds = __attribute__((address_space(3))) s16x4;
  struct Both {
    s16x4 lo, hi;
  } r;
  r.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(p));
  r.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(p + 16 * stride));
  (void)one;
  return {__builtin_bit_cast(bf16x8, r)};
}
__device__ __forceinline__ Frag<float> cols_of(const float* tile, int stride, int row0, int four,
                                               int one) {
  const int l = threadIdx.x % 64;
  const float* p = tile + (row0 + 4 * (l / 16)) * stride + one;
  Frag<float> f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = p[(16 * (i / 4) + i % 4) * stride];
  (void)four;
  return f;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, int(uint32_t(u)), CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, int(uint32_t(u >> 32)), CTRL, ROWS, 0xf, false);
  return v + __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
// Sum over the lanes of this half wave up to this one.
__device__ __forceinline__ double prefix_sum32(double v) {
  v = dpp_add<0x111, 0xf>(v);  // from 1, 2, 4 and 8 lanes below, within 16
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  return dpp_add<0x142, 0xa>(v);  // lane 15 of the 16 below
}
template <int LANE>
__device__ __forceinline__ double from_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane(int(uint32_t(u)), LANE);
  const uint32_t hi = __builtin_amdgcn_readlane(int(uint32_t(u >> 32)), LANE);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
// 2^v to a few units in the last place also where v is large.
__device__ __forceinline__ float pow2(double v) {
  const double n = rint(v);
  return ldexpf(exp2_fast(float(v - n)), int(n));
}

// The largest log2 by which a chunk's factors are scaled (to either side): its sums keep the
// rest of float32's range.
constexpr float kSpan = 64.f;

// A value that all lanes have.
__device__ __forceinline__ float uniform(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}

// kWide values of a row from column col of `width`, zero past it and where !on.
template <typename T>
__device__ __forceinline__ Pack<T, kWide<T>> load_row(const T* row, int col, int width, bool on) {
  Pack<T, kWide<T>> r{};
#pragma unroll
  for (int i = 0; i < kWide<T>; ++i)
    if (on && col + i < width) r.v[i] = row[col + i];
  return r;
}
// The same 16 bytes wide, zero out of the buffer's range.
template <typename T>
__device__ __forceinline__ Pack<T, kWide<T>> load_pack_at(__amdgpu_buffer_rsrc_t r, int voff,
                                                          int soff) {
  return __builtin_bit_cast(Pack<T, kWide<T>>,
                            __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0));
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T, int W>
__device__ __forceinline__ void store_pack_at(__amdgpu_buffer_rsrc_t r, int voff,
                                              const Pack<T, W>& v) {
  if constexpr (sizeof(v) == 16)
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, voff, 0, 0);
  else
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), r, voff, 0, 0);
}

template <typename T, int NT, int PT>
struct Tile {
  static constexpr int Q = kChunk;
  static constexpr int NW = NT * 16, PW = PT * 16;
  // Row strides: rows read as operand rows lie 16 bytes beside a multiple of the 64 banks (or
  // spread as well), rows that the transposing read gathers 32 bytes.
  static constexpr int CS = NW + 16 / int(sizeof(T));
  static constexpr int BS = sizeof(T) == 2 ? NW + 16 : CS;
  static constexpr int XS = PW + 16 / int(sizeof(T));
  static constexpr int QT = Q / 16;

  T b[Q * BS];
  T c[Q * CS];
  T x[kWaves][Q * XS];
  f32x4 bc[kPairs][64];
  float grow[kWaves][Q], weight[kWaves][Q];  // with the base in them
};

// Makes ws_bc and ws_decay: a wave the tiles of B . C of a chunk, or two chunks of kHeads heads.
// Bound by latency (memory, and a new kernel's instructions), so few waves with much on the way
// and without branches between their loads (16 ragged prompts of 8 groups 12.6 -> 9.9 us).
constexpr int kHeads = 4;
template <typename T, bool WIDE>
__global__ __launch_bounds__(kBlock) void scan_prepare_kernel(ChunkArgs a) {
  const co_scan_desc& d = a.c.d;
  const co_scan_call& io = a.c.c;
  const int lane = threadIdx.x % 64, g16 = lane / 16, l16 = lane % 16;
  const uint32_t doubles = uint32_t(a.chunks + 1) / 2;
  const int two = int(blockIdx.x % doubles), b = int(blockIdx.x / doubles);
  const int job = int(blockIdx.y) * (kBlock / 64) +
                  __builtin_amdgcn_readfirstlane(int(threadIdx.x / 64));
  const int head_jobs = (d.heads + kHeads - 1) / kHeads;
  if (job >= head_jobs + 2 * d.groups) return;
  const int len = stream_tokens(a.c.c.lengths, b, a.c.c.T);
  if (job >= head_jobs) {
    const int j = job - head_jobs, group = j / 2, chunk = 2 * two + j % 2;
    const int64_t t0 = int64_t(chunk) * kChunk;
    if (t0 >= len) return;  // nobody reads it
    const int left = int(min(len - t0, int64_t(kChunk))), N = d.state_size;
    // rows 0..15 and 16..31 of B and of C, as depth-32 operands: both take depth 8 g16 + i as i
    const int64_t stride[2] = {io.b.token_stride, io.c.token_stride};
    const T* base[2] = {static_cast<const T*>(io.b.data) + b * io.b.batch_stride +
                            int64_t(group) * N + t0 * stride[0],
                        static_cast<const T*>(io.c.data) + b * io.c.batch_stride +
                            int64_t(group) * N + t0 * stride[1]};
    f32x4 acc[kPairs] = {};
    constexpr int AHEAD = 2;  // depth blocks on the way together
    constexpr int V = kWide<T>, es = sizeof(T);
    struct Eight {
      Pack<T, V> v[8 / V];
    };
    for (int k0 = 0; k0 < N; k0 += 32 * AHEAD) {
      Eight v[AHEAD][2][2];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int row = 16 * half + l16;
#pragma unroll
            for (int w = 0; w < 8 / V; ++w) {
              const int n = k0 + 32 * u + 8 * g16 + V * w;
              if (WIDE)
                v[u][side][half].v[w] = load_pack_at<T>(
                    make_rsrc(base[side], kOutOfRange),
                    row < left && n < N ? (row * int(stride[side]) + n) * es : kOutOfRange, 0);
              else
                v[u][side][half].v[w] =
                    load_row<T>(base[side] + row * stride[side], n, N, row < left);
            }
          }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const auto op = [&](int side, int half) {
          return __builtin_bit_cast(Frag<T>, v[u][side][half]);
        };
        mma(acc[0], op(0, 0), op(1, 0));  // rows s, columns t
        mma(acc[1], op(0, 0), op(1, 1));
        mma(acc[2], op(0, 1), op(1, 1));
      }
    }
    f32x4* o = a.ws_bc + ((int64_t(b) * d.groups + group) * a.chunks + chunk) * kPairs * 64 + lane;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) o[64 * i] = acc[i];
    return;
  }
  const int64_t t = int64_t(two) * 64 + lane;
  const int chunk = 2 * two + lane / 32, q = lane % 32;
  // read whether or not the stream has the token, so that its length is not waited for first
  const int64_t at = b * io.dt.batch_stride + min(t, int64_t(a.c.c.T - 1)) * io.dt.token_stride;
  float raw[kHeads], bias[kHeads], A2[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = min(job * kHeads + i, d.heads - 1);
    raw[i] = d.dt_dtype == CO_BF16 ? bf16_to_f32(static_cast<const bf16_t*>(io.dt.data)[at + h])
                                   : static_cast<const float*>(io.dt.data)[at + h];
    bias[i] = a.c.c.dt_bias ? a.c.c.dt_bias[h] : 0.f;
    A2[i] = a.c.c.A[h] * kLog2e;
  }
  if (int64_t(two) * 64 >= len) return;  // nobody reads them
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = job * kHeads + i;
    if (h >= d.heads) break;
    float dt = raw[i] + bias[i];
    if (d.dt_softplus) dt = softplus(dt);
    dt = t < len ? dt : 0.f;
    const float log_a = t < len ? fmaxf(dt * A2[i], -160.f) : 0.f;
    // 64 bits keep the differences of far sums exact
    const double cum = prefix_sum32(double(log_a));
    const double total = lane < 32 ? from_lane<31>(cum) : from_lane<63>(cum);
    float reach = fabsf(float(cum));  // steps of either sign may turn the sums round
    if (d.dt_softplus) {
      reach = fabsf(float(total));
    } else {
#pragma unroll
      for (int m = 16; m > 0; m /= 2) reach = fmaxf(reach, __shfl_xor(reach, m));
    }
    if (chunk >= a.chunks) continue;
    ChunkDecay& o = a.ws_decay[(int64_t(b) * d.heads + h) * a.chunks + chunk];
    if (q == 0) {
      o.total = float(total);
      o.reach = reach;
    }
    o.factor[q] = pow2(cum);
    o.factor[kChunk + q] = dt * pow2(reach <= kSpan ? -cum : total - cum);
    if (reach <= kSpan) continue;  // what follows is for the chunks that go far
    o.step[q] = dt;
    o.cum[q] = float(cum);
    o.cum_low[q] = float(cum - double(float(cum)));
  }
}

// FULL: outputs and final states; otherwise a segment's own sum and decay.
template <typename T, int NT, int PT, bool FULL, bool WIDE>
__global__ __launch_bounds__(kWaves * 64, !FULL && sizeof(T) == 2 ? 3 : 2) void scan_chunk_kernel(ChunkArgs a) {
  using L = Tile<T, NT, PT>;
  using F = Frag<T>;
  constexpr int Q = L::Q, V = kWide<T>;
  constexpr int NK = NT / 2;                        // depth-32 blocks of N
  constexpr int BC_ROW = L::NW / V, BC_LOADS = (Q * BC_ROW + 255) / 256;
  constexpr int X_ROW = L::PW / V, X_LOADS = Q * X_ROW / 64;
  // Terms of a float32 value as an operand: of the factors of y, of the state's sum.
  constexpr int FACTORS = sizeof(T) == 2 ? 2 : 1, TERMS = sizeof(T) == 2 ? 3 : 1;
  static_assert(NT % 2 == 0 && 256 % BC_ROW == 0 && Q * X_ROW % 64 == 0 && 64 % X_ROW == 0);
  // Two tiles where two workgroups of a CU have them: the next chunk's is written over this one's
  // products, and a chunk has one barrier.
  constexpr int BUFS = FULL && 2 * sizeof(L) <= 80 * 1024 ? 2 : 1;
  __shared__ __align__(16) unsigned char lds[BUFS * sizeof(L)];

  const co_scan_desc& d = a.c.d;
  const co_scan_call& io = a.c.c;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g16 = lane / 16, l16 = lane % 16;
  const int per_group = d.heads / d.groups;
  const int P = d.head_dim, N = d.state_size;

  // Workgroups go to the 8 XCDs in turn.  In long segments those that read the same B and C go to
  // one, whose L2 then has them (16 ragged prompts of 24 heads 72.7 -> 69.9 us, 16384 tokens of 64
  // heads 205 either way); in segments of 8 chunks that is slower (1000 tokens 42 -> 50 us).
  const uint32_t eighth = gridDim.x / 8;
  const bool together = gridDim.x % 8 == 0 && a.seg_chunks >= 16;
  const uint32_t place = together ? blockIdx.x % 8 * eighth + blockIdx.x / 8 : blockIdx.x;
  const int ub = int(place % uint32_t(a.unit_blocks));
  int rest = int(place / uint32_t(a.unit_blocks));
  const int group = rest % d.groups;
  rest /= d.groups;
  const int seg = rest % a.segments, b = rest / a.segments;

  if (!FULL && seg == a.segments - 1) return;  // nothing begins after it
  const int unit = ub * kWaves + wave;
  const bool on = unit < per_group * a.p_blocks;    // a wave without a unit only helps
  const int h = group * per_group + (on ? unit / a.p_blocks : 0);
  const int p0 = on ? unit % a.p_blocks * L::PW : 0;
  const int width = on ? min(P - p0, L::PW) : 0;    // its rows of the head
  const int64_t bh = int64_t(b) * d.heads + h;

  const int len = stream_tokens(a.c.c.lengths, b, a.c.c.T);
  const int64_t t_begin = int64_t(seg) * a.seg_chunks * Q;
  const int64_t t_stop = min(int64_t(a.c.c.T), t_begin + int64_t(a.seg_chunks) * Q);
  const int64_t t_end = min(int64_t(len), t_stop);

  const T* xg = static_cast<const T*>(io.x.data) + b * io.x.batch_stride + int64_t(h) * P + p0;
  const T* bg = static_cast<const T*>(io.b.data) + b * io.b.batch_stride + int64_t(group) * N;
  const T* cg = static_cast<const T*>(io.c.data) + b * io.c.batch_stride + int64_t(group) * N;
  T* yg = static_cast<T*>(io.y.data) + b * io.y.batch_stride + int64_t(h) * P + p0;

  // Row r of a unit's tile pt: with two tiles a lane's 4 + 4 result rows are neighbours.
  const auto p_of = [](int pt, int r) { return PT == 2 ? 8 * (r / 4) + 4 * pt + r % 4 : r; };
  const auto x_four = [&](int pt) { return PT == 2 ? 8 * (lane % 4) + 4 * pt : 4 * (lane % 4); };

  // S^T: rows n = 16 nt + 4 g16 + i, columns p = p_of(pt, l16)
  f32x4 S[NT][PT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) S[nt][pt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto scale_state = [&](float by) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) S[nt][pt] *= by;
  };
  const auto each_state = [&](float* base, auto&& use) {
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
      const int p = p_of(pt, l16);
      if (p >= width) continue;
      float* row = base + int64_t(p) * N;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int n = 16 * nt + 4 * g16;
        if (WIDE) {
          if (n < N) use(*reinterpret_cast<f32x4*>(row + n), S[nt][pt]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (n + i < N) {
              float s = S[nt][pt][i];
              use(row[n + i], s);
              S[nt][pt][i] = s;
            }
        }
      }
    }
  };
  float* first = nullptr;
  if (FULL) {
    if (a.segments > 1)
      first = a.ws_state + ((bh * a.segments + seg) * P + p0) * N;
    else if (a.c.c.state)
      first = a.c.c.state + (bh * P + p0) * N;
  }
  if (first) each_state(first, [](auto& mem, auto& s) { s = mem; });

  const float D = a.c.c.D ? a.c.c.D[h] : 0.f;
  const int64_t chunk0 = int64_t(seg) * a.seg_chunks;
  const ChunkDecay* decay = a.ws_decay + bh * a.chunks + chunk0;
  const f32x4* bc_at =
      a.ws_bc + ((int64_t(b) * d.groups + group) * a.chunks + chunk0) * kPairs * 64;

  // The next chunk on its way from memory.  A thread's pieces of B and C lie 256 / BC_ROW tokens
  // apart, a lane's of x 64 / X_ROW.
  Pack<T, V> rb[BC_LOADS], rc[FULL ? BC_LOADS : 1], rx[X_LOADS];
  f32x4 rbc;
  float rdecay, rtotal, rreach;
  constexpr int BC_BY = 256 / BC_ROW, X_BY = 64 / X_ROW;
  const int bc_row = tid / BC_ROW, bc_col = tid % BC_ROW * V;
  const int x_row = lane / X_ROW, x_col = lane % X_ROW * V;
  // this thread's places in a chunk: bytes from its first token, or out of range
  const int es = sizeof(T);
  const int bc_off = bc_col < N ? (bc_row * int(io.b.token_stride) + bc_col) * es : kOutOfRange;
  const int c_off = bc_col < N ? (bc_row * int(io.c.token_stride) + bc_col) * es : kOutOfRange;
  const int x_off = x_col < width ? (x_row * int(io.x.token_stride) + x_col) * es : kOutOfRange;
  const T* b_at = bg + t_begin * io.b.token_stride;
  const T* c_at = cg + t_begin * io.c.token_stride;
  const T* x_at = xg + t_begin * io.x.token_stride;
  const auto fetch = [&](int64_t t0) {
    const int left = int(min(t_end - t0, int64_t(Q)));
    const __amdgpu_buffer_rsrc_t br = make_rsrc(b_at, kOutOfRange), cr = make_rsrc(c_at, kOutOfRange),
                                 xr = make_rsrc(x_at, kOutOfRange);
#pragma unroll
    for (int i = 0; i < BC_LOADS; ++i) {
      const int row = bc_row + i * BC_BY;
      if (WIDE) {
        const bool in = row < left;
        rb[i] = load_pack_at<T>(br, in ? bc_off : kOutOfRange, i * BC_BY * int(io.b.token_stride) * es);
        if (FULL)
          rc[i] = load_pack_at<T>(cr, in ? c_off : kOutOfRange, i * BC_BY * int(io.c.token_stride) * es);
      } else {
        rb[i] = load_row<T>(b_at + row * io.b.token_stride, bc_col, N, row < left);
        if (FULL) rc[i] = load_row<T>(c_at + row * io.c.token_stride, bc_col, N, row < left);
      }
    }
#pragma unroll
    for (int i = 0; i < X_LOADS; ++i) {
      const int row = x_row + i * X_BY;
      if (WIDE)
        rx[i] = load_pack_at<T>(xr, row < left ? x_off : kOutOfRange,
                                i * X_BY * int(io.x.token_stride) * es);
      else
        rx[i] = load_row<T>(x_at + row * io.x.token_stride, x_col, width, row < left);
    }
    if (FULL) rbc = bc_at[min(tid, kPairs * 64 - 1)];
    const ChunkDecay& c = decay[(t0 - t_begin) / Q];
    rdecay = c.factor[lane];
    rtotal = c.total;
    rreach = c.reach;
    b_at += Q * io.b.token_stride;
    c_at += Q * io.c.token_stride;
    x_at += Q * io.x.token_stride;
    bc_at += kPairs * 64;
  };

  // The accumulators hold the state times 2^-base: a chunk whose decays stay within kSpan of the
  // base neither scales them nor takes a power for each pair of its tokens.
  double base = 0.0, seg_log = 0.0;
  float rescale = 1.f, total = 0.f;  // of the accumulators before the chunk; its log decay
  bool far = false;                  // its decays alone pass the span
  const auto stage = [&](L& sh) {
#pragma unroll
    for (int i = 0; i < BC_LOADS; ++i) {
      const int row = bc_row + i * BC_BY;
      if (Q % BC_BY && row >= Q) break;
      store_pack<T, V>(sh.b + row * L::BS + bc_col, rb[i]);
      if (FULL) store_pack<T, V>(sh.c + row * L::CS + bc_col, rc[i]);
    }
#pragma unroll
    for (int i = 0; i < X_LOADS; ++i)
      store_pack<T, V>(sh.x[wave] + (x_row + i * X_BY) * L::XS + x_col, rx[i]);
    if (FULL && wave < kPairs) sh.bc[wave][lane] = rbc;
    total = uniform(rtotal);
    const float reach = uniform(rreach);
    far = !(reach <= kSpan);
    const bool fits = !far && fabs(base) + reach <= kSpan;
    rescale = fits ? 1.f : pow2(base);
    if (!fits) base = 0.0;
    (lane < Q ? sh.grow[wave] : sh.weight[wave])[lane % Q] =
        rdecay * pow2(lane < Q ? base : -base);
    base = far ? 0.0 : base + total;
    seg_log += total;
  };
  if (t_begin < t_end) fetch(t_begin);
  if (BUFS == 2 && t_begin < t_end) {
    stage(*reinterpret_cast<L*>(lds));
    if (t_begin + Q < t_end) fetch(t_begin + Q);
  }
  int buf = 0;
  // Of two workgroups of a CU the older one's waves go first: it was done after 85 us of 105, and
  // the younger one ran its last chunks alone.  So in long segments the younger, of the grid's
  // second half, goes first over half of its chunks, and both end together (16384 tokens of 64
  // heads of 64 x 128, all launches: 215 -> 205 us; in segments of 8 chunks no faster).
  const int64_t t_even = a.seg_chunks >= 16 && blockIdx.x >= gridDim.x / 2
                             ? t_begin + (t_end - t_begin) / (2 * Q) * Q
                             : t_begin;
  if (t_even > t_begin) __builtin_amdgcn_s_setprio(1);
  for (int64_t t0 = t_begin; t0 < t_end; t0 += Q) {
    if (t0 == t_even) __builtin_amdgcn_s_setprio(0);
    L& sh = *reinterpret_cast<L*>(lds + buf);
    if (BUFS == 1) {
      __syncthreads();  // the last chunk's tiles are read
      stage(sh);
      if (t0 + Q < t_end) fetch(t0 + Q);  // in flight over this one's products
    }
    __syncthreads();
    if (rescale != 1.f) scale_state(rescale);

    F x[PT];
#pragma unroll
    for (int pt = 0; pt < PT; ++pt)
      x[pt] = cols_of(sh.x[wave], L::XS, 0, x_four(pt), p_of(pt, l16));
    if constexpr (FULL) {
      float grow[L::QT];
#pragma unroll
      for (int j = 0; j < L::QT; ++j) grow[j] = sh.grow[wave][16 * j + l16];
      // the chunk's own tokens: e^{cum_t - cum_s} d_s, but for what y is scaled by in the end
      f32x4 w[kPairs];
      w[0] = w[1] = *reinterpret_cast<const f32x4*>(&sh.weight[wave][4 * g16]);
      w[2] = *reinterpret_cast<const f32x4*>(&sh.weight[wave][16 + 4 * g16]);
      if (far) {
        const ChunkDecay& c = decay[(t0 - t_begin) / Q];
#pragma unroll
        for (int j = 0; j < L::QT; ++j) {
          const float cum = c.cum[16 * j + l16], low = c.cum_low[16 * j + l16];
#pragma unroll
          for (int si = 0; si <= j; ++si) {
            const int s0 = 16 * si + 4 * g16;
            const f32x4 cs = *reinterpret_cast<const f32x4*>(&c.cum[s0]);
            const f32x4 ls = *reinterpret_cast<const f32x4*>(&c.cum_low[s0]);
            const f32x4 ds = *reinterpret_cast<const f32x4*>(&c.step[s0]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              w[j + si][i] = exp2_fast((cum - cs[i]) + (low - ls[i])) * ds[i];
          }
        }
      }
      // The product takes 0 x_s for s > t: a NaN or an infinity among x would reach the tokens
      // before it.  Where there is one the product does without it, and NaN goes to its places.
      bool odd = false;
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) odd |= not_finite(x[pt]);
      odd = __any(odd);
      F bad[PT];
      if (odd) {
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) part_finite(x[pt], bad[pt]);
      }
      F m[L::QT][FACTORS];  // columns t, depths s
#pragma unroll
      for (int j = 0; j < L::QT; ++j) {
        float v[8] = {};
#pragma unroll
        for (int si = 0; si <= j; ++si) {
          const f32x4 bc = sh.bc[j + si][lane];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[4 * si + i] = si < j || 4 * g16 + i <= l16 ? w[j + si][i] * bc[i] : 0.f;
        }
#pragma unroll
        for (int f = 0; f < FACTORS; ++f) take(m[j][f], v);
      }
      // y^T = S C_t + own: rows p, columns t
      f32x4 y[L::QT][PT];
      const auto from_state = [&] {
#pragma unroll
        for (int j = 0; j < L::QT; ++j)
#pragma unroll
          for (int pt = 0; pt < PT; ++pt) y[j][pt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          F c[L::QT];
#pragma unroll
          for (int j = 0; j < L::QT; ++j) c[j] = rows_of<T>(sh.c, L::CS, 16 * j, 32 * k);
#pragma unroll
          for (int pt = 0; pt < PT; ++pt) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = S[2 * k + i / 4][pt][i % 4];
#pragma unroll
            for (int f = 0; f < FACTORS; ++f) {
              F s;
              take(s, v);
#pragma unroll
              for (int j = 0; j < L::QT; ++j) mma(y[j][pt], s, c[j]);
            }
          }
        }
      };
      const auto from_own = [&] {
#pragma unroll
        for (int j = 0; j < L::QT; ++j)
#pragma unroll
          for (int pt = 0; pt < PT; ++pt)
#pragma unroll
            for (int f = 0; f < FACTORS; ++f) mma(y[j][pt], x[pt], m[j][f]);
      };
      from_state();
      if (far) {
#pragma unroll
        for (int j = 0; j < L::QT; ++j) {
#pragma unroll
          for (int pt = 0; pt < PT; ++pt) y[j][pt] *= grow[j];
          grow[j] = 1.f;
        }
        scale_state(pow2(double(total)));
      }
      from_own();
      if (odd) {
#pragma unroll
        for (int j = 0; j < L::QT; ++j) {
          float one[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            one[i] = i / 4 < j || (i / 4 == j && 4 * g16 + i % 4 <= l16) ? 1.f : 0.f;
          F ones;
          round_to(ones, one);
#pragma unroll
          for (int pt = 0; pt < PT; ++pt) {
            f32x4 count{0.f, 0.f, 0.f, 0.f};
            mma(count, bad[pt], ones);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (count[i] > 0.f) y[j][pt][i] = __builtin_nanf("");
          }
        }
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
          x[pt] = cols_of(sh.x[wave], L::XS, 0, x_four(pt), p_of(pt, l16));
      }
      const __amdgpu_buffer_rsrc_t yr = make_rsrc(yg + t0 * io.y.token_stride, kOutOfRange);
      // tokens of the call, and of the stream: past those the sums may be 0 times what is not finite
      const int rows_left = int(min(t_stop - t0, int64_t(Q)));
      const int rows_own = int(min(t_end - t0, int64_t(Q)));
#pragma unroll
      for (int j = 0; j < L::QT; ++j) {
        const int r = 16 * j + l16;
        const T* xr = sh.x[wave] + r * L::XS;
        constexpr int RUN = PT * 4;  // neighbours of this lane
        const int p = RUN * g16;
        float out[RUN];
#pragma unroll
        for (int i = 0; i < RUN; ++i)
          out[i] = fmaf(D, to_f32<T>(xr[p + i]), y[j][i / 4][i % 4] * grow[j]);
        if (rows_own < Q) {  // the stream ends here
#pragma unroll
          for (int i = 0; i < RUN; ++i) out[i] = r < rows_own ? out[i] : 0.f;
        }
        if (WIDE) {
          constexpr int W = RUN < V ? RUN : V;
#pragma unroll
          for (int q = 0; q < RUN; q += W) {
            Pack<T, W> o;
#pragma unroll
            for (int i = 0; i < W; ++i) o.v[i] = from_f32<T>(out[q + i]);
            const bool in = r < rows_left && p + q < width;
            store_pack_at<T, W>(yr, in ? (r * int(io.y.token_stride) + p + q) * es : kOutOfRange, o);
          }
        } else {
          T* row = yg + (t0 + r) * io.y.token_stride;
#pragma unroll
          for (int i = 0; i < RUN; ++i)
            if (r < rows_left && p + i < width) row[p + i] = from_f32<T>(out[i]);
        }
      }
    } else {
      if (far) scale_state(pow2(double(total)));
    }

    // S' = e^{cum_Q} S + B^T (weighted x)
    F xw[PT][TERMS];
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
      float left[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        left[i] = get(x[pt], i) * sh.weight[wave][16 * (i / 4) + 4 * g16 + i % 4];
#pragma unroll
      for (int term = 0; term < TERMS; ++term) take(xw[pt][term], left);
    }
    buf = BUFS == 2 ? int(sizeof(L)) - buf : 0;
    if (BUFS == 2 && t0 + Q < t_end) {  // over the products below
      stage(*reinterpret_cast<L*>(lds + buf));
      if (t0 + 2 * Q < t_end) fetch(t0 + 2 * Q);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const F bt = cols_of(sh.b, L::BS, 0, 16 * nt + 4 * (lane % 4), 16 * nt + l16);
#pragma unroll
      for (int pt = 0; pt < PT; ++pt)
#pragma unroll
        for (int term = TERMS - 1; term >= 0; --term) mma(S[nt][pt], bt, xw[pt][term]);
    }
  }
  if (base != 0.0) scale_state(pow2(base));

  if (FULL) {
    // tokens past the stream's
    const int64_t from = t_begin < t_end ? t_begin + (t_end - t_begin + Q - 1) / Q * Q : t_begin;
    for (int64_t t = from + lane / 16; t < t_stop; t += 4)
      for (int p = l16; p < width; p += 16) yg[t * io.y.token_stride + p] = T{};
    if (a.c.c.state && a.c.c.update_state && seg == a.segments - 1 && len > 0)
      each_state(a.c.c.state + (bh * P + p0) * N, [](auto& mem, auto& s) { mem = s; });
  } else {
    each_state(a.ws_state + ((bh * a.segments + seg) * P + p0) * N,
               [](auto& mem, auto& s) { mem = s; });
    if (on && p0 == 0 && lane == 0) a.ws_total[bh * a.segments + seg] = float(seg_log);
  }
}

// Turns the segments' sums into the states that they begin with, V values a thread.
template <int V>
__global__ __launch_bounds__(kBlock) void scan_carry_kernel(ChunkArgs a, uint32_t head_blocks) {
  using P = Pack<float, V>;
  const int64_t size = int64_t(a.c.d.head_dim) * a.c.d.state_size;
  const int64_t bh = blockIdx.x / head_blocks;
  const int64_t i = (int64_t(blockIdx.x % head_blocks) * kBlock + threadIdx.x) * V;
  if (i >= size) return;
  float* w = a.ws_state + bh * a.segments * size + i;
  const float* total = a.ws_total + bh * a.segments;
  P s{};
  if (a.c.c.state) s = load_pack<float, V>(a.c.c.state + bh * size + i);
  const int last = a.segments - 1;
  constexpr int AHEAD = 8;  // loads in flight
  for (int k0 = 0; k0 < last; k0 += AHEAD) {
    P sum[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (k0 + u < last) sum[u] = load_pack<float, V>(w + (k0 + u) * size);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (k0 + u < last) {
        store_pack<float, V>(w + (k0 + u) * size, s);
        const float decay = exp2_fast(total[k0 + u]);
#pragma unroll
        for (int v = 0; v < V; ++v) s.v[v] = fmaf(decay, s.v[v], sum[u].v[v]);
      }
  }
  store_pack<float, V>(w + last * size, s);
}

// The launch before the chunks has prepare_doubles x prepare_jobs workgroups, the carry
// carry_blocks a head, V values a thread.
int64_t prepare_doubles(const co_scan_desc& d, int64_t chunks) { return (chunks + 1) / 2 * d.batch; }
int64_t prepare_jobs(const co_scan_desc& d) {
  const int64_t waves = (int64_t(d.heads) + kHeads - 1) / kHeads + 2 * int64_t(d.groups);
  return (waves + kBlock / 64 - 1) / (kBlock / 64);
}
int64_t carry_blocks(const co_scan_desc& d, int64_t V) {
  return (int64_t(d.head_dim) * d.state_size + V * kBlock - 1) / (V * kBlock);
}

// Workgroups of an uncut call with units of so many rows.
int64_t workgroups(const co_scan_desc& d, int64_t rows) {
  const int64_t units = int64_t(d.heads / d.groups) * ((d.head_dim + rows - 1) / rows);
  return (units + kWaves - 1) / kWaves * d.groups * d.batch;
}

// Rows of a unit.  32 share the most between them: 64 heads of 64 x 128 in bfloat16, 16000 tokens
// 202 us with 32 and 303 us with 16.  16 where 256 states take a lane's registers, where a fifth
// or more of the waves' rows would be empty with 32 and are not with 16 (heads of 40 rows; groups
// of three heads of 64: 16 streams of 1000 tokens of 24 such heads x 64 states 83 and 80 us, of
// ragged ones 80 and 70; 64 streams of 500 of 8 groups of one head x 128 87 and 73), and where a
// call has too few units to fill the card however it is cut: its time is then that of one wave's
// chunks, which are shorter (256 tokens 33 and 26 us; 3 streams of 10 heads of 40 x 20, float32,
// 256 tokens 29 and 22 us).
int unit_rows(const co_scan_desc& d, int64_t T) {
  if (d.state_size > 128) return 16;
  if (2 * workgroups(d, 32) * 4 >= 5 * workgroups(d, 16)) return 16;
  const int64_t chunks = (T + kChunk - 1) / kChunk;
  return workgroups(d, 32) * ((chunks + 3) / 4) < 600 ? 16 : 32;
}

template <typename T, int NT, int PT, bool WIDE>
hipError_t launch_tiles(ChunkArgs a, hipStream_t s) {
  const co_scan_desc& d = a.c.d;
  a.p_blocks = int32_t((int64_t(d.head_dim) + 16 * PT - 1) / (16 * PT));
  const int64_t units = int64_t(d.heads / d.groups) * a.p_blocks;
  a.unit_blocks = int32_t((units + kWaves - 1) / kWaves);
  const int64_t grid = int64_t(a.unit_blocks) * d.groups * d.batch;
  const int64_t jobs = prepare_jobs(d), doubles = prepare_doubles(d, a.chunks);
  constexpr int CV = WIDE ? 4 : 1;  // a state row is then whole pieces of 16 bytes
  const int64_t head_blocks = carry_blocks(d, CV);
  hipLaunchKernelGGL((scan_prepare_kernel<T, WIDE>), dim3(unsigned(doubles), unsigned(jobs)),
                     dim3(kBlock), 0, s, a);
  if (a.segments > 1) {
    hipLaunchKernelGGL((scan_chunk_kernel<T, NT, PT, false, WIDE>),
                       dim3(unsigned(grid * a.segments)), dim3(kWaves * 64), 0, s, a);
    hipLaunchKernelGGL(scan_carry_kernel<CV>, dim3(unsigned(head_blocks * d.batch * d.heads)),
                       dim3(kBlock), 0, s, a, uint32_t(head_blocks));
  }
  hipLaunchKernelGGL((scan_chunk_kernel<T, NT, PT, true, WIDE>), dim3(unsigned(grid * a.segments)),
                     dim3(kWaves * 64), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool WIDE>
hipError_t launch_state(const ChunkArgs& a, hipStream_t s) {
  const int N = a.c.d.state_size;
  if (unit_rows(a.c.d, a.c.c.T) == 32) {
    if (N <= 32) return launch_tiles<T, 2, 2, WIDE>(a, s);
    if (N <= 64) return launch_tiles<T, 4, 2, WIDE>(a, s);
    return launch_tiles<T, 8, 2, WIDE>(a, s);
  }
  if (N <= 32) return launch_tiles<T, 2, 1, WIDE>(a, s);
  if (N <= 64) return launch_tiles<T, 4, 1, WIDE>(a, s);
  if (N <= 128) return launch_tiles<T, 8, 1, WIDE>(a, s);
  return launch_tiles<T, 16, 1, WIDE>(a, s);
}

template <typename T>
hipError_t launch_t(const ChunkArgs& a, hipStream_t s) {
  constexpr int V = kWide<T>;
  const auto wide = [](const co_tokens& t) {
    return reinterpret_cast<uintptr_t>(t.data) % 16 == 0 && t.batch_stride % V == 0 &&
           t.token_stride % V == 0 && t.token_stride < (1 << 22);
  };
  const co_scan_call& io = a.c.c;
  // 16-byte accesses where every one of them is aligned and a chunk's offsets take 31 bits, values
  // otherwise
  const bool fits = a.c.d.head_dim % V == 0 && a.c.d.state_size % V == 0 && wide(io.x) &&
                    wide(io.b) && wide(io.c) && wide(io.y) &&
                    reinterpret_cast<uintptr_t>(a.c.c.state) % 16 == 0 &&
                    reinterpret_cast<uintptr_t>(a.ws_state) % 16 == 0;
  return fits ? launch_state<T, true>(a, s) : launch_state<T, false>(a, s);
}

// Segments of a call over T tokens, and their chunks: the cut that is estimated to be fastest.
// In units of a chunk's time in a workgroup that has its CU alone, two on a CU take 1.5 (64 heads
// of 64 x 128, bfloat16: 3.0 and 4.8 us); a segment's own sum takes about half of the whole (70 of
// 155 us, 89 of 194), and carrying the states a launch and their bytes.  Chunks of other tiles and
// types take other times, beside which the last two weigh more or less: the cut was measured for
// 64 x 128 and 64 x 64 in bfloat16.  16 ragged prompts of 24 heads of 64 x 64, 32 chunks, 70 us
// uncut, 73 in two segments and 76 in three (with units of 32 rows 80 and 85); 16384 tokens of 64
// heads of 64 x 128 in 8, 16 and 24 segments 279, 206 and 234.
void cut(const co_scan_desc& d, int64_t T, int64_t* segments, int64_t* seg_chunks) {
  const int64_t chunks = (T + kChunk - 1) / kChunk;
  const int64_t groups = workgroups(d, unit_rows(d, T));
  const double states = double(d.batch) * d.heads * d.head_dim * d.state_size;
  const auto cost = [&](int64_t n) {
    const double wgs = double(groups) * double(n);
    const double load = wgs <= 256 ? 1.0 : wgs <= 512 ? 1.5 : 1.5 * wgs / 512;
    const double pass = load * double((chunks + n - 1) / n);
    return n == 1 ? pass : 1.55 * pass + 2.0 + states * double(n) * 8 / 12e6;
  };
  int64_t best = 1;
  for (int64_t n = 2; n <= chunks / 4 && n <= 64; n += n < 8 ? 1 : n < 16 ? 2 : 8)
    if (cost(n) < cost(best)) best = n;
  *seg_chunks = (chunks + best - 1) / best;
  *segments = (chunks + *seg_chunks - 1) / *seg_chunks;
}

// Where each part of the workspace lies, in bytes (all multiples of 16 but the last).
struct Space {
  int64_t decay, state, total, bytes;
};
Space space_of(const co_scan_desc& d, int64_t chunks, int64_t segments) {
  const int64_t bh = int64_t(d.batch) * d.heads;
  Space s;
  s.decay = int64_t(d.batch) * d.groups * chunks * kPairs * 64 * int64_t(sizeof(f32x4));
  s.state = s.decay + bh * chunks * int64_t(sizeof(ChunkDecay));
  s.total = s.state + (segments > 1 ? bh * segments * d.head_dim * d.state_size * 4 : 0);
  s.bytes = s.total + (segments > 1 ? bh * segments * 4 : 0);
  return s;
}

}  // namespace

// Token by token a call takes about 0.3 us a token and 0.11 us a million state values and token;
// chunks take 9 us more to begin with, and 0.3 us a million values.  Measured, us, by token and in
// chunks: 16.8 million values, 4 tokens 29 and 37, 8 tokens 38 and 37, 32 tokens 97 and 39;
// 0.5 million, 16 tokens 10 and 12, 32 tokens 17 and 12.
//
// Calls whose chunks would pass what a launch may have of workgroups go token by token.
bool scan_chunk_takes(const co_scan_desc& d, int32_t T) {
  const double millions = 1e-6 * d.batch * d.heads * double(d.head_dim) * d.state_size;
  if (!(T * (0.3 + 0.11 * millions) > 9.0 + 0.3 * millions)) return false;
  int64_t segments, seg_chunks;
  cut(d, T, &segments, &seg_chunks);
  const int64_t chunks = (int64_t(T) + kChunk - 1) / kChunk, jobs = prepare_jobs(d);
  return grid_fits(workgroups(d, unit_rows(d, T)) * segments) && jobs <= 65535 &&
         grid_fits(prepare_doubles(d, chunks) * jobs) &&
         grid_fits(carry_blocks(d, 1) * d.batch * d.heads);
}

int64_t scan_chunk_workspace(const co_scan_desc& d, int32_t T) {
  int64_t segments, seg_chunks;
  cut(d, T, &segments, &seg_chunks);
  return space_of(d, (int64_t(T) + kChunk - 1) / kChunk, segments).bytes;
}

hipError_t launch_scan_chunk(const ScanCall& c, hipStream_t stream) {
  int64_t segments, seg_chunks;
  cut(c.d, c.c.T, &segments, &seg_chunks);
  const int64_t chunks = (int64_t(c.c.T) + kChunk - 1) / kChunk;
  const Space at = space_of(c.d, chunks, segments);
  char* w = static_cast<char*>(c.c.workspace);
  ChunkArgs a{};
  a.c = c;
  a.ws_bc = reinterpret_cast<f32x4*>(w);
  a.ws_decay = reinterpret_cast<ChunkDecay*>(w + at.decay);
  a.ws_state = reinterpret_cast<float*>(w + at.state);
  a.ws_total = reinterpret_cast<float*>(w + at.total);
  a.chunks = int32_t(chunks);
  a.segments = int32_t(segments);
  a.seg_chunks = int32_t(seg_chunks);
  if (c.d.dtype == CO_BF16) return launch_t<bf16_t>(a, stream);
  return launch_t<float>(a, stream);
}

}  // namespace coinf
