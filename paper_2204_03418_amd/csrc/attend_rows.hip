// Attention of many rows (tokens times the query heads of a kv head) over the cache:
// a workgroup 128 rows, a wave 32, all of them over the same keys, one pass with the
// running maximum and sum of the softmax.
//
// Scores come transposed, S^T = K Q^T, so that a lane has one row's scores (32 x 32
// tiles: column = row of queries), and the weights are the operand of O^T = V^T P^T without
// leaving their lanes.  The first product takes the cache's codes as they are: matrix
// instructions with a scale a block of 32 channels read 4-bit keys against queries in
// 8-bit terms, which hold them exactly, at the rate of 16-bit products (two terms);
// LDS holds and moves a quarter of the bytes.  Values become 16-bit floats in LDS, once a
// workgroup (exactly, but for what is below 2^-35 of its tile's largest scale), and the
// weights 16-bit floats with 11 bits (two terms, 22 bits, for float32).
#include "attend.hpp"

namespace coinf {

namespace {

template <typename T, int NB>
struct Rows {
  static constexpr int QT = kQueryTerms<T>, PT = kWeightTerms<T>;
  static constexpr bool EVEN = NB % 2 == 0;
  static constexpr int MMA = QT * NB / 2;              // of a 32 x 32 tile of scores, depth 64
  static constexpr int FRAGS = EVEN ? NB / 2 : NB;     // of keys
  static constexpr int CHUNKS = NB * kKeys;            // 16 bytes of codes of a tile
  static constexpr int PER = (CHUNKS + kBlock - 1) / kBlock;
  static constexpr int WORDS = (CHUNKS / 4 + 63) / 64;  // of scales a lane
  static constexpr int VS = NB * 32 + 32;              // rows 64 bytes apart modulo the banks
  // term and block of the half h of instruction j
  static __device__ int term(int j, int h) { return EVEN ? 2 * j / NB : 2 * (j / NB) + h; }
  static __device__ int block(int j, int h) { return EVEN ? 2 * j % NB + h : j % NB; }
};

template <typename T, int NB>
struct RowsLds {
  using R = Rows<T, NB>;
  alignas(16) uint8_t k[2][R::CHUNKS * 16];
  alignas(16) _Float16 v[2][kKeys * R::VS];
  uint32_t ks[2][R::CHUNKS / 4], vs[2][R::CHUNKS / 4];
  int32_t pages[2];  // bit i: 16 tokens i have a page
  int32_t bad[2];    // the tile, where a value is not finite
};

template <typename T, int NB>
__global__ __launch_bounds__(kBlock, NB <= 4 ? 2 : 1) void attend_rows_kernel(AttendArgs a) {
  using R = Rows<T, NB>;
  __shared__ RowsLds<T, NB> s;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, col = lane % 32, half = lane / 32;

  // which unit: all parts and row tiles of a pair on one XCD where the pairs allow it, the rows
  // that see most first
  int u = blockIdx.x;
  int pair, rt, split;
  if (a.pairs % 8 == 0) {
    const int xcd = u % 8, k = u / 8, px = a.pairs / 8;
    const int rest = k / px;
    pair = (k - rest * px) * 8 + xcd;
    rt = fdiv(rest, a.by_splits);
    split = rest - rt * a.splits;
  } else {
    const int rest = u / a.pairs;
    pair = u - rest * a.pairs;
    rt = fdiv(rest, a.by_splits);
    split = rest - rt * a.splits;
  }
  rt = a.row_tiles - 1 - rt;
  const int b = fdiv(pair, a.by_kv), kv = pair - b * a.d.kv_heads;
  const Span span(a, b);
  const int rows = span.n * a.group, row0 = rt * kRows;

  const int row = row0 + wave * 32 + col;
  const int t = fdiv(row, a.by_group), head = kv * a.group + row - t * a.group;
  // of tokens that the stream does not have
  const auto no_output = [&] {
    if (t >= a.T) return;
    T* y = static_cast<T*>(a.y.data) + b * a.y.batch_stride + t * a.y.token_stride +
           int64_t(head) * a.d.head_dim;
    const float none[4] = {};
    for (int c = 4 * half; c < a.d.head_dim; c += 8) store4<T>(y, c, a.d.head_dim, a.wide, none);
  };
  if (row0 >= rows) {
    if (split == 0) no_output();
    return;
  }
  const int t_last = fdiv(min(row0 + kRows, rows) - 1, a.by_group);
  const Part part(span.lo(a, fdiv(row0, a.by_group)), span.base + t_last + 1, a.splits, split);
  if (split >= part.parts) return;

  // queries, as 8-bit terms
  const bool live = row < rows;
  const T* q = static_cast<const T*>(a.q.data) + b * a.q.batch_stride +
               int64_t(live ? t : 0) * a.q.token_stride + int64_t(live ? head : 0) * a.d.head_dim;
  i32x8 qo[R::MMA];
  int qs[R::MMA];
  bool q_bad = false;
#pragma unroll
  for (int blk = 0; blk < NB; ++blk) {
    float v[16];
#pragma unroll
    for (int w = 0; w < 4; ++w)
      load4<T>(q, live ? blk * 32 + 16 * half + 4 * w : a.d.head_dim, a.d.head_dim, a.wide, v + 4 * w);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[i] *= a.q_sign;
      most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
    }
    most = max(most, uint32_t(__shfl_xor(int(most), 32)));
    const bool bad = most >= 0x7f800000u;
    q_bad |= bad;
    const int byte = bad ? 127 : query_scale(most);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = bad ? 0.f : v[i];
    i32x4 words[R::QT];
    to_terms<R::QT>(v, byte, words);
#pragma unroll
    for (int j = 0; j < R::MMA; ++j) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (R::block(j, h) != blk) continue;
        const i32x4 w = words[R::term(j, h)];
#pragma unroll
        for (int i = 0; i < 4; ++i) qo[j][4 * h + i] = w[i];
        if (h == half) qs[j] = byte - 4 * R::term(j, h);
      }
    }
  }

  // one thread's 16 bytes of keys and of values of a tile, on their way
  const char* pool = static_cast<const char*>(a.c.pool) + int64_t(kv) * a.lay.bytes();
  const int32_t* table = a.c.table + int64_t(b) * a.d.stream_pages;
  const int tile_bytes = NB * 256;
  i32x4 rk[R::PER], rv[R::PER];
  uint32_t rks[R::WORDS], rvs[R::WORDS];
  int page[R::PER], page_w[R::WORDS];
  // the pages of a tile's chunks and words of scales
  const auto page_of = [&](int tile, int sub) {
    const int64_t pos = int64_t(tile) * kKeys + sub * kCacheTile;
    const int lp = int(pos >> a.page_shift);
    const int p = table[lp - fdiv(lp, a.by_W) * a.d.stream_pages];
    return p >= 0 && p < a.d.pages ? p : -1;
  };
  const auto fetch_pages = [&](int tile) {
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
      const int c = tid + i * kBlock;
      page[i] = c < R::CHUNKS ? page_of(tile, c / (NB * 16)) : -1;
    }
#pragma unroll
    for (int i = 0; i < R::WORDS; ++i) {
      const int w = lane + 64 * i;
      page_w[i] = w < R::CHUNKS / 4 ? page_of(tile, w / (NB * 4)) : -1;
    }
  };
  const auto fetch = [&](int tile) {
    const int in = int(int64_t(tile) * kKeys & (a.lay.P - 1)) / kCacheTile;  // of a page's tiles
    const int sub_mask = a.lay.P / kCacheTile - 1;
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
      const int c = tid + i * kBlock, sub = c / (NB * 16), rest = c - sub * NB * 16;
      rk[i] = rv[i] = i32x4{0, 0, 0, 0};
      if (page[i] >= 0) {
        const char* p = pool + page[i] * a.page_bytes + ((in + sub) & sub_mask) * tile_bytes +
                        rest * 16;
        rk[i] = *reinterpret_cast<const i32x4*>(p);
        rv[i] = *reinterpret_cast<const i32x4*>(p + a.lay.codes(1));
      }
    }
#pragma unroll
    for (int i = 0; i < R::WORDS; ++i) {
      const int w = lane + 64 * i, sub = w / (NB * 4), rest = w - sub * NB * 4;
      rks[i] = rvs[i] = 0;
      if (page_w[i] >= 0) {
        const char* p = pool + page_w[i] * a.page_bytes + ((in + sub) & sub_mask) * NB * 16 +
                        rest * 4;
        if (wave == 0) rks[i] = *reinterpret_cast<const uint32_t*>(p + a.lay.scales(0));
        rvs[i] = *reinterpret_cast<const uint32_t*>(p + a.lay.scales(1));
      }
    }
  };

  const int64_t hi = span.base + span.n;
  f32x16 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x16{};
  float m = -1e30f, l = 0.f;  // the row's reference score, and its sum
  int E = 0;                  // the values' exponent, 0: none yet

  // what was fetched into LDS
  const auto fill = [&](int tile, int buf) {
    const int64_t pos0 = int64_t(tile) * kKeys;
    // keys of the stream: what else a page holds may be anything
    const int from = int(min(max(span.lowest - pos0, int64_t(0)), int64_t(kKeys)));
    const int to = int(min(hi - pos0, int64_t(kKeys)));
    int top = 0;
    uint32_t bytes[R::WORDS];
#pragma unroll
    for (int i = 0; i < R::WORDS; ++i) {
      const int w = lane + 64 * i, tok = w / (NB * 4) * 16 + w % 4 * 4;
      bytes[i] = rvs[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int v = bytes[i] >> (8 * k) & 255;
        const bool on = tok + k >= from && tok + k < to && v != 255;
        top = max(top, on ? v : 0);
      }
      if (wave == 0 && w < R::CHUNKS / 4) {
        s.ks[buf][w] = rks[i];
        s.vs[buf][w] = bytes[i];
      }
    }
    if (__any(top > E)) {
#pragma unroll
      for (int k = 1; k < 64; k *= 2) top = max(top, __shfl_xor(top, k));
      const int next = __builtin_amdgcn_readfirstlane(top) + kValueSlack;
      if (E) {
        const float down = exponent_to_f32(127 + E - next);
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] *= down;
      }
      E = next;
    }
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
      const int c = tid + i * kBlock, sub = c / (NB * 16), rest = c - sub * NB * 16;
      const int tok = sub * 16 + rest % 16, blk = rest / 16;
      // the chunk's scale is byte c of the words, which all waves have
      const uint32_t word = R::WORDS == 1 || c < 256
                                ? uint32_t(__shfl(int(bytes[0]), c / 4 % 64))
                                : uint32_t(__shfl(int(bytes[R::WORDS - 1]), c / 4 % 64));
      if (c >= R::CHUNKS) break;
      const int v = word >> (8 * (c % 4)) & 255;
      *reinterpret_cast<i32x4*>(s.k[buf] + c * 16) = rk[i];
      const bool on = tok >= from && tok < to && page[i] >= 0;
      if (on && v == 255) s.bad[buf] = tile;
      const float scale = on && v != 255 ? exponent_to_f32(127 + v - E + kValueLift) : 0.f;
      _Float16* dst = s.v[buf] + tok * R::VS + blk * 32;
      f16x8 w[2];
      decode16(rv[i][0], rv[i][1], scale, w);
      *reinterpret_cast<f16x8*>(dst) = w[0];
      *reinterpret_cast<f16x8*>(dst + 8) = w[1];
      decode16(rv[i][2], rv[i][3], scale, w);
      *reinterpret_cast<f16x8*>(dst + 16) = w[0];
      *reinterpret_cast<f16x8*>(dst + 24) = w[1];
    }
    if (wave == 0) {
      // one lane of each 16 tokens' first chunk or word
      uint32_t on = 0;
#pragma unroll
      for (int i = 0; i < R::WORDS; ++i) {
        const int w = lane + 64 * i;
        if (w < R::CHUNKS / 4 && w % (NB * 4) == 0 && page_w[i] >= 0) on |= 1u << (w / (NB * 4));
      }
#pragma unroll
      for (int k = 1; k < 64; k *= 2) on |= uint32_t(__shfl_xor(int(on), k));
      if (lane == 0) s.pages[buf] = int(on);
    }
  };

  // the wave's rows: keys that some of them see
  const int wt0 = fdiv(row0 + wave * 32, a.by_group);
  const int wrows = min(row0 + wave * 32 + 32, rows);
  const int wt1 = fdiv(max(wrows, 1) - 1, a.by_group);
  const bool wave_on = row0 + wave * 32 < rows;
  const int64_t wave_lo = span.lo(a, wt0), wave_hi = span.base + wt1;   // both included
  const int64_t wave_lo_all = span.lo(a, wt1), wave_hi_all = span.base + wt0;  // that all see
  const int64_t my_lo = span.lo(a, t), my_hi = live ? span.base + t : -1;

  if (tid < 2) s.bad[tid] = -1;
  if (part.first < part.end) {
    fetch_pages(part.first);
    fetch(part.first);
    __syncthreads();  // bad
    fill(part.first, 0);
    if (part.first + 1 < part.end) fetch_pages(part.first + 1);
  }
  __syncthreads();

  for (int tile = part.first; tile < part.end; ++tile) {
    const int buf = (tile - part.first) & 1;
    const bool more = tile + 1 < part.end;
    if (more) fetch(tile + 1);
    const int64_t pos0 = int64_t(tile) * kKeys;
    if (wave_on && pos0 <= wave_hi && pos0 + kKeys > wave_lo) {
      f32x16 sc[2];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        i32x8 kf[R::FRAGS];
        int ks[R::FRAGS];
#pragma unroll
        for (int f = 0; f < R::FRAGS; ++f) {
          const int blk = R::EVEN ? 2 * f + half : f;
          const int at = ((2 * g + col / 16) * NB + blk) * 16 + col % 16;
          const i32x4 w = *reinterpret_cast<const i32x4*>(s.k[buf] + at * 16);
          kf[f] = i32x8{w[0], w[1], w[2], w[3], 0, 0, 0, 0};
          ks[f] = reinterpret_cast<const uint8_t*>(s.ks[buf])[at];
        }
        sc[g] = f32x16{};
#pragma unroll
        for (int j = 0; j < R::MMA; ++j)
          sc[g] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
              kf[j % R::FRAGS], qo[j], sc[g], 4, 0, 0, ks[j % R::FRAGS], 0, qs[j]);
      }
      const bool whole = pos0 + kKeys - 1 <= wave_hi_all && pos0 >= wave_lo_all &&
                         s.pages[buf] == 15;
      if (!whole) {
        const int pages = s.pages[buf];
        const int from = int(min(max(my_lo - pos0, int64_t(-1)), int64_t(kKeys)));
        const int to = int(min(max(my_hi - pos0, int64_t(-1)), int64_t(kKeys)));
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int k = 32 * g + 8 * (i / 4) + 4 * half + i % 4;
            const bool see = k >= from && k <= to && (pages >> (k / 16) & 1);
            sc[g][i] = see ? sc[g][i] : -__builtin_inff();
          }
      }
      float top = fmaxf(sc[0][0], sc[1][0]);
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(fmaxf(top, sc[0][i]), sc[1][i]);
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m + a.slack)) {
        const float next = fmaxf(top, m);
        const float down = exp2_fast((m - next) * a.scale_log2);
        l *= down;
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] *= down;
        m = next;
      }
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        f16x8 p[R::PT][2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          // the difference first: far scores have no digits to lose
          f32x2 w = {exp2_fast(fmaf(sc[g][i] - m, a.scale_log2, kLift)),
                     exp2_fast(fmaf(sc[g][i + 1] - m, a.scale_log2, kLift))};
#pragma unroll
          for (int k = 0; k < R::PT; ++k) {
            const f16x2 r = __builtin_convertvector(w, f16x2);
            p[k][i / 8][i % 8] = r[0];
            p[k][i / 8][i % 8 + 1] = r[1];
            // the sum of the weights as they are used
            l = __builtin_amdgcn_fdot2(r, f16x2{1, 1}, l, false);
            if (k + 1 < R::PT) w -= __builtin_convertvector(r, f32x2);
          }
        }
        const int j16 = lane % 16;
        const _Float16* base = s.v[buf] + (32 * g + 4 * half + j16 / 4) * R::VS +
                               16 * (lane / 16 % 2) + 4 * (j16 % 4);
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            struct Both {
              s16x4 lo, hi;
            } r;
            r.lo = turned4(base + 16 * d * R::VS + 32 * blk);
            r.hi = turned4(base + (16 * d + 8) * R::VS + 32 * blk);
            const f16x8 v = __builtin_bit_cast(f16x8, r);
#pragma unroll
            for (int k = 0; k < R::PT; ++k)
              o[blk] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[k][d], o[blk], 0, 0, 0);
          }
        }
      }
      if (s.bad[buf] == tile) {  // a block that is not finite, to the rows that see its token
        for (int c = 0; c < R::CHUNKS; ++c) {
          if (reinterpret_cast<const uint8_t*>(s.vs[buf])[c] != 255) continue;
          const int tok = c / (NB * 16) * 16 + c % 16, blk = c % (NB * 16) / 16;
          const int64_t pos = pos0 + tok;
          const bool see = pos >= my_lo && pos <= my_hi && (s.pages[buf] >> (tok / 16) & 1);
          const float nan = see ? __builtin_nanf("") : 0.f;
#pragma unroll
          for (int i = 0; i < NB; ++i)
            if (i == blk)
#pragma unroll
              for (int k = 0; k < 16; ++k) o[i][k] += nan;
        }
      }
    }
    if (more) {
      fill(tile + 1, buf ^ 1);
      if (tile + 2 < part.end) fetch_pages(tile + 2);
    }
    __syncthreads();
  }

  l += __shfl_xor(l, 32);
  if (!live) {
    if (split == 0) no_output();
    return;
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  // 2^{E - 127 - kValueLift} in two steps, neither out of range
  const float up = exponent_to_f32(E - kValueSlack);
  const float less = exponent_to_f32(127 + kValueSlack - kValueLift);
  const float bad = q_bad && l > 0.f ? __builtin_nanf("") : 0.f;
  const auto value = [&](int blk, int i) { return o[blk][i] * inv * less * up + bad; };
  if (part.parts == 1) {
    T* y = static_cast<T*>(a.y.data) + b * a.y.batch_stride + t * a.y.token_stride +
           int64_t(head) * a.d.head_dim;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float v[4] = {value(blk, i), value(blk, i + 1), value(blk, i + 2), value(blk, i + 3)};
        store4<T>(y, blk * 32 + 2 * i + 4 * half, a.d.head_dim, a.wide, v);
      }
    return;
  }
  const int64_t at = ((int64_t(pair) * a.row_tiles + rt) * a.splits + split) * kRows +
                     wave * 32 + col;
  float* o_part = a.part + at * (NB * 32);
#pragma unroll
  for (int blk = 0; blk < NB; ++blk)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const Pack<float, 4> v = {{value(blk, i), value(blk, i + 1), value(blk, i + 2),
                                 value(blk, i + 3)}};
      store_pack<float, 4>(o_part + blk * 32 + 2 * i + 4 * half, v);
    }
  if (half == 0) a.part_stat[at] = {m, l};
}

template <typename T>
void run(const AttendArgs& a, int NB, unsigned grid, hipStream_t s) {
  switch (NB) {
    case 1: attend_rows_kernel<T, 1><<<grid, kBlock, 0, s>>>(a); break;
    case 2: attend_rows_kernel<T, 2><<<grid, kBlock, 0, s>>>(a); break;
    case 3: attend_rows_kernel<T, 3><<<grid, kBlock, 0, s>>>(a); break;
    case 4: attend_rows_kernel<T, 4><<<grid, kBlock, 0, s>>>(a); break;
    case 5: attend_rows_kernel<T, 5><<<grid, kBlock, 0, s>>>(a); break;
    case 6: attend_rows_kernel<T, 6><<<grid, kBlock, 0, s>>>(a); break;
    case 7: attend_rows_kernel<T, 7><<<grid, kBlock, 0, s>>>(a); break;
    default: attend_rows_kernel<T, 8><<<grid, kBlock, 0, s>>>(a); break;
  }
}

}  // namespace

void launch_attend_rows(const AttendArgs& a, int NB, hipStream_t stream) {
  const unsigned grid = unsigned(int64_t(a.pairs) * a.row_tiles * a.splits);
  if (a.d.dtype == CO_BF16)
    run<bf16_t>(a, NB, grid, stream);
  else
    run<float>(a, NB, grid, stream);
}

}  // namespace coinf
