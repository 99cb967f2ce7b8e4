// Attention of many rows (tokens times the query heads of a kv head) over the cache:
// a workgroup 128 rows, a wave 32, all of them over the same keys, one pass with the
// running maximum and sum of the softmax.
//
// Scores come transposed, S^T = K Q^T, so that a lane has one row's scores (32 x 32
// tiles: column = row of queries), and the weights are the operand of O^T = V^T P^T without
// leaving their lanes.  The first product takes the cache's codes as they are: matrix
// instructions with a scale a block of 32 channels read 4-bit keys against queries in
// 8-bit terms, which hold a bfloat16 down to 2^-21 of its block's largest, at the rate of 16-bit
// products (two terms);
// LDS holds and moves a quarter of the bytes.  Values become 16-bit floats in LDS, once a
// workgroup, and the weights 16-bit floats with 11 bits (two terms, 22 bits, for float32).
// For float32 the keys become bfloat16 before the first product, and the queries three terms.
//
// 16-bit floats hold values 2^31 apart exactly (attend.hpp).  A workgroup that meets others among its
// part's keys, hidden or not, goes over them again with values as bfloat16, whose exponents span the
// cache's, and weights in two or three bfloat16 terms: 1.7 to 2.3 times as long in all (four prompts
// as below, every eighth token's values 2^60 larger: 1282 us for 565).  Looking for them costs nothing
// measurable at 128 channels and 15 in 1000 of a prompt of heads of 64.
//
// Four prompts of 4096 tokens, 32 heads of 128 over 8, bfloat16: 565 to 605 us, 910 to 970
// TFLOP/s (a large bfloat16 matrix product: 1287); 512 tokens over 32768: 254 to 266 us, 1.04 to
// 1.09 PFLOP/s.  The matrix units work half of the time.  At two waves a SIMD, which the sums and
// operands leave room for, the rest is issue and latency of the vector and LDS work between the
// products: without any matrix instruction a call takes as long to 4 parts in 100.  Exponentials
// and roundings of the weights are a quarter of that, reading the turned values a tenth.  Heads past
// 128 channels, past 64 in float32, have one wave a SIMD, and registers in scratch at 224 and 256
// channels, in float32 from 192 on (the first pass by itself: 33 and 46 a lane; 26, 128 and 138).  No faster:
// 64 rows a wave (its registers spill), the scheduler's own grouping of the instructions,
// apart code for tiles at the mask's edge, loads for the first tiles ahead of the queries.
#include <utility>

#include "attend.hpp"

namespace coinf {

namespace {

// A workgroup of W waves: 32 W rows, 16 W keys a tile (a wave brings 16 of them).
template <typename T, int NB, int W>
struct Rows {
  static constexpr int KEYS = kCacheTile * W, HALVES = KEYS / 32;
  static constexpr int QT = kQueryTerms<T>, PT = kWeightTerms<T>;
  // float32: keys as bfloat16, products from 0
  static constexpr bool WIDE = sizeof(T) == 4;
  static constexpr bool EVEN = NB % 2 == 0;
  // of a 32 x 32 tile of scores: depth 64, or 16
  static constexpr int MMA = WIDE ? QT * NB * 2 : QT * NB / 2;
  static constexpr int FRAGS = EVEN ? NB / 2 : NB;  // of keys
  static constexpr int CHUNKS = NB * kCacheTile;    // 16 bytes of codes of 16 tokens
  static constexpr int PER = (CHUNKS + 63) / 64;
  static constexpr int VS = NB * 32 + 32;           // rows 64 bytes apart modulo the banks
  // term and block of the half h of instruction j
  static __device__ int term(int j, int h) { return EVEN ? 2 * j / NB : 2 * (j / NB) + h; }
  static __device__ int block(int j, int h) { return EVEN ? 2 * j % NB + h : j % NB; }
};

// f(0), f(1), .. f(N - 1), of constants: long bodies too, which loops are not unrolled for.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

// Has v made by here.
__device__ __forceinline__ void hold(float& v) { asm volatile("" : "+v"(v)); }

constexpr int kNoPage = 1, kNotFinite = 2;  // flags of 16 tokens

template <typename T, int NB, int W>
struct RowsLds {
  using R = Rows<T, NB, W>;
  alignas(16) uint8_t k[3][W * R::CHUNKS * 16];  // by tile modulo 3, the others modulo 2
  alignas(16) _Float16 v[2][R::KEYS * R::VS];
  uint8_t ks[3][W * R::CHUNKS];
  alignas(16) uint8_t vs[4][W * R::CHUNKS];  // by tile modulo 4, 0 of keys not the stream's
  int32_t flags[4][W];           // by tile modulo 4
  int32_t lost;
};

// A workgroup's pass over its part, to the end or, true, until its values' range is known to be too
// wide: E is the values' exponent, 0 before the first pass, and the pass for far values takes it as
// it is.
template <typename T, int NB, int W, bool FAR>
__device__ __forceinline__ bool attend_rows(const AttendArgs& a, RowsLds<T, NB, W>& s, int& E) {
  using R = Rows<T, NB, W>;
  using Value = std::conditional_t<FAR, bf16x8, f16x8>;
  constexpr int kRows = 32 * W, kKeys = R::KEYS, PT = FAR ? kFarTerms<T> : R::PT;
  int tid = threadIdx.x;
  // nothing of the first pass is kept for the second
  if constexpr (FAR) asm volatile("" : "+v"(tid));
  const int lane = tid % 64, col = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);

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
    return false;
  }
  const int t_last = fdiv(min(row0 + kRows, rows) - 1, a.by_group);
  const Part part(a, span.lo(a, fdiv(row0, a.by_group)), span.base + t_last + 1, split);
  if (split >= part.parts) return false;
  if (!FAR && tid == 0) s.lost = 0;

  // queries, as 8-bit terms
  const bool live = row < rows;
  const T* q = static_cast<const T*>(a.q.data) + b * a.q.batch_stride +
               int64_t(live ? t : 0) * a.q.token_stride + int64_t(live ? head : 0) * a.d.head_dim;
  std::conditional_t<R::WIDE, bf16x8, i32x8> qo[R::MMA];
  int qs[R::MMA];
  bool q_bad = false;
  if constexpr (R::WIDE) {
    // instruction f, m, term: this half's channels 8 m of block 2 f + half, or 16 m + 8 half of block f
#pragma unroll
    for (int i = 0; i < R::MMA / R::QT; ++i) {
      const int c = R::EVEN ? 64 * (i / 4) + 32 * half + 8 * (i % 4)
                            : 32 * (i / 2) + 16 * (i % 2) + 8 * half;
      float v[8];
#pragma unroll
      for (int w = 0; w < 2; ++w)
        load4<T>(q, live ? c + 4 * w : a.d.head_dim, a.d.head_dim, a.wide, v + 4 * w);
      uint32_t most = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] *= a.q_sign;
        most = max(most, __float_as_uint(v[k]) & 0x7fffffffu);
      }
      const bool bad = most >= 0x7f800000u;
      q_bad |= bad;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = bad ? 0.f : v[k];
      bf16x8 terms[R::QT];
      to_bf16_terms<R::QT>(v, terms);
#pragma unroll
      for (int k = 0; k < R::QT; ++k) qo[i * R::QT + k] = terms[k];
    }
    q_bad |= __shfl_xor(int(q_bad), 32) != 0;
  } else {
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      float v[16];
#pragma unroll
      for (int w = 0; w < 4; ++w)
        load4<T>(q, live ? blk * 32 + 16 * half + 4 * w : a.d.head_dim, a.d.head_dim, a.wide,
                 v + 4 * w);
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
  }

  // The keys' way: pages three tiles ahead, codes of keys and scales of values two, codes of values
  // one.  A wave brings 16 of a tile's tokens, from one page: nothing of them is read out of
  // a page's range, and without a page they are 0.
  const char* pool = static_cast<const char*>(a.c.pool) + int64_t(kv) * a.lay.bytes();
  const int32_t* table = a.c.table + int64_t(b) * a.d.stream_pages;
  const int sub_mask = a.lay.P / kCacheTile - 1, head_bytes = a.lay.bytes();
  const auto load_page = [&](int tile) {
    const int lp = (tile * W + wave) >> (a.page_shift - 4);
    return table[lp - fdiv(lp, a.by_W) * a.d.stream_pages];
  };
  const auto page_ok = [&](int p) {
    p = __builtin_amdgcn_readfirstlane(p);
    return p >= 0 && p < a.d.pages ? p : -1;
  };
  const auto page_rsrc = [&](int page) {
    return make_rsrc(pool + max(page, 0) * a.page_bytes, page < 0 ? 0 : head_bytes);
  };
  // which 16 tokens of the page are this wave's of the tile
  const auto place = [&](int tile) { return (tile * W + wave) & sub_mask; };
  int at16[R::PER], at1[R::PER];  // this lane's bytes of 16 tokens' codes and scales
#pragma unroll
  for (int i = 0; i < R::PER; ++i) {
    const int c = lane + 64 * i;
    at16[i] = c < R::CHUNKS ? c * 16 : kOutOfRange;
    at1[i] = c < R::CHUNKS ? c : kOutOfRange;
  }
  const int hi = span.base + span.n;
  i32x4 rk[R::PER], rv[R::PER];
  int rks[R::PER], rvs[R::PER], rvs_next[R::PER];
  const auto fetch_keys = [&](int page, int tile) {  // and the values' scales
    const auto r = page_rsrc(page);
    const int n = place(tile);
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
      rk[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                            r, at16[i], n * (R::CHUNKS * 16), 0));
      rks[i] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(
          r, at1[i], a.lay.scales(0) + n * R::CHUNKS, 0));
      rvs_next[i] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(
          r, at1[i], a.lay.scales(1) + n * R::CHUNKS, 0));
    }
  };
  const auto fetch_values = [&](int page, int tile) {
    const auto r = page_rsrc(page);
    const int n = place(tile);
#pragma unroll
    for (int i = 0; i < R::PER; ++i)
      rv[i] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                     r, at16[i], a.lay.codes(1) + n * (R::CHUNKS * 16), 0));
  };
  // The keys and the values' scales into LDS: the scales of the stream's own tokens, what else a
  // page holds may be anything.
  const auto fill_keys = [&](int page, int tile, int slot) {
    const int pos0 = tile * kKeys + wave * kCacheTile;
    if (pos0 < span.lowest || pos0 + kCacheTile > hi) {
      const int tok = lane % 16;
#pragma unroll
      for (int i = 0; i < R::PER; ++i)
        rvs_next[i] = tok >= span.lowest - pos0 && tok < hi - pos0 ? rvs_next[i] : 0;
    }
    bool bad = false;
#pragma unroll
    for (int i = 0; i < R::PER; ++i) bad |= rvs_next[i] == 255;
    s.flags[tile & 3][wave] = (page < 0 ? kNoPage : 0) | (__any(bad) ? kNotFinite : 0);
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
      const int c = lane + 64 * i;
      if (c >= R::CHUNKS) break;
      *reinterpret_cast<i32x4*>(s.k[slot] + (wave * R::CHUNKS + c) * 16) = rk[i];
      s.ks[slot][wave * R::CHUNKS + c] = uint8_t(rks[i]);
      s.vs[tile & 3][wave * R::CHUNKS + c] = uint8_t(rvs_next[i]);
    }
  };

  f32x16 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x16{};
  // Minus the row's reference score, and its sum.  The products begin there (all 16 alike): what
  // they give is the difference.  over: what a difference may reach, everything before the first.
  f32x16 below = f32x16{};
  float l[2] = {0.f, 0.f}, over = -3e38f;
  int E0 = 0;         // the first exponent
  uint64_t lost = 0;  // lanes whose values were
  if (FAR) E = far_exponent(E);

  // The values into LDS, a quarter of a lane's 32 at a time.  The quarters of a row's blocks change
  // places by (row / 4) % 4, so that 16 rows' lie in all banks.
  const auto fill_values = [&](int buf, int E, int piece) {
#pragma unroll
    for (int i = 0; i < R::PER; ++i) {
      const int c = lane + 64 * i;
      if (c >= R::CHUNKS) break;
      _Float16* dst = s.v[buf] + (wave * kCacheTile + c % 16) * R::VS + c / 16 * 32 +
                      8 * (piece ^ c / 4 % 4);
      if constexpr (FAR) {
        *reinterpret_cast<bf16x8*>(dst) = decode8_far(rv[i][piece], rvs[i], E);
      } else {
        // without a scale: 0
        const int e = max(127 + kValueLift + rvs[i] - E, 0);
        const float scale = __uint_as_float(uint32_t(rvs[i] == 0 || rvs[i] == 255 ? 0 : e) << 23);
        *reinterpret_cast<f16x8*>(dst) = decode8(rv[i][piece], scale);
      }
    }
    if (!FAR && piece == 0)
#pragma unroll
      for (int i = 0; i < R::PER; ++i) lost |= __ballot(lost_values<T>(rvs[i], E));
  };
  // the values' exponent for a tile
  const auto exponent = [&](int tile) {
    if (FAR) return E;
    constexpr int WORDS = W * R::CHUNKS / 4;  // of scales
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const auto word = [&](int i) {
      const int w = lane + 64 * i;
      return reinterpret_cast<const uint32_t*>(s.vs[tile & 3])[WORDS % 64 ? min(w, WORDS - 1) : w];
    };
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < (WORDS + 63) / 64; ++i) {
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, word(i) & 0xff00ffu));
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, word(i) >> 8 & 0xff00ffu));
    }
    if (!__any(max(top[0], top[1]) > E)) return E;
    int most = 0;  // but for those that are not finite
#pragma unroll
    for (int i = 0; i < (WORDS + 63) / 64; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = word(i) >> (8 * k) & 255;
        most = max(most, e == 255 ? 0 : e);
      }
    most = wave_max(most);
    return most > E ? most + kValueSlack : E;
  };
  // the sums follow it
  const auto follow = [&](int next) {
    if (next == E) return;
    if (E) {
      const float down = exponent_to_f32(127 + E - next);
#pragma unroll
      for (int i = 0; i < NB; ++i) o[i] *= down;
    } else {
      E0 = next;
    }
    E = next;
  };

  // the wave's rows: their tokens, and the keys that some and that all of them see
  const int wave_rows = min(row0 + wave * 32 + 32, rows) - (row0 + wave * 32);
  const int wt0 = fdiv(row0 + wave * 32, a.by_group);
  const int wt1 = fdiv(row0 + wave * 32 + max(wave_rows, 1) - 1, a.by_group);
  const int some_lo = span.lo(a, wt0), some_hi = wave_rows > 0 ? span.base + wt1 : -1;
  const int all_lo = span.lo(a, wt1), all_hi = span.base + wt0;
  const int my_lo = span.lo(a, t), my_hi = live ? span.base + t : -1;

  // Scores of 32 keys (a half): those of two halves are held, and the largest of the newer one's.
  f32x16 sc[2];
  float top[2];  // of even and odd ones
  i32x4 kf[R::FRAGS];
  int ks[R::FRAGS];
  const auto load_keys = [&](int h, int slot) {
#pragma unroll
    for (int f = 0; f < R::FRAGS; ++f) {
      const int blk = R::EVEN ? 2 * f + half : f;
      const int at = ((2 * h + col / 16) * NB + blk) * 16 + col % 16;
      kf[f] = *reinterpret_cast<const i32x4*>(s.k[slot] + at * 16);
      ks[f] = s.ks[slot][at];
    }
  };
  bf16x8 key;
  const auto score = [&](int g, int i) {  // instruction i of them: the lowest terms first
    const f32x16 from = i ? sc[g] : R::WIDE ? f32x16{} : below;
    if constexpr (R::WIDE) {
      const int sub = i / R::QT, f = R::EVEN ? sub / 4 : sub / 2;
      if (i % R::QT == 0)
        key = decode8_bf16(R::EVEN ? kf[f][sub % 4] : half ? kf[f][sub % 2 * 2 + 1]
                                                           : kf[f][sub % 2 * 2], ks[f]);
      sc[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, qo[sub * R::QT + R::QT - 1 - i % R::QT],
                                                      from, 0, 0, 0);
    } else {
      const int j = R::MMA - 1 - i;
      const i32x4 k = kf[j % R::FRAGS];
      sc[g] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
          i32x8{k[0], k[1], k[2], k[3], 0, 0, 0, 0}, qo[j], from, 4, 0, 0, ks[j % R::FRAGS], 0,
          qs[j]);
    }
  };
  const auto largest = [&](int g, int i0, int i1) {
#pragma unroll
    for (int i = i0; i < i1; ++i) top[i % 2] = i < 2 ? sc[g][i] : fmaxf(top[i % 2], sc[g][i]);
  };
  // half h's scores within the row's keys and the reference
  const auto settle = [&](int h, int pos0, bool edge, int no_page) {
    const int g = h % 2;
    if (edge) {
      const int from = my_lo - pos0, to = my_hi - pos0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = 32 * h + 8 * (i / 4) + 4 * half + i % 4;
        const bool see = k >= from && k <= to && !(no_page >> (2 * h + i / 8) & 1);
        sc[g][i] = see ? sc[g][i] : -__builtin_inff();
      }
      largest(g, 0, 16);
    }
    const uint32_t all = __float_as_uint(fmaxf(top[0], top[1]));
    const auto both = __builtin_amdgcn_permlane32_swap(all, all, false, false);
    const float high = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) +
                       (R::WIDE ? below[0] : 0.f);
    if (__any(high > over)) {
      const float more = high > over ? high : 0.f;
      const float down = over < 0.f ? 1.f : exp2_fast(-more * a.scale_log2);
      over = high > over ? a.slack : over;
      l[0] *= down;
      l[1] *= down;
#pragma unroll
      for (int i = 0; i < NB; ++i) o[i] *= down;
#pragma unroll
      for (int i = 0; i < (R::WIDE ? 1 : 16); ++i) {
        if (!R::WIDE) sc[g][i] -= more;
        below[i] -= more;
      }
    }
  };
  // Half h's weights and what they add, beside the scores of half `h_other`, whose keys are loaded; then
  // those of half h_keys are.
  // A matrix instruction that waits for its unit keeps the other waves' vector instructions
  // waiting too, so a part of the vector work follows each of them, about as long as it takes:
  // weights, the largest of the next scores, and what `beside` has (NB pieces).  The scheduler would
  // put the matrix instructions side by side, so it is held to this order.
  const auto advance = [&](int h, int buf, int h_other, int h_keys, int slot_keys, auto&& beside) {
    const int g = h % 2, other = h_other % 2;
    const int j16 = lane % 16;
    const int quarter = 2 * (lane / 16 % 2) + j16 % 4 / 2;  // of a block, before they change places
    const _Float16* base = s.v[buf] + (32 * h + 4 * half + j16 / 4) * R::VS + 4 * (j16 % 2);
    const _Float16* lo = base + 8 * (quarter ^ half);
    const _Float16* hi = base + 8 * R::VS + 8 * (quarter ^ (2 + half));
    const auto values = [&](int i) {  // 16 keys i / NB, block i % NB
      const int at = 16 * (i / NB) * R::VS + 32 * (i % NB);
      struct Both {
        s16x4 lo, hi;
      } r;
      r.lo = turned4(lo + at);
      r.hi = turned4(hi + at);
      return __builtin_bit_cast(Value, r);
    };
    // weights in four groups of four, each a stage behind the one before: arguments, powers, operands
    Value p[PT][2], v[NB];
    float x[16];
    const auto weigh = [&](int stage) {
#pragma unroll
      for (int i = 4 * stage; i < 4 * stage + 4; ++i)
        if (i < 16)
          x[i] = fmaf(R::WIDE ? sc[g][i] + below[0] : sc[g][i], a.scale_log2, kLift);
#pragma unroll
      for (int i = 4 * stage - 4; i < 4 * stage; ++i)
        if (i >= 0 && i < 16) x[i] = exp2_fast(x[i]);
#pragma unroll
      for (int i = 4 * stage - 8; i < 4 * stage - 4; i += 2) {
        if (i < 0) continue;
        f32x2 w = {x[i], x[i + 1]};
        if constexpr (FAR) {
          l[i / 2 % 2] += w[0] + w[1];
#pragma unroll
          for (int k = 0; k < PT; ++k)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const __bf16 r = __bf16(w[n]);
              p[k][i / 8][i % 8 + n] = r;
              w[n] -= float(r);
            }
        } else {
#pragma unroll
          for (int k = 0; k < PT; ++k) {
            const f16x2 r = __builtin_convertvector(w, f16x2);
            p[k][i / 8][i % 8] = r[0];
            p[k][i / 8][i % 8 + 1] = r[1];
            // the sum of the weights as they are used
            l[i / 2 % 2] = __builtin_amdgcn_fdot2(r, f16x2{1, 1}, l[i / 2 % 2], false);
            if (k + 1 < PT) w -= __builtin_convertvector(r, f32x2);
          }
        }
      }
    };
    const auto add = [&](int i) {
#pragma unroll
      for (int k = 0; k < PT; ++k)
        if constexpr (FAR)
          o[i % NB] =
              __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[i % NB], p[k][i / NB], o[i % NB], 0, 0, 0);
        else
          o[i % NB] =
              __builtin_amdgcn_mfma_f32_32x32x16_f16(v[i % NB], p[k][i / NB], o[i % NB], 0, 0, 0);
    };
    constexpr int STAGES = 6;
    each<R::MMA>([&](auto j) {
      score(other, j);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = STAGES * j / R::MMA; i < STAGES * (j + 1) / R::MMA; ++i) weigh(i);
#pragma unroll
      for (int i = NB * j / R::MMA; i < NB * (j + 1) / R::MMA; ++i) v[i] = values(i);
      __builtin_amdgcn_sched_barrier(0);
    });
    load_keys(h_keys, slot_keys);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      add(i);
      __builtin_amdgcn_sched_barrier(0);
      v[i] = values(NB + i);
      beside(i);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      add(NB + i);
      __builtin_amdgcn_sched_barrier(0);
      largest(other, 16 * i / NB, 16 * (i + 1) / NB);
      __builtin_amdgcn_sched_barrier(0);
    }
    // made here, not where they are used
    hold(top[0]);
    hold(top[1]);
    hold(l[0]);
    hold(l[1]);
  };

  // The pages of the next tiles.  Past the part's end there are none, and what goes to LDS is 0.
  const auto page_at = [&](int tile, int loaded) { return tile < part.end ? page_ok(loaded) : -1; };
  int page0 = -1, page1 = -1, page2 = -1, flags = 0;
  if (part.first < part.end) {
    page0 = page_at(part.first, load_page(part.first));
    page1 = page_at(part.first + 1, load_page(part.first + 1));
    page2 = page_at(part.first + 2, load_page(part.first + 2));
    fetch_values(page0, part.first);
    fetch_keys(page0, part.first);
    fill_keys(page0, part.first, 0);
#pragma unroll
    for (int i = 0; i < R::PER; ++i) rvs[i] = rvs_next[i];
    fetch_keys(page1, part.first + 1);
    fill_keys(page1, part.first + 1, 1);
    __syncthreads();
    follow(exponent(part.first));
#pragma unroll
    for (int i = 0; i < 4; ++i) fill_values(part.first & 1, E, i);
    load_keys(0, 0);
    each<R::MMA>([&](auto j) { score(0, j); });
    largest(0, 0, 16);
    load_keys(1, 0);
    flags = s.flags[part.first & 3][lane % W];
  }
  __syncthreads();

  int slot = 0;  // of the tile's keys
  for (int tile = part.first; tile < part.end; ++tile) {
    const int buf = tile & 1;
    const int pos0 = tile * kKeys;
    const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot1 == 2 ? 0 : slot1 + 1;
    const int coming = load_page(tile + 3);
#pragma unroll
    for (int i = 0; i < R::PER; ++i) rvs[i] = rvs_next[i];
    fetch_values(page1, tile + 1);
    fetch_keys(page2, tile + 2);
    const int no_page = int(__ballot(flags & kNoPage)) & ((1 << W) - 1);
    const bool not_finite = __any(flags & kNotFinite);
    int E1;
    if (pos0 <= some_hi && pos0 + kKeys > some_lo) {
      const bool edge = pos0 + kKeys - 1 > all_hi || pos0 < all_lo || no_page;
#pragma unroll
      for (int h = 0; h < R::HALVES; ++h) {
        settle(h, pos0, edge, no_page);
        if (h == R::HALVES - 1) E1 = exponent(tile + 1);
        // past the last tile: 0
        const int h1 = (h + 1) % R::HALVES, h2 = (h + 2) % R::HALVES;
        advance(h, buf, h1, h2, h + 2 < R::HALVES ? slot : slot1, [&](int i) {
          // the next tiles' values and keys, as late as may be: they are on their way
          if (h == R::HALVES - 1) {
#pragma unroll
            for (int k = 4 * i / NB; k < 4 * (i + 1) / NB; ++k)
              fill_values(buf ^ 1, E1, k);
            if (i == NB - 1) fill_keys(page2, tile + 2, slot2);
          }
        });
      }
      if (not_finite) {  // a block that is not finite, to the rows that see its token
        for (int c = 0; c < W * R::CHUNKS; ++c) {
          if (s.vs[tile & 3][c] != 255) continue;
          const int sub = c / R::CHUNKS, blk = c % R::CHUNKS / 16;
          const int pos = pos0 + sub * 16 + c % 16;
          const bool see = pos >= my_lo && pos <= my_hi && !(no_page >> sub & 1);
          const float nan = see ? __builtin_nanf("") : 0.f;
#pragma unroll
          for (int i = 0; i < NB; ++i)
            if (i == blk)
#pragma unroll
              for (int k = 0; k < 16; ++k) o[i][k] += nan;
        }
      }
    } else {
      E1 = exponent(tile + 1);
      fill_keys(page2, tile + 2, slot2);
#pragma unroll
      for (int i = 0; i < 4; ++i) fill_values(buf ^ 1, E1, i);
      load_keys(0, slot1);
      each<R::MMA>([&](auto j) { score(0, j); });
      largest(0, 0, 16);
      load_keys(1, slot1);
    }
    flags = s.flags[(tile + 1) & 3][lane % W];
    follow(E1);
    page1 = page2;
    page2 = page_at(tile + 3, coming);
    slot = slot1;
    __syncthreads();
  }

  if constexpr (!FAR) {
    if (lost || E - E0 > kMostRise) s.lost = 1;
    __syncthreads();
    if (__builtin_expect(s.lost, 0)) return true;
  }
  float sum = l[0] + l[1];
  sum += __shfl_xor(sum, 32);
  if (!live) {
    if (split == 0) no_output();
    return false;
  }
  const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
  // 2^{E - 127 - kValueLift} in two steps, neither out of range; 2^{E - 127 - kFarLift} is in it
  const float up = exponent_to_f32(FAR ? E - kFarLift : E - kValueSlack);
  const float less = FAR ? 1.f : exponent_to_f32(127 + kValueSlack - kValueLift);
  const float bad = q_bad && sum > 0.f ? __builtin_nanf("") : 0.f;
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
    return false;
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
  if (half == 0) a.part_stat[at] = {-below[0], sum};
  return false;
}

template <typename T, int NB, int W>
__global__ __launch_bounds__(64 * W, NB <= kWideBlocks<T> ? 2 : 1) void attend_rows_kernel(AttendArgs a) {
  __shared__ RowsLds<T, NB, W> s;
  int E = 0;
  if (__builtin_expect(attend_rows<T, NB, W, false>(a, s, E), 0))
    attend_rows<T, NB, W, true>(again(a), s, E);
}

template <typename T, int NB>
void run(const AttendArgs& a, int rows, unsigned grid, hipStream_t s) {
  if constexpr (NB <= kWideBlocks<T>) {
    if (rows == 256) {
      attend_rows_kernel<T, NB, 8><<<grid, 512, 0, s>>>(a);
      return;
    }
  }
  attend_rows_kernel<T, NB, 4><<<grid, 256, 0, s>>>(a);
}

template <typename T>
void run(const AttendArgs& a, int NB, int rows, unsigned grid, hipStream_t s) {
  switch (NB) {
    case 1: run<T, 1>(a, rows, grid, s); break;
    case 2: run<T, 2>(a, rows, grid, s); break;
    case 3: run<T, 3>(a, rows, grid, s); break;
    case 4: run<T, 4>(a, rows, grid, s); break;
    case 5: run<T, 5>(a, rows, grid, s); break;
    case 6: run<T, 6>(a, rows, grid, s); break;
    case 7: run<T, 7>(a, rows, grid, s); break;
    default: run<T, 8>(a, rows, grid, s); break;
  }
}

}  // namespace

void launch_attend_rows(const AttendArgs& a, int NB, int rows, hipStream_t stream) {
  const unsigned grid = unsigned(int64_t(a.pairs) * a.row_tiles * a.splits);
  if (a.d.dtype == CO_BF16)
    run<bf16_t>(a, NB, rows, grid, stream);
  else
    run<float>(a, NB, rows, grid, stream);
}

}  // namespace coinf
