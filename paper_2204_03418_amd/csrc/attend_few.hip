// Attention of few rows (single and drafted tokens) over the cache: bound by the
// cache's bytes.  A workgroup takes a part of one stream's keys of a kv head, and its
// four waves go over it 32 keys at a time, each by itself and without barriers: keys come
// from memory as the operand that they are, values pass through the wave's own LDS to be
// turned.  The products are as in the kernel of many rows, in 16 x 16 tiles, a column
// tile for each 16 rows.  At the end the waves' sums are joined in LDS, and the parts' in
// a launch of their own.  Values too far apart for 16-bit floats, as in that kernel: the workgroup
// goes over its part again (64 streams of 8192: 227 us for 114).
//
// One token of 64 streams of 8192, 32 heads of 128 over 8, bfloat16: 106 to 111 us and 5 for the
// joining, 571 MB at 5.1 TB/s beside it, a copy's rate.  Short calls are latency: 32 x 6 tokens
// over 2500, 16 heads of 64 over 4, 17 and 4 us (the way to the pages, then four steps of 32 keys a
// wave, each a load, two products and the softmax between); one token over 300, float32, 7.5 us.
#include <algorithm>

#include "attend.hpp"

namespace coinf {

namespace {

constexpr int kWaves = kBlock / 64;
constexpr int kStep = 32;  // keys

template <typename T, int NB>
struct Few {
  static constexpr int QT = kQueryTerms<T>, PT = kWeightTerms<T>;
  // a matrix instruction has four slots of 32 channels: four blocks of a term, or two of two terms,
  // or one of four
  static constexpr int NBP = NB <= 2 ? NB : (NB + 3) / 4 * 4;
  static constexpr int FRAGS = NBP >= 4 ? NBP / 4 : 1;
  // float32: keys as bfloat16, an instruction a term and 8 of a lane's channels
  static constexpr bool WIDE = sizeof(T) == 4;
  static constexpr int SUBS = NBP >= 4 ? 4 : NBP;  // of a fragment
  static constexpr int MMA = WIDE         ? QT * FRAGS * SUBS
                             : NBP >= 4   ? QT * FRAGS
                             : NBP == 2   ? QT / 2
                                          : (QT + 3) / 4;
  static constexpr int CHUNKS = NB * kStep;  // 16 bytes of values of a step
  static constexpr int VC = (CHUNKS + 63) / 64;
  static constexpr int VS = NB * 32 + 16;    // rows 32 bytes beside a multiple of the banks
  // of a slot of fragment f
  static __device__ int block(int f, int slot) {
    return NBP >= 4 ? 4 * f + slot : NBP == 2 ? slot % 2 : 0;
  }
};

// Waves a SIMD: what the first pass's registers and LDS leave room for.
template <typename T, int NB, int CT>
constexpr int few_waves() {
  if (NB > 4) return 1;
  if (sizeof(T) == 2) return CT == 1 || NB <= 2 ? 4 : 2;
  return CT == 1 ? (NB <= 2 ? 4 : 3) : NB <= 1 ? 4 : NB <= 2 ? 3 : 2;
}

// One wave's values, and at the end its sums (16 rows of NB * 32, 64 bytes more each).
template <typename T, int NB>
struct FewLds {
  union {
    alignas(16) _Float16 v[kStep * Few<T, NB>::VS];
    alignas(16) float o[16 * (NB * 32 + 16)];
  };
};

template <typename T, int NB>
struct FewAll {
  FewLds<T, NB> wave[kWaves];
  float2 stats[kWaves][16];
  int32_t lost[kWaves];
};

// A workgroup's pass over its part, to the end or, true, until its values' range is known to be too
// wide: E is the wave's values' exponent, 0 before the first pass, and the pass for far values takes
// it as it is.
template <typename T, int NB, int CT, bool FAR>
__device__ __forceinline__ bool attend_few(const AttendArgs& a, FewAll<T, NB>& s, int& E) {
  using F = Few<T, NB>;
  using Value = std::conditional_t<FAR, bf16x8, f16x8>;
  constexpr int PT = FAR ? kFarTerms<T> : F::PT;
  auto& lds = s.wave;
  auto& stats = s.stats;
  int tid = threadIdx.x;
  // nothing of the first pass is kept for the second
  if constexpr (FAR) asm volatile("" : "+v"(tid));
  const int lane = tid % 64, col = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int split = blockIdx.x / a.pairs, pair = blockIdx.x - split * a.pairs;
  const int b = fdiv(pair, a.by_kv), kv = pair - b * a.d.kv_heads;
  const Span span(a, b);
  const int rows = span.n * a.group;
  const auto token_of = [&](int row) { return fdiv(row, a.by_group); };
  const auto out_row = [&](int row) {
    const int t = token_of(row), head = kv * a.group + row - t * a.group;
    return static_cast<T*>(a.y.data) + b * a.y.batch_stride + t * a.y.token_stride +
           int64_t(head) * a.d.head_dim;
  };
  if (!FAR && split == 0) {  // outputs of tokens that the stream does not have
    const float none[4] = {};
    for (int i = tid; i < (a.T - span.n) * a.group * (NB * 8); i += kBlock)
      store4<T>(out_row(rows + i / (NB * 8)), i % (NB * 8) * 4, a.d.head_dim, a.wide, none);
  }
  if (rows == 0) return false;
  const Part part(a, span.lo(a, 0), span.base + span.n, split);
  if (split >= part.parts) return false;

  // The keys' way: pages two steps ahead, codes and scales one.  Nothing is read out of a page's
  // range, and without a page all is 0.  The two tiles of 16 tokens of a step lie in one page, or
  // with pages of 16 in two.
  const char* pool = static_cast<const char*>(a.c.pool) + int64_t(kv) * a.lay.bytes();
  const int32_t* table = a.c.table + int64_t(b) * a.d.stream_pages;
  constexpr int tile_bytes = NB * 256;
  const int sub_mask = a.lay.P / kCacheTile - 1, head_bytes = a.lay.bytes();
  const bool two = a.lay.P == kCacheTile;
  const auto load_page = [&](int tile) {  // of 16 tokens
    const int lp = tile >> (a.page_shift - 4);
    return table[lp - fdiv(lp, a.by_W) * a.d.stream_pages];
  };
  const auto page_rsrc = [&](int page) {
    return make_rsrc(pool + max(page, 0) * a.page_bytes, page < 0 ? 0 : head_bytes);
  };
  int at_k[F::FRAGS], at_v[F::VC], at_vs[F::VC];  // this lane's bytes of the keys' codes and the values'
  bool tile1[F::VC];                              // whether those are of the second tile
#pragma unroll
  for (int f = 0; f < F::FRAGS; ++f) {
    const int blk = F::block(f, g);
    at_k[f] = blk < NB ? blk * 16 + col : kOutOfRange / 16;
  }
#pragma unroll
  for (int i = 0; i < F::VC; ++i) {
    const int c = lane + 64 * i, tile = c / (NB * 16), rest = c - tile * NB * 16;
    tile1[i] = tile > 0;
    at_v[i] = c < F::CHUNKS ? (two ? 0 : tile * tile_bytes) + rest * 16 : kOutOfRange;
    at_vs[i] = c < F::CHUNKS ? (two ? 0 : tile * NB * 16) + rest : kOutOfRange;
  }
  int page[2], coming[2];
  i32x4 rk[2][F::FRAGS], rv[F::VC];
  int rks[2][F::FRAGS], rvs[F::VC];
  const auto fetch_pages = [&](int step) {
    coming[0] = load_page(2 * step);
    if (two) coming[1] = load_page(2 * step + 1);
  };
  const auto take_pages = [&] {
    const auto ok = [&](int p) {
      p = __builtin_amdgcn_readfirstlane(p);
      return p >= 0 && p < a.d.pages ? p : -1;
    };
    page[0] = ok(coming[0]);
    page[1] = two ? ok(coming[1]) : page[0];
  };
  const auto fetch = [&](int step) {
    const auto r0 = page_rsrc(page[0]), r1 = page_rsrc(page[1]);
    const int n0 = (2 * step) & sub_mask, n1 = (2 * step + 1) & sub_mask;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto r = i ? r1 : r0;
      const int n = i ? n1 : n0;
#pragma unroll
      for (int f = 0; f < F::FRAGS; ++f) {
        rk[i][f] = __builtin_bit_cast(
            i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at_k[f] * 16, n * tile_bytes, 0));
        rks[i][f] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(
            r, at_k[f], a.lay.scales(0) + n * NB * 16, 0));
      }
    }
#pragma unroll
    for (int i = 0; i < F::VC; ++i) {
      const int v = a.lay.codes(1) + n0 * tile_bytes, vs = a.lay.scales(1) + n0 * NB * 16;
      rv[i] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                     r0, two && tile1[i] ? kOutOfRange : at_v[i], v, 0));
      rvs[i] = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(
          r0, two && tile1[i] ? kOutOfRange : at_vs[i], vs, 0));
    }
    if (two) {  // n0 = n1 = 0
#pragma unroll
      for (int i = 0; i < F::VC; ++i) {
        rv[i] |= __builtin_bit_cast(
            i32x4, __builtin_amdgcn_raw_buffer_load_b128(r1, tile1[i] ? at_v[i] : kOutOfRange,
                                                         a.lay.codes(1), 0));
        rvs[i] |= uint8_t(__builtin_amdgcn_raw_buffer_load_b8(
            r1, tile1[i] ? at_vs[i] : kOutOfRange, a.lay.scales(1), 0));
      }
    }
  };

  const int hi = span.base + span.n;
  const int end = min(part.end * (kFewKeys / kStep), (hi + kStep - 1) / kStep);
  int step = part.first * (kFewKeys / kStep) + wave;
  if (step < end) {  // on their way beside the queries
    fetch_pages(step);
    take_pages();
    fetch(step);
    if (step + kWaves < end) fetch_pages(step + kWaves);
  }

  // queries, as 8-bit terms
  std::conditional_t<F::WIDE, bf16x8, i32x8> qo[CT][F::MMA];
  int qs[CT][F::MMA];
  bool q_bad[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int row = 16 * c + col;
    const bool live = row < rows;
    const int t = token_of(live ? row : 0), head = kv * a.group + (live ? row - t * a.group : 0);
    const T* q = static_cast<const T*>(a.q.data) + b * a.q.batch_stride + t * a.q.token_stride +
                 int64_t(head) * a.d.head_dim;
    q_bad[c] = false;
    if constexpr (F::WIDE) {
      // the channels that a lane's keys have: 8 of sub m of its block's four eights
#pragma unroll
      for (int i = 0; i < F::FRAGS * F::SUBS; ++i) {
        const int f = i / F::SUBS, m = i % F::SUBS;
        const int eight = F::NBP >= 4 ? m : F::NBP == 2 ? 2 * m + g / 2 : g;
        const int at = F::block(f, g) * 32 + 8 * eight;
        float v[8];
#pragma unroll
        for (int w = 0; w < 2; ++w)
          load4<T>(q, live ? at + 4 * w : a.d.head_dim, a.d.head_dim, a.wide, v + 4 * w);
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[k] *= a.q_sign;
          most = max(most, __float_as_uint(v[k]) & 0x7fffffffu);
        }
        const bool bad = most >= 0x7f800000u;
        q_bad[c] |= bad;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = bad ? 0.f : v[k];
        bf16x8 terms[F::QT];
        to_bf16_terms<F::QT>(v, terms);
#pragma unroll
        for (int k = 0; k < F::QT; ++k) qo[c][i * F::QT + k] = terms[k];
      }
    } else {
#pragma unroll
      for (int f = 0; f < F::FRAGS; ++f) {
        int byte[2];
        i32x4 words[2][F::QT];
        // this lane's halves of 16 channels: of slots g / 2 and 2 + g / 2
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (w == 1 && F::NBP <= 2) {  // the same block again
            byte[1] = byte[0];
#pragma unroll
            for (int k = 0; k < F::QT; ++k) words[1][k] = words[0][k];
            continue;
          }
          const int blk = F::NBP == 2 ? g / 2 : F::block(f, 2 * w + g / 2);
          float v[16];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            load4<T>(q, live ? blk * 32 + 16 * (g % 2) + 4 * i : a.d.head_dim, a.d.head_dim, a.wide,
                     v + 4 * i);
          uint32_t most = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            v[i] *= a.q_sign;
            most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
          }
          most = max(most, uint32_t(__shfl_xor(int(most), 16)));
          const bool bad = most >= 0x7f800000u;
          q_bad[c] |= bad;
          byte[w] = bad ? 127 : query_scale(most);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = bad ? 0.f : v[i];
          to_terms<F::QT>(v, byte[w], words[w]);
        }
        // scales: of slot g, which lanes of group 2 (g % 2) have
        const int b0 = __shfl(byte[0], col + 32 * (g % 2)), b1 = __shfl(byte[1], col + 32 * (g % 2));
        const int mine = g / 2 ? b1 : b0;
#pragma unroll
        for (int k = 0; k < F::MMA / F::FRAGS; ++k) {
          const int j = k * F::FRAGS + f;
#pragma unroll
          for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if constexpr (F::NBP >= 4) {
                qo[c][j][4 * w + i] = words[w][k][i];
              } else if constexpr (F::NBP == 2) {
                qo[c][j][4 * w + i] = words[w][2 * k + w][i];
              } else {
                const int t0 = 4 * k + 2 * w;
                const int lo = t0 < F::QT ? words[w][t0 < F::QT ? t0 : 0][i] : 0;
                const int hi = t0 + 1 < F::QT ? words[w][t0 + 1 < F::QT ? t0 + 1 : 0][i] : 0;
                qo[c][j][4 * w + i] = g / 2 ? hi : lo;
              }
            }
          qs[c][j] = mine - 4 * (F::NBP >= 4 ? k : F::NBP == 2 ? 2 * k + g / 2 : 4 * k + g);
        }
      }
    }
    // all lanes of a column
    q_bad[c] |= __shfl_xor(int(q_bad[c]), 16) != 0;
    q_bad[c] |= __shfl_xor(int(q_bad[c]), 32) != 0;
  }

  f32x4 o[CT][NB * 2];
  float m[CT], l[CT];
  int E0 = 0;         // the first exponent
  uint64_t lost = 0;  // lanes whose values were
  if (FAR) E = far_exponent(E);
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    m[c] = -3e38f;  // below every score
    l[c] = 0.f;
#pragma unroll
    for (int i = 0; i < NB * 2; ++i) o[c][i] = f32x4{};
  }
  const int lo_all = span.lo(a, span.n - 1), hi_all = span.base;  // that all rows see
  int my_lo[CT], my_hi[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int row = 16 * c + col, t = token_of(row);
    my_lo[c] = span.lo(a, t);
    my_hi[c] = row < rows ? span.base + t : -1;
  }
  _Float16* vbuf = lds[wave].v;
  for (; step < end; step += kWaves) {
    const int pos0 = step * kStep;
    const int pages = (page[0] >= 0) | (page[1] >= 0) << 1;
    // scores: the keys are used up first
    f32x4 sc[CT][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int c = 0; c < CT; ++c) sc[c][i] = f32x4{};
      if constexpr (F::WIDE) {
#pragma unroll
        for (int n = 0; n < F::FRAGS * F::SUBS; ++n) {
          const i32x4 w = rk[i][n / F::SUBS];
          const int m = n % F::SUBS;
          const int eight = F::NBP >= 4   ? w[m]
                            : F::NBP == 2 ? (g / 2 ? w[2 * m + 1] : w[2 * m])
                            : g / 2       ? (g % 2 ? w[3] : w[2])
                                          : (g % 2 ? w[1] : w[0]);
          const bf16x8 key = decode8_bf16(eight, rks[i][n / F::SUBS]);
#pragma unroll
          for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int k = F::QT - 1; k >= 0; --k)  // the lowest terms first
              sc[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, qo[c][n * F::QT + k],
                                                                 sc[c][i], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int j = F::MMA - 1; j >= 0; --j) {  // the lowest terms first
            const i32x4 w = rk[i][j % F::FRAGS];
            sc[c][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                i32x8{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, qo[c][j], sc[c][i], 4, 0, 0,
                rks[i][j % F::FRAGS], 0, qs[c][j]);
          }
      }
    }
    // values, as 16-bit floats into LDS
    if (pos0 < span.lowest || pos0 + kStep > hi) {  // of the stream's own tokens
#pragma unroll
      for (int i = 0; i < F::VC; ++i) {
        const int tok = (tile1[i] ? 16 : 0) + lane % 16;
        rvs[i] = tok >= span.lowest - pos0 && tok < hi - pos0 ? rvs[i] : 0;
      }
    }
    int top_s = 0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < F::VC; ++i) {
      bad |= rvs[i] == 255;
      top_s = max(top_s, rvs[i] == 255 ? 0 : rvs[i]);
    }
    if (!FAR && __any(top_s > E)) {
      const int next = wave_max(top_s) + kValueSlack;
      if (E) {
        const float down = exponent_to_f32(127 + E - next);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int i = 0; i < NB * 2; ++i) o[c][i] *= down;
      } else {
        E0 = next;
      }
      E = next;
    }
    if (!FAR)
#pragma unroll
      for (int i = 0; i < F::VC; ++i) lost |= __ballot(lost_values<T>(rvs[i], E));
#pragma unroll
    for (int i = 0; i < F::VC; ++i) {
      const int c = lane + 64 * i, tile = c / (NB * 16), rest = c - tile * NB * 16;
      if (c >= F::CHUNKS) break;
      // without a scale: 0
      const int e = max(127 + kValueLift + rvs[i] - E, 0);
      const float scale = __uint_as_float(uint32_t(rvs[i] == 0 || rvs[i] == 255 ? 0 : e) << 23);
      _Float16* dst = vbuf + (tile * 16 + rest % 16) * F::VS + rest / 16 * 32;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if constexpr (FAR)
          *reinterpret_cast<bf16x8*>(dst + 8 * k) = decode8_far(rv[i][k], rvs[i], E);
        else
          *reinterpret_cast<f16x8*>(dst + 8 * k) = decode8(rv[i][k], scale);
    }
    int raw[F::VC];
#pragma unroll
    for (int i = 0; i < F::VC; ++i) raw[i] = rvs[i];
    if (step + kWaves < end) {
      take_pages();
      fetch(step + kWaves);
      if (step + 2 * kWaves < end) fetch_pages(step + 2 * kWaves);
    }
    const bool whole = pos0 >= lo_all && pos0 + kStep - 1 <= hi_all && pages == 3;
    Value p[CT][PT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (!whole || 16 * (c + 1) > rows) {
        const int first = my_lo[c] - pos0, last = my_hi[c] - pos0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = 16 * (i / 4) + 4 * g + i % 4;
          const bool see = k >= first && k <= last && (pages >> (i / 4) & 1);
          sc[c][i / 4][i % 4] = see ? sc[c][i / 4][i % 4] : -__builtin_inff();
        }
      }
      float top = sc[c][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[c][i / 4][i % 4]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m[c] + a.slack)) {
        const float next = fmaxf(top, m[c]);
        const float down = exp2_fast((m[c] - next) * a.scale_log2);
        l[c] *= down;
#pragma unroll
        for (int i = 0; i < NB * 2; ++i) o[c][i] *= down;
        m[c] = next;
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        f32x2 w;
#pragma unroll
        for (int k = 0; k < 2; ++k)
          w[k] = exp2_fast(fmaf(sc[c][(i + k) / 4][(i + k) % 4] - m[c], a.scale_log2, kLift));
        if constexpr (FAR) {
          l[c] += w[0] + w[1];
#pragma unroll
          for (int k = 0; k < PT; ++k)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const __bf16 r = __bf16(w[n]);
              p[c][k][i + n] = r;
              w[n] -= float(r);
            }
        } else {
#pragma unroll
          for (int k = 0; k < PT; ++k) {
            const f16x2 r = __builtin_convertvector(w, f16x2);
            p[c][k][i] = r[0];
            p[c][k][i + 1] = r[1];
            l[c] = __builtin_amdgcn_fdot2(r, f16x2{1, 1}, l[c], false);
            if (k + 1 < PT) w -= __builtin_convertvector(r, f32x2);
          }
        }
      }
    }
    __builtin_amdgcn_wave_barrier();  // a wave's LDS instructions stay in order
    const _Float16* base = vbuf + (4 * g + col / 4) * F::VS + 4 * (col % 4);
#pragma unroll
    for (int i = 0; i < NB * 2; ++i) {
      struct Both {
        s16x4 lo, hi;
      } r;
      r.lo = turned4(base + 16 * i);
      r.hi = turned4(base + 16 * F::VS + 16 * i);
      const Value v = __builtin_bit_cast(Value, r);
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int k = 0; k < PT; ++k)
          if constexpr (FAR)
            o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[c][k], o[c][i], 0, 0, 0);
          else
            o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[c][k], o[c][i], 0, 0, 0);
    }
    __builtin_amdgcn_wave_barrier();
    if (__any(bad)) {  // blocks that are not finite, to the rows that see their tokens
#pragma unroll
      for (int i = 0; i < F::VC; ++i)
        for (int k = 0; k < 64; ++k) {
          const int c = k + 64 * i;
          if (c >= F::CHUNKS) break;
          if (__builtin_amdgcn_readlane(raw[i], k) != 255) continue;
          const int tile = c / (NB * 16), blk = c % (NB * 16) / 16;
          const int pos = pos0 + tile * 16 + c % 16;
#pragma unroll
          for (int q = 0; q < CT; ++q) {
            const bool see = pos >= my_lo[q] && pos <= my_hi[q] && (pages >> tile & 1);
            const float nan = see ? __builtin_nanf("") : 0.f;
#pragma unroll
            for (int n = 0; n < NB * 2; ++n)
              if (n / 2 == blk) o[q][n] += nan;
          }
        }
    }
  }

  if (!FAR) s.lost[wave] = lost || E - E0 > kMostRise;
  // the waves' sums together, a column tile at a time
  constexpr int OS = NB * 32 + 16;
  // 2^{E - 127 - kValueLift} in two steps, neither out of range; 2^{E - 127 - kFarLift} is in it
  const float up = exponent_to_f32(FAR ? E - kFarLift : E - kValueSlack);
  const float less = FAR ? 1.f : exponent_to_f32(127 + kValueSlack - kValueLift);
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    if (16 * c >= rows) break;
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
    const float inv = l[c] > 0.f || l[c] != l[c] ? 1.f / l[c] : 0.f;
    const float nan = q_bad[c] && l[c] > 0.f ? __builtin_nanf("") : 0.f;
    if (c) __syncthreads();
#pragma unroll
    for (int i = 0; i < NB * 2; ++i) {
      Pack<float, 4> v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v.v[k] = o[c][i][k] * inv * less * up + nan;
      store_pack<float, 4>(lds[wave].o + col * OS + 16 * i + 4 * g, v);
    }
    if (g == 0) stats[wave][col] = {m[c], l[c]};
    __syncthreads();
    if (!FAR && c == 0) {
      int any = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) any |= s.lost[w];
      if (__builtin_expect(any, 0)) return true;
    }
    for (int i = tid; i < 16 * NB * 8; i += kBlock) {
      const int r = i / (NB * 8), ch = i % (NB * 8) * 4, row = 16 * c + r;
      if (row >= rows) break;
      float top = -__builtin_inff(), sum = 0.f, v[4] = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stats[w][r].x);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 st = stats[w][r];
        if (st.y == 0.f) continue;  // sees nothing there
        const float weight = exp2_fast((st.x - top) * a.scale_log2) * st.y;
        sum += weight;
        const Pack<float, 4> x = load_pack<float, 4>(lds[w].o + r * OS + ch);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = fmaf(weight, x.v[k], v[k]);
      }
      const float all = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] *= all;
      if (part.parts == 1) {
        store4<T>(out_row(row), ch, a.d.head_dim, a.wide, v);
      } else {
        const int64_t at = (int64_t(pair) * a.splits + split) * (CT * 16) + row;
        store_pack<float, 4>(a.part + at * (NB * 32) + ch, Pack<float, 4>{{v[0], v[1], v[2], v[3]}});
        if (ch == 0) a.part_stat[at] = {top, sum};
      }
    }
  }
  return false;
}

template <typename T, int NB, int CT>
__global__ __launch_bounds__(kBlock, (few_waves<T, NB, CT>())) void attend_few_kernel(
    AttendArgs a) {
  __shared__ FewAll<T, NB> s;
  int E = 0;
  if (__builtin_expect(attend_few<T, NB, CT, false>(a, s, E), 0))
    attend_few<T, NB, CT, true>(again(a), s, E);
}

template <typename T, int NB>
void run(const AttendArgs& a, int tiles, unsigned grid, hipStream_t s) {
  if (tiles == 1)
    attend_few_kernel<T, NB, 1><<<grid, kBlock, 0, s>>>(a);
  else
    attend_few_kernel<T, NB, 2><<<grid, kBlock, 0, s>>>(a);
}

template <typename T>
void run(const AttendArgs& a, int NB, int tiles, unsigned grid, hipStream_t s) {
  switch (NB) {
    case 1: run<T, 1>(a, tiles, grid, s); break;
    case 2: run<T, 2>(a, tiles, grid, s); break;
    case 3: run<T, 3>(a, tiles, grid, s); break;
    case 4: run<T, 4>(a, tiles, grid, s); break;
    case 5: run<T, 5>(a, tiles, grid, s); break;
    case 6: run<T, 6>(a, tiles, grid, s); break;
    case 7: run<T, 7>(a, tiles, grid, s); break;
    default: run<T, 8>(a, tiles, grid, s); break;
  }
}

}  // namespace

void launch_attend_few(const AttendArgs& a, int NB, int tiles, hipStream_t stream) {
  const unsigned grid = unsigned(a.pairs) * a.splits;
  if (a.d.dtype == CO_BF16)
    run<bf16_t>(a, NB, tiles, grid, stream);
  else
    run<float>(a, NB, tiles, grid, stream);
}

}  // namespace coinf
