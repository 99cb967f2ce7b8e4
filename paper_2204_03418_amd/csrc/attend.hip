// Attention over the cache: which kernel a call takes, and the parts of its keys joined.
#include <algorithm>

#include "attend.hpp"

namespace coinf {

namespace {

// Joins the parts of a row, each weighed by its sum and reference: four values a lane, `lanes` (a
// power of two, 4 lanes >= width) a row.  Latency: 4 to 5.6 us a call, 10 us for 512 x 32 rows of 4 parts.
template <typename T>
__global__ __launch_bounds__(kBlock) void attend_join_kernel(AttendArgs a, int rows_of, int width,
                                                             int lanes, int64_t all_rows) {
  const int64_t r = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / lanes;
  if (r >= all_rows) return;
  const int ch = int(threadIdx.x) % lanes * 4;
  const int unit = int(r / rows_of), in = int(r - int64_t(unit) * rows_of);
  const int pair = fdiv(unit, a.by_row_tiles), rt = unit - pair * a.row_tiles;
  const int b = fdiv(pair, a.by_kv), kv = pair - b * a.d.kv_heads;
  const Span span(a, b);
  const int rows = span.n * a.group, row0 = rt * rows_of, row = row0 + in;
  if (row >= rows || ch >= width) return;
  const int t = fdiv(row, a.by_group), head = kv * a.group + row - t * a.group;
  const int t_last = fdiv(min(row0 + rows_of, rows) - 1, a.by_group);
  const Part part(a, span.lo(a, fdiv(row0, a.by_group)), span.base + t_last + 1, 0);
  if (part.parts == 1) return;
  const int64_t at = int64_t(unit) * a.splits * rows_of + in;
  // eight parts on their way at a time
  constexpr int AHEAD = 8;
  float top = -__builtin_inff(), sum = 0.f, v[4] = {};
  for (int s0 = 0; s0 < part.parts; s0 += AHEAD) {
    float2 stat[AHEAD];
    Pack<float, 4> x[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int64_t i = at + int64_t(min(s0 + s, part.parts - 1)) * rows_of;
      stat[s] = a.part_stat[i];
      if (s0 + s >= part.parts) stat[s].y = 0.f;
      x[s] = load_pack<float, 4>(a.part + i * width + ch);
    }
    float next = top;
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) next = stat[s].y == 0.f ? next : fmaxf(next, stat[s].x);
    const float down = top == next ? 1.f : exp2_fast((top - next) * a.scale_log2);
    sum *= down;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= down;
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      if (stat[s].y == 0.f) continue;  // sees nothing there
      const float w = exp2_fast((stat[s].x - next) * a.scale_log2) * stat[s].y;
      sum += w;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = fmaf(w, x[s].v[k], v[k]);
    }
    top = next;
  }
  T* y = static_cast<T*>(a.y.data) + b * a.y.batch_stride + t * a.y.token_stride +
         int64_t(head) * a.d.head_dim;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] *= inv;
  store4<T>(y, ch, a.d.head_dim, a.wide, v);
}

// How the rows of a call are cut.
struct Cut {
  int64_t pairs, row_tiles, splits, rows;
  int few;  // column tiles of the kernel of few rows, or 0
  int part_keys;  // of a part at least
  int64_t units() const { return pairs * row_tiles; }
};

// A call of fewer units than the card holds workgroups has its keys cut in parts: two a CU of many
// rows, one of large heads; four of few, which is what up to 16 bfloat16 rows of heads to 128 and float32
// ones to 64 have, and up to 32 of half such heads (others one to three: their parts run in rounds).
// Both counts go by the room of the
// table's rows, which the host knows, not by what streams hold.
Cut cut_of(const co_attn_desc& d, int32_t T) {
  Cut c;
  c.pairs = int64_t(d.batch) * d.kv_heads;
  const int64_t rows = int64_t(T) * (d.heads / d.kv_heads);
  const int64_t keys = std::min<int64_t>(int64_t(d.stream_pages) * d.page_tokens,
                                         d.window ? int64_t(d.window) + T + kMostKeys : INT64_MAX);
  c.few = rows <= kFewTiles * 16 ? int((rows + 15) / 16) : 0;
  // 256 rows share what a tile of keys costs to bring, but nothing runs beside the start and end of
  // their workgroups: they take long contexts to be made up for (512 tokens over 32768: 266 us,
  // 293 with 128 rows; 4 prompts of 4096: 610 and 605)
  const int most = d.dtype == CO_BF16 ? kWideBlocks<bf16_t> : kWideBlocks<float>;
  c.rows = c.few ? c.few * 16 : rows > 128 && keys >= 8192 && cache_blocks(d.head_dim) <= most
                                    ? 256 : 128;
  c.row_tiles = (rows + c.rows - 1) / c.rows;
  // large heads: one a CU (2 x 1000 bfloat16 tokens, 8 heads of 256: 66 us, 84 with parts for two)
  const bool two = c.rows == 128 && cache_blocks(d.head_dim) <= most;
  const int64_t room = (c.few ? 1024 : two ? 512 : 256) / c.units();
  const auto cut = [&](int part_keys) {
    c.part_keys = part_keys;
    c.splits = std::max<int64_t>(1, std::min(room, (keys + part_keys - 1) / part_keys));
  };
  cut(c.few ? 512 : 256);
  // Smaller parts where joining them stays short, 24 of a row and 6 MB of sums at most (16 streams of
  // 45 float32 tokens, 6 heads of 40, window 250: 16.5 us for 20, 4.4 MB; 64 tokens over 2000, 32
  // heads of 128: 42 for 31, 17 MB; 40 over 8000, 63 parts: 25 for 22), and not the first cut of a
  // call that needs no joining (128 tokens: 14 for 11).
  if (!c.few && keys > 256) {
    cut(128);
    if (c.splits > 24 || rows * c.pairs * c.splits * cache_blocks(d.head_dim) * 128 > 6 << 20)
      cut(256);
  }
  return c;
}

}  // namespace

int64_t attend_workspace(const co_attn_desc& d, int32_t T) {
  if (T == 0) return 0;
  const Cut c = cut_of(d, T);
  if (c.splits == 1) return 0;
  return c.units() * c.splits * c.rows * (cache_blocks(d.head_dim) * 32 + 2) * 4;
}

hipError_t launch_attend(const co_attn_desc& d, const co_attn_cache& cache, const co_tokens& q,
                         const co_tokens& y, int32_t T, void* workspace, hipStream_t stream) {
  AttendArgs a{d, cache, q, y, T};
  const int NB = cache_blocks(d.head_dim);
  a.lay = {d.page_tokens, NB};
  a.page_bytes = int64_t(a.lay.bytes()) * d.kv_heads;
  const float scale = d.scale * kLog2e;
  a.q_sign = scale > 0 ? 1.f : scale < 0 ? -1.f : 0.f;
  a.scale_log2 = scale == 0 ? 1.f : fabsf(scale);
  a.slack = kSlack / a.scale_log2;
  a.group = d.heads / d.kv_heads;
  const Cut c = cut_of(d, T);
  if (int64_t(T) * a.group + c.rows >= INT32_MAX || c.units() * c.splits >= 1 << 23)
    return hipErrorInvalidConfiguration;
  a.by_group = make_fastdiv(a.group);
  a.by_W = make_fastdiv(d.stream_pages);
  a.by_kv = make_fastdiv(d.kv_heads);
  while ((1 << a.page_shift) < d.page_tokens) ++a.page_shift;
  a.pairs = int32_t(c.pairs);
  a.row_tiles = int32_t(c.row_tiles);
  a.splits = int32_t(c.splits);
  a.keys = c.few ? kFewKeys : int32_t(c.rows / 2);
  a.part_tiles = c.part_keys / a.keys;
  a.by_row_tiles = make_fastdiv(a.row_tiles);
  a.by_splits = make_fastdiv(a.splits);
  const int es = d.dtype == CO_BF16 ? 2 : 4;
  a.wide = 1;
  for (const co_tokens* v : {&q, &y})
    if ((v->batch_stride | v->token_stride | d.head_dim |
         int64_t(reinterpret_cast<uintptr_t>(v->data) / es)) % 4)
      a.wide = 0;
  a.part = static_cast<float*>(workspace);
  a.part_stat = reinterpret_cast<float2*>(a.part + c.units() * c.splits * c.rows * NB * 32);
  if (c.few)
    launch_attend_few(a, NB, c.few, stream);
  else
    launch_attend_rows(a, NB, int(c.rows), stream);
  if (a.splits > 1) {
    const int64_t rows = c.units() * c.rows;
    const int lanes = NB <= 1 ? 8 : NB <= 2 ? 16 : NB <= 4 ? 32 : 64;
    const unsigned grid = unsigned((rows * lanes + kBlock - 1) / kBlock);
    if (d.dtype == CO_BF16)
      attend_join_kernel<bf16_t>
          <<<grid, kBlock, 0, stream>>>(a, int(c.rows), NB * 32, lanes, rows);
    else
      attend_join_kernel<float><<<grid, kBlock, 0, stream>>>(a, int(c.rows), NB * 32, lanes, rows);
  }
  return hipGetLastError();
}

}  // namespace coinf
