// Pages of the cache: reserve (with copies of shared pages), truncate, select
// (fork, reorder, free) and compact.
//
// The tables are small: what decides runs in one workgroup, whose prefix sums make
// every choice by order alone (streams in order, lowest free pages first), so that
// results do not depend on how atomics fall.  The counts of a page's holders change by
// integer atomics, which any order leaves the same.  What moves bytes is a launch of
// its own over as many workgroups as the bytes may need.
//
// 64 streams of 2000 tokens, 4 layers of 8 heads of 128: select 5.3 us, reserve 7.3 and its
// copies of half a page 5.7, truncate 2.9, all of them latency (passes over the table and the
// counts that depend on each other).  Compaction, 209 MB of pages in 2 layers:
// the plan 8 us (one workgroup), the moves 86 us, 4.8 TB/s of reading and writing.
#include <algorithm>

#include "cache.hpp"
#include "launch.hpp"
#include "token.hpp"

namespace coinf {

namespace {

constexpr int kOne = 1024;  // threads of the workgroup that decides

__device__ __forceinline__ int ref_load(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void ref_store(int32_t* p, int v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void ref_add(int32_t* p, int v) {
  __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Sum of v over the workgroup's threads before this one; total: over all.  All threads call it.
__device__ __forceinline__ int prefix_before(int v, int* scratch, int& total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  int sum = v;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const int up = __shfl_up(sum, m);
    sum += lane >= m ? up : 0;
  }
  if (lane == 63) scratch[wave] = sum;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < int(blockDim.x) / 64; ++w) {
    before += w < wave ? scratch[w] : 0;
    total += scratch[w];
  }
  __syncthreads();
  return before + sum - v;
}

struct PagesArgs {
  co_pages_desc d;
  co_pages s;
  const int32_t* lengths;
  int32_t T, keep;
  int32_t most;        // pages that T tokens touch at most
  int32_t* rank;       // (B, most): pages wanted up to this one
  int32_t* list;       // (B most): new pages, lowest first
  int32_t* copies;     // (B, 2): from, to; -1: none
};

constexpr int kFar = INT32_MAX - 4096;  // no position passes it

// Entry of the table that holds a stream's page lp, or -1 where it names none.
__device__ __forceinline__ int valid_page(int page, int pages) {
  return page >= 0 && page < pages ? page : -1;
}

// Decides: one workgroup.
__global__ __launch_bounds__(kOne) void reserve_kernel(PagesArgs a) {
  __shared__ int scratch[kOne / 64];
  const int B = a.d.batch, P = a.d.page_tokens, W = a.d.stream_pages, tid = threadIdx.x;
  // what the streams give up, and what they ask for
  for (int b = tid; b < B; b += kOne) {
    const int base = max(a.s.tokens[b], 0);
    int first = min(max(a.s.first[b], 0), base);
    if (a.keep > 0 && base - a.keep >= first) {
      const int to = base - a.keep + 1;
      for (int lp = first / P; lp < to / P; ++lp) {
        int32_t* entry = a.s.table + int64_t(b) * W + lp % W;
        const int page = valid_page(*entry, a.d.pages);
        if (page >= 0) ref_add(a.s.refs + page, -1);
        *entry = -1;
        if (lp - first / P >= W) break;
      }
      first = to;
    }
    int n = stream_tokens(a.lengths, b, a.T);
    int refused = 0;
    // its row has no room, or the positions no bits
    if (n > 0 && (base > kFar - n || (base + n - 1) / P - first / P >= W)) refused = n, n = 0;
    a.s.first[b] = first;
    a.s.base[b] = base;
    a.s.granted[b] = n;
    if (refused) a.s.refused[b] += refused;
    a.copies[2 * b] = -1;
  }
  __syncthreads();
  // pages wanted: rank by stream and position
  const int64_t items = int64_t(B) * a.most;
  int wanted = 0;
  for (int64_t i0 = 0; i0 < items; i0 += kOne) {
    const int64_t i = i0 + tid;
    int want = 0;
    if (i < items) {
      const int b = int(i / a.most), k = int(i % a.most);
      const int base = a.s.base[b], n = a.s.granted[b];
      const int lp = base / P + k;
      if (n > 0 && lp <= (base + n - 1) / P) {
        const int page = valid_page(a.s.table[int64_t(b) * W + lp % W], a.d.pages);
        want = page < 0 || ref_load(a.s.refs + page) > 1;
      }
    }
    int total;
    const int before = prefix_before(want, scratch, total);
    // sign bit: wants one
    if (i < items) a.rank[i] = (wanted + before + want) | (want << 31);
    wanted += total;
  }
  // as many of the lowest free pages
  int found = 0;
  for (int p0 = 0; p0 < a.d.pages && found < wanted; p0 += 4 * kOne) {
    bool free[4];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + 4 * tid + i;
      free[i] = p < a.d.pages && ref_load(a.s.refs + min(p, a.d.pages - 1)) <= 0;
      mine += free[i];
    }
    int total;
    int at = found + prefix_before(mine, scratch, total);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free[i] && at < wanted) a.list[at++] = p0 + 4 * tid + i;
    found += total;
  }
  found = min(found, wanted);
  __syncthreads();
  for (int b = tid; b < B; b += kOne) {
    const int n = a.s.granted[b];
    if (n == 0) continue;
    const int32_t* rank = a.rank + int64_t(b) * a.most;
    const int last = rank[a.most - 1] & INT32_MAX;
    const int before = (rank[0] & INT32_MAX) - (rank[0] < 0);
    if (last > before && last > found) {
      a.s.granted[b] = 0;
      a.s.refused[b] += n;
    }
  }
  __syncthreads();
  for (int64_t i = tid; i < items; i += kOne) {
    const int rank = a.rank[i];
    if (rank >= 0) continue;
    const int b = int(i / a.most), k = int(i % a.most);
    if (a.s.granted[b] == 0) continue;
    const int base = a.s.base[b];
    int32_t* entry = a.s.table + int64_t(b) * W + (base / P + k) % W;
    const int old = valid_page(*entry, a.d.pages), page = a.list[(rank & INT32_MAX) - 1];
    if (old >= 0) {
      ref_add(a.s.refs + old, -1);
      if (k == 0 && base % P) {
        a.copies[2 * b] = old;
        a.copies[2 * b + 1] = page;
      }
    }
    *entry = page;
    ref_store(a.s.refs + page, 1);
  }
  for (int b = tid; b < B; b += kOne) a.s.tokens[b] = a.s.base[b] + a.s.granted[b];
}

// The tiles that hold a stream's tokens in a page that it shared, to its new page: a workgroup a
// stream, layer and kv head.
__global__ __launch_bounds__(kBlock) void copy_shared_kernel(PagesArgs a) {
  const int b = blockIdx.y;
  const int from = a.copies[2 * b];
  if (from < 0) return;
  const int to = a.copies[2 * b + 1];
  const int P = a.d.page_tokens;
  const PageHead lay{P, (a.d.head_dim + kCacheBlock - 1) / kCacheBlock};
  const int tiles = (a.s.base[b] % P + kCacheTile - 1) / kCacheTile;
  const int64_t bytes = lay.bytes();
  for (int unit = blockIdx.x; unit < a.d.layers * a.d.kv_heads; unit += gridDim.x) {
    const int layer = unit / a.d.kv_heads, h = unit - layer * a.d.kv_heads;
    char* pool = static_cast<char*>(a.s.pool);
    const char* src = pool + ((int64_t(layer) * a.d.pages + from) * a.d.kv_heads + h) * bytes;
    char* dst = pool + ((int64_t(layer) * a.d.pages + to) * a.d.kv_heads + h) * bytes;
    const int n = tiles * lay.tile_bytes() / 16, ns = tiles * kCacheTile * lay.NB / 16;
    for (int i = threadIdx.x; i < 2 * (n + ns); i += kBlock) {
      int at;  // 16 bytes each: codes of K and V, scales of K and V
      if (i < 2 * n)
        at = lay.codes(i >= n) + (i >= n ? i - n : i) * 16;
      else
        at = lay.scales(i - 2 * n >= ns) + ((i - 2 * n) % ns) * 16;
      store_pack<int32_t, 4>(reinterpret_cast<int32_t*>(dst + at),
                             load_pack<int32_t, 4>(reinterpret_cast<const int32_t*>(src + at)));
    }
  }
}

// Page of a stream that slot s of its row is for, counted from its oldest.
__device__ __forceinline__ int slot_page(int s, int oldest, int W) {
  int k = s - oldest % W;
  k += k < 0 ? W : 0;
  return oldest + k;
}

// A workgroup a stream.
__global__ __launch_bounds__(kBlock) void truncate_kernel(PagesArgs a) {
  const int b = blockIdx.x, P = a.d.page_tokens, W = a.d.stream_pages;
  const int tokens = max(a.s.tokens[b], 0), to = min(tokens, max(a.lengths[b], 0));
  const int first = min(max(a.s.first[b], 0), tokens);
  const bool none = to <= first;
  for (int s = threadIdx.x; s < W; s += kBlock) {
    int32_t* entry = a.s.table + int64_t(b) * W + s;
    const int page = *entry;
    if (page < 0 || (!none && int64_t(slot_page(s, first / P, W)) * P < to)) continue;
    if (page < a.d.pages) ref_add(a.s.refs + page, -1);
    *entry = -1;
  }
  __syncthreads();
  if (threadIdx.x) return;
  a.s.first[b] = min(first, to);
  a.s.tokens[b] = a.s.base[b] = to;
  a.s.granted[b] = 0;
}

// New rows of the table beside it; refs to 0.
__global__ __launch_bounds__(kBlock) void select_gather_kernel(PagesArgs a, const int32_t* source,
                                                               int32_t* rows) {
  const int B = a.d.batch, P = a.d.page_tokens, W = a.d.stream_pages;
  const int64_t n = int64_t(B) * W, at = blockIdx.x * int64_t(kBlock) + threadIdx.x;
  const int64_t step = int64_t(gridDim.x) * kBlock;
  for (int64_t i = at; i < n; i += step) {
    const int b = int(i / W), s = int(i % W), from = source[b];
    int page = -1;
    if (from >= 0 && from < B) {
      const int tokens = a.s.tokens[from], first = min(max(a.s.first[from], 0), tokens);
      if (int64_t(slot_page(s, first / P, W)) * P < tokens)
        page = valid_page(a.s.table[int64_t(from) * W + s], a.d.pages);
    }
    rows[i] = page;
  }
  for (int64_t b = at; b < B; b += step) {
    const int from = source[b];
    const bool some = from >= 0 && from < B;
    rows[n + b] = some ? max(a.s.tokens[from], 0) : 0;
    rows[n + B + b] = some ? max(a.s.first[from], 0) : 0;
  }
  for (int64_t p = at; p < a.d.pages; p += step) a.s.refs[p] = 0;
}

__global__ __launch_bounds__(kBlock) void select_store_kernel(PagesArgs a, const int32_t* rows) {
  const int B = a.d.batch;
  const int64_t n = int64_t(B) * a.d.stream_pages;
  const int64_t at = blockIdx.x * int64_t(kBlock) + threadIdx.x;
  const int64_t step = int64_t(gridDim.x) * kBlock;
  for (int64_t i = at; i < n; i += step) {
    const int page = rows[i];
    a.s.table[i] = page;
    if (page >= 0) ref_add(a.s.refs + page, 1);
  }
  for (int64_t b = at; b < B; b += step) {
    a.s.tokens[b] = a.s.base[b] = rows[n + b];
    a.s.first[b] = rows[n + B + b];
    a.s.granted[b] = 0;
  }
}

// Both in one workgroup, whose threads hold the new rows.
constexpr int kHeld = 8;
__global__ __launch_bounds__(kOne) void select_one_kernel(PagesArgs a, const int32_t* source) {
  const int B = a.d.batch, P = a.d.page_tokens, W = a.d.stream_pages, n = B * W;
  const int tid = threadIdx.x;
  int page[kHeld], tokens = 0, first = 0;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = k * kOne + tid;
    page[k] = -1;
    if (i >= n) continue;
    const int b = i / W, s = i - b * W, from = source[b];
    if (from < 0 || from >= B) continue;
    const int end = a.s.tokens[from], low = min(max(a.s.first[from], 0), end);
    if (int64_t(slot_page(s, low / P, W)) * P < end)
      page[k] = valid_page(a.s.table[from * W + s], a.d.pages);
  }
  if (tid < B && source[tid] >= 0 && source[tid] < B) {
    tokens = max(a.s.tokens[source[tid]], 0);
    first = max(a.s.first[source[tid]], 0);
  }
  for (int p = tid; p < a.d.pages; p += kOne) ref_store(a.s.refs + p, 0);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = k * kOne + tid;
    if (i >= n) continue;
    a.s.table[i] = page[k];
    if (page[k] >= 0) ref_add(a.s.refs + page[k], 1);
  }
  if (tid >= B) return;
  a.s.tokens[tid] = a.s.base[tid] = tokens;
  a.s.first[tid] = first;
  a.s.granted[tid] = 0;
}

// Bit i: whether a page p + i has holders, p + i < n.
constexpr int kEach = 8;
__device__ __forceinline__ int used_pages(const int32_t* refs, int p, int n) {
  int v[kEach], bits = 0;
  if (p + kEach <= n) {
    __builtin_memcpy(v, refs + p, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = p + i < n ? refs[p + i] : 0;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) bits |= (v[i] > 0) << i;
  return bits;
}

// Which pages move where: one workgroup.  moves: their number, then (from, to) each; rank: which of
// them a page is.
__global__ __launch_bounds__(kOne) void compact_plan_kernel(PagesArgs a, int32_t* moves,
                                                            int32_t* rank) {
  __shared__ int scratch[kOne / 64];
  constexpr int PASS = kEach * kOne;
  const int n = a.d.pages, tid = threadIdx.x;
  int mine_used = 0, used, kept = 0;  // kept: the first four passes' bits
  for (int p0 = 0; p0 < n; p0 += PASS) {
    const int bits = used_pages(a.s.refs, p0 + kEach * tid, n);
    mine_used += __popc(bits);
    if (p0 < 4 * PASS) kept |= bits << (p0 / PASS * kEach);
  }
  prefix_before(mine_used, scratch, used);
  // the k-th free page below `used` takes the k-th used one above
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < n; p0 += PASS) {
    const int p = p0 + kEach * tid;
    int bits = p0 < 4 * PASS ? kept >> (p0 / PASS * kEach) & 255 : used_pages(a.s.refs, p, n);
    // below `used`: the free ones
    const int below = p + kEach <= used ? 255 : p < used ? (1 << (used - p)) - 1 : 0;
    bits ^= below;
    int total;  // at most 8 k of either in a pass
    const int at = prefix_before(__popc(bits & below) | __popc(bits & ~below) << 16, scratch, total);
    int hole = holes + (at & 0xffff), mover = movers + (at >> 16);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (!(bits >> i & 1)) continue;
      if (below >> i & 1) {
        moves[2 + 2 * hole++] = p + i;
      } else {
        rank[p + i] = mover;
        moves[1 + 2 * mover++] = p + i;
      }
    }
    holes += total & 0xffff;
    movers += total >> 16;
  }
  if (tid == 0) moves[0] = movers;
}

constexpr int kPiece = 16384;  // bytes that a workgroup moves at a time

// Moves the pages and names them anew in the table.
__global__ __launch_bounds__(kBlock) void compact_move_kernel(PagesArgs a, const int32_t* moves,
                                                              const int32_t* rank,
                                                              int64_t page_bytes) {
  const int count = moves[0];
  if (count == 0) return;
  const int64_t n = int64_t(a.d.batch) * a.d.stream_pages;
  const int used_first = moves[1];  // the lowest page that moves; all used ones above do
  for (int64_t i = blockIdx.x * int64_t(kBlock) + threadIdx.x; i < n;
       i += int64_t(gridDim.x) * kBlock) {
    const int page = a.s.table[i];
    if (page < used_first || page >= a.d.pages) continue;
    const int k = rank[page];  // anything, for a page that nobody counts
    if (k >= 0 && k < count && moves[1 + 2 * k] == page) a.s.table[i] = moves[2 + 2 * k];
  }
  for (int i = blockIdx.x * kBlock + threadIdx.x; i < count; i += gridDim.x * kBlock) {
    const int from = moves[1 + 2 * i];
    a.s.refs[moves[2 + 2 * i]] = a.s.refs[from];
    a.s.refs[from] = 0;
  }
  const int pieces = int((page_bytes + kPiece - 1) / kPiece);
  const int64_t units = int64_t(count) * a.d.layers * pieces;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t row = u / pieces;
    const int64_t at = (u % pieces) * kPiece, layer = row / count;
    const int64_t move = row % count;
    char* pool = static_cast<char*>(a.s.pool) + layer * a.d.pages * page_bytes;
    const char* src = pool + moves[1 + 2 * move] * page_bytes + at;
    char* dst = pool + moves[2 + 2 * move] * page_bytes + at;
    const int left = int(min(int64_t(kPiece), page_bytes - at));
    Pack<int32_t, 4> v[kPiece / 16 / kBlock];
#pragma unroll
    for (int i = 0; i < kPiece / 16 / kBlock; ++i) {
      const int o = (i * kBlock + threadIdx.x) * 16;
      if (o < left) v[i] = load_pack<int32_t, 4>(reinterpret_cast<const int32_t*>(src + o));
    }
#pragma unroll
    for (int i = 0; i < kPiece / 16 / kBlock; ++i) {
      const int o = (i * kBlock + threadIdx.x) * 16;
      if (o < left) store_pack<int32_t, 4>(reinterpret_cast<int32_t*>(dst + o), v[i]);
    }
  }
}

int64_t round16(int64_t v) { return (v + 15) / 16 * 16; }

}  // namespace

int64_t page_bytes(const co_pages_desc& d) {
  return int64_t(PageHead{d.page_tokens, cache_blocks(d.head_dim)}.bytes()) * d.kv_heads;
}

// reserve: ranks and a list, of a page a table entry and one more a stream at most, and copies;
// select: rows, tokens, firsts; compact: moves and ranks.
int64_t pages_workspace(const co_pages_desc& d) {
  const int64_t B = d.batch, items = B * (d.stream_pages + 1);
  return round16(4 * std::max(2 * items + 2 * B, 3 * int64_t(d.pages) + 1));
}

hipError_t launch_pages_reserve(const co_pages_desc& d, const co_pages& s, int32_t T,
                                const int32_t* lengths, int32_t keep, hipStream_t stream) {
  PagesArgs a{d, s, lengths, T, keep};
  // a stream that touches more has no room for them, and is refused before its items count
  a.most = int32_t(std::min<int64_t>(T > 0 ? (int64_t(T) - 1) / d.page_tokens + 2 : 1,
                                     d.stream_pages + 1));
  int32_t* ws = static_cast<int32_t*>(s.workspace);
  a.rank = ws;
  a.list = ws + int64_t(d.batch) * a.most;
  a.copies = a.list + int64_t(d.batch) * a.most;
  reserve_kernel<<<1, kOne, 0, stream>>>(a);
  const dim3 grid(unsigned(std::min<int64_t>(int64_t(d.layers) * d.kv_heads, 1024)),
                  unsigned(d.batch));
  copy_shared_kernel<<<grid, kBlock, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_truncate(const co_pages_desc& d, const co_pages& s, const int32_t* lengths,
                                 hipStream_t stream) {
  const PagesArgs a{d, s, lengths, 0, 0};
  truncate_kernel<<<unsigned(d.batch), kBlock, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_select(const co_pages_desc& d, const co_pages& s, const int32_t* source,
                               hipStream_t stream) {
  const PagesArgs a{d, s, nullptr, 0, 0};
  int32_t* rows = static_cast<int32_t*>(s.workspace);
  // one launch where a workgroup holds the table (64 streams of 34 pages: 3.7 us for 5.8)
  if (d.batch <= kOne && int64_t(d.batch) * d.stream_pages <= kHeld * kOne &&
      d.pages <= 16 * kHeld * kOne) {
    select_one_kernel<<<1, kOne, 0, stream>>>(a, source);
    return hipGetLastError();
  }
  const int64_t most = std::max<int64_t>(int64_t(d.batch) * d.stream_pages, d.pages);
  const unsigned grid = unsigned(std::min<int64_t>(grid_for(most), 2048));
  select_gather_kernel<<<grid, kBlock, 0, stream>>>(a, source, rows);
  select_store_kernel<<<grid, kBlock, 0, stream>>>(a, rows);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const co_pages_desc& d, const co_pages& s, hipStream_t stream) {
  const PagesArgs a{d, s, nullptr, 0, 0};
  int32_t* moves = static_cast<int32_t*>(s.workspace);
  int32_t* rank = moves + 2 * int64_t(d.pages) + 1;
  compact_plan_kernel<<<1, kOne, 0, stream>>>(a, moves, rank);
  compact_move_kernel<<<2048, kBlock, 0, stream>>>(a, moves, rank, page_bytes(d));
  return hipGetLastError();
}

}  // namespace coinf
