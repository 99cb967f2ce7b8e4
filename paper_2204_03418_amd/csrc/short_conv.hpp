// How the short convolution's tokens are cut between threads (host and device).
#pragma once

#include <cstdint>

namespace coinf {

constexpr int kRun = 2;             // tokens a thread loads and sums together
constexpr int kConvThreads = 256;   // of a workgroup

struct ShortConvCut {
  int32_t lanes;     // threads of a workgroup across the channels; the others along the tokens
  int32_t run;       // tokens of a run: kRun, 1 for a call over single tokens
  int32_t runs;      // of a thread
  int32_t t_blocks;  // workgroups along the tokens
};

// The first token of the thread in row `row` of workgroup `block` along the tokens.
constexpr int64_t shortconv_first(const ShortConvCut& c, int64_t block, int64_t row) {
  return (block * (kConvThreads / c.lanes) + row) * c.run * c.runs;
}

// More runs a thread load the tokens before them less often, where that leaves two waves for each
// of 1024 SIMDs.  4 x 4096 tokens of 4352 channels in bfloat16 (285 MB): one run of 8 tokens a
// thread 91 us, 4 of 8 81 us (at half the occupancy), 8 of 4 64 us, 8 of 2 59 us.
//
// The K - 1 inputs before a thread's first token are the carried state as far as they lie before
// token 0.  The threads of token 0 alone write the new state, in place, and nothing makes the
// others wait: so none of those may read it, and a thread takes K - 1 tokens at least.
inline ShortConvCut shortconv_cut(int32_t B, int64_t packs, int32_t T, int32_t K) {
  if (T == 1) return {kConvThreads, 1, 1, 1};
  const int64_t threads = packs * B * ((int64_t(T) + kRun - 1) / kRun);
  int32_t runs = 8;
  while (runs > 1 && threads / runs < 2 * 1024 * 64 && kRun * (runs / 2) >= K - 1) runs /= 2;
  // few tokens: threads across the channels
  const int32_t lanes = T <= 4 * kRun ? 64 : 32;
  return {lanes, kRun, runs, (T - 1) / (kRun * runs * (kConvThreads / lanes)) + 1};
}

}  // namespace coinf
