// How the short convolution cuts its tokens between threads: every token is
// some thread's, and no thread but those of token 0, which write the carried
// state, reads it.  argv[1] = "old": the same checks over the cut that let a
// thread take fewer tokens than the state has, which must be found out.
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "../../paper_2204_03418_amd/csrc/short_conv.hpp"

using namespace coinf;

static ShortConvCut short_runs(int32_t B, int64_t packs, int32_t T, int32_t K) {
  ShortConvCut c = shortconv_cut(B, packs, T, K);
  if (T > 1) {
    const int64_t threads = packs * B * ((int64_t(T) + kRun - 1) / kRun);
    c.runs = 8;
    while (c.runs > 1 && threads / c.runs < 2 * 1024 * 64) c.runs /= 2;
    c.t_blocks = (T - 1) / (kRun * c.runs * (kConvThreads / c.lanes)) + 1;
  }
  return c;
}

int main(int argc, char** argv) {
  const bool old = argc > 1 && !std::strcmp(argv[1], "old");
  long bad = 0, cuts = 0;
  const int32_t lengths[] = {1,  2,  3,  4,  5,   6,   7,   8,    9,    10,   11,         15, 16,
                             17, 31, 32, 33, 100, 127, 128, 1000, 4096, 65535, 0x7fffffff};
  const int64_t widths[] = {1, 7, 54, 544, 1088, 4352, 65536, 1 << 20};
  for (int32_t K = 1; K <= 8; ++K)
    for (int32_t T : lengths)
      for (int64_t packs : widths)
        for (int32_t B : {1, 2, 16, 32, 64, 1024}) {
          const ShortConvCut c = old ? short_runs(B, packs, T, K) : shortconv_cut(B, packs, T, K);
          ++cuts;
          const int64_t rows = kConvThreads / c.lanes, own = int64_t(c.run) * c.runs;
          bool ok = c.runs >= 1 && c.t_blocks >= 1 && kConvThreads % c.lanes == 0;
          // threads follow each other without a gap, past the last token
          ok = ok && shortconv_first(c, 0, 0) == 0 && shortconv_first(c, 0, 1) == own &&
               shortconv_first(c, 1, 0) == rows * own && c.t_blocks * rows * own >= T &&
               (c.t_blocks - 1) * rows * own < T;
          // the second thread is the nearest to the state; it reads tokens from t0 - (K - 1) on
          const int64_t t0 = own;
          if (t0 < T && t0 < K - 1) ok = false;
          if (!ok && ++bad < 5)
            std::printf("K %d T %d packs %ld B %d: lanes %d runs %d blocks %d\n", K, T, long(packs),
                        B, c.lanes, c.runs, c.t_blocks);
        }
  std::printf("%ld cuts, %ld bad\n", cuts, bad);
  return bad != 0;
}
