// The search of the eviction's choice as its kernel runs it, on the host, for
// test_choice_search.py: a row may be another in each pass.
#include "compact.h"

// rows: `passes` versions of n numbers, the last for good. Returns the passes taken (-1:
// more than there are bits, or a counter that is none); out: the threshold, and how many of
// those equal to it are among the k.
extern "C" int search(const uint32_t *rows, int passes, int n, uint32_t k, uint32_t lo, uint32_t hi, uint32_t *out) {
  cp::Search x{lo, hi, k};
  int pass = 0;
  for (bool more = lo < hi; more; ++pass) {
    if (pass > 32) return -1;
    const uint32_t *const row = rows + (int64_t)n * (pass < passes ? pass : passes - 1);
    static uint32_t hist[cp::kBins];
    for (uint32_t &h : hist) h = 0;
    const int s = cp::search_shift(x);
    for (int i = 0; i < n; ++i)
      if (row[i] - x.lo <= x.hi - x.lo) {
        if ((row[i] - x.lo) >> s >= (uint32_t)cp::kBins) return -1;
        ++hist[(row[i] - x.lo) >> s];
      }
    uint32_t before = 0, bin = 0, left = 0, in_bin = 0;
    for (int b = cp::kBins - 1; b >= 0 && !in_bin; --b) {
      if (before < x.need && x.need <= before + hist[b]) bin = (uint32_t)b, left = x.need - before, in_bin = hist[b];
      before += hist[b];
    }
    more = cp::search_narrow(&x, bin, left, in_bin);
  }
  out[0] = x.lo;
  out[1] = x.need;
  return pass;
}
