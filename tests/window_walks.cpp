// Host check of the kernels' window arithmetic (csrc/window.hpp): every walk that the plan or the
// tile map lists for a chunk, over all small lengths, chunks, windows and tile heights, reads
// no block before the first key that its rows see, and all that they see.
#include <algorithm>
#include <cstdio>
#include <cstdlib>

#include "window.hpp"

using namespace kvattn;

static void fail(const char* what, int L, int n, int window, int rows, int q0) {
  std::printf("%s: L %d, chunk %d, window %d, %d rows from %d\n", what, L, n, window, rows, q0);
  std::exit(1);
}

// Rows q0 .. q0 + rows of a chunk of n new tokens that ends a context of L, one of them at least.
static void check(int L, int n, int window, int q0, int rows) {
  const int pos = L - n + q0, last = std::min(pos + std::min(rows, n - q0) - 1, L - 1);
  const int steps = walk_steps(pos, last, window);
  if (last < 0) {
    if (steps != 0) fail("steps of rows that see nothing", L, n, window, rows, q0);
    return;
  }
  const int seen = std::max(0, pos - window + 1);   // by the definition
  const long long from = walk_start(pos, window), end = from + 64LL * steps;
  if (from % 16) fail("not a block", L, n, window, rows, q0);
  if (from / 16 != seen / 16) fail("not the block of the first key seen", L, n, window, rows, q0);
  if (end <= last || end - 64 > last)
    fail("not the steps up to the last row", L, n, window, rows, q0);
  if (first_key(pos, window) != seen) fail("not the first key", L, n, window, rows, q0);
}

int main() {
  long long n_checked = 0;
  const int windows[] = {1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 128, 500, 1000, kNoWindow};
  for (int window : windows)
    for (int L = 0; L <= 1200; L += L < 300 ? 1 : 37)
      for (int n : {1, 2, 16, 31, 64, 100, 257, 300})   // chunks longer than their context too
        for (int rows : {1, 32, 64, 128, 256})
          for (int q0 = 0; q0 < n; q0 += rows) {
            check(L, n, window, q0, rows);
            ++n_checked;
          }
  const int far = 0x7ffffff0;   // positions near the type's end
  for (int window : windows) check(far, 64, window, 0, 64), ++n_checked;
  std::printf("ok: %lld walks\n", n_checked);
  return 0;
}
