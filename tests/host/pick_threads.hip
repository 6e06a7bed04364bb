// The workgroups that form the logits of a teacher's entries, on the host: one a token fits a launch for every number of
// tokens and entries that the call takes.
#include <stdio.h>

#include "lm_head.h"

using namespace estp::detail;

int main() {
  int bad = 0, of[2] = {0, 0};
  for (size_t n = 1; n <= size_t(1) << 22; n += n < 1000 || n + 3 >= size_t(1) << 22 ? 1 : n < (size_t(1) << 22) - 5000 ? 997 : 1)
    for (int K = 1; K <= 128; ++K) {
      const int threads = pick_threads(n, K);
      if (!(threads == 256 || threads == 1024) || !estp::fits_launch(n, size_t(threads))) {
        if (bad++ < 5) printf("%zu tokens of %d entries: %d threads\n", n, K, threads);
      }
      ++of[threads == 1024];
    }
  printf("%d launches of 256 threads, %d of 1024, %d wrong\n", of[0], of[1], bad);
  return bad != 0 || !of[0] || !of[1];
}
