// The shares of dX's vocabulary rows, on the host: every row of a piece once, and an empty share starts at row 0, so
// that no kernel forms an address or a range from where it would have been.
#include <stdio.h>

#include "loss_shares.h"

using namespace estp::detail;

int main() {
  int empty = 0, bad = 0;
  const int ns[] = {0, 1, 64, 65, 257, 700, 2048, 3000, 8192, 16400, 70000};
  const int ds[] = {32, 64, 1024, 1536, 2048, 4096};
  const int vcs[] = {256, 8192, 13056, 43520, 65536, 262144, 524288};
  for (int n : ns)
    for (int d : ds)
      for (int vc : vcs)
        for (int tile : {32, 64, 128, 256})
          for (int split : {1, 3, 32, 256}) {
            const size_t room = size_t(split) * size_t(n > 0 ? n : 1) * size_t(d);
            const Shares sh = dx_shares(n, d, vc, tile, 256, room);
            bool ok = sh.n >= 1 && sh.rows >= 64 && sh.rows % 64 == 0 && (n == 0 || size_t(sh.n) * n * d <= room);
            for (int live : {1, 63, 64, 100, vc / 3, vc - 1, vc}) {
              int at = 0;
              for (int s = 0; s < sh.n; ++s) {
                const Depth k = sh.depth(s, live);
                if (k.k0 == k.k1) {
                  ++empty;
                  ok = ok && k.k0 == 0;
                } else {
                  ok = ok && k.k0 == at && k.k1 > k.k0 && k.k1 - k.k0 <= sh.rows;
                  at = k.k1;
                }
              }
              ok = ok && at == live;
            }
            if (!ok && bad++ < 5) printf("n %d, d %d, piece of %d, tile %d, room for %d\n", n, d, vc, tile, split);
          }
  printf("%d empty shares, %d wrong\n", empty, bad);
  return bad != 0 || empty == 0;
}
