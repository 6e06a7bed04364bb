// What transfers along rows may read, on the host: within the rows that there are, and of none of them with an offset of 0
// (the fp32 products by parts); every stage of every tile once and then the first one alone (the entropy kernels).
#include <stdio.h>

#include "f32_split.h"

using namespace estp::detail;

int main() {
  int empty = 0, bad = 0;
  for (int d : {64, 72, 264, 1536, 4096, 1 << 20}) {
    const uint32_t dp = uint32_t(split::padded(d));
    for (int rows : {-1000000, -17, -1, 0, 1, 15, 16, 255, 256})
      for (uint32_t k = 0; k < dp; k += split::kDepth)
        for (uint32_t size : {4u, 2u}) {  // W's rows of d numbers, the parts' of dp
          if (size == 2 && rows > 16) continue;
          const uint32_t pitch = size == 4 ? uint32_t(d) * 4u : dp * 2u;
          const estp::Window w = estp::window(rows, pitch, k * size);
          const bool ok = rows > 0 ? uint64_t(w.bytes) == uint64_t(rows) * pitch && w.offset == k * size && w.offset < w.bytes
                                   : w.bytes == 0 && w.offset == 0;
          empty += w.bytes == 0;
          if (!ok && bad++ < 5) printf("d %d, %d rows, k %u: %u bytes at %u\n", d, rows, k, w.bytes, w.offset);
        }
  }
  for (int nk : {1, 2, 3, 7, 64})
    for (int tiles : {0, 1, 2, 5}) {
      int tile = 0, ks = 0;
      for (int i = 0; i < (tiles + 3) * nk; ++i) {
        const bool live = tile < tiles, wrap = ks + 1 == nk;
        const bool ok = live ? tile == i / nk && ks == i % nk : ks == 0;
        if (!ok && bad++ < 5) printf("%d tiles of %d stages: stage %d is %d\n", tiles, nk, i, ks);
        ks = estp::next_stage(ks, nk, live);
        tile += wrap;
      }
    }
  printf("%d empty windows, %d wrong\n", empty, bad);
  return bad != 0 || empty == 0;
}
