// The plans of estp_token_logprobs, on the host: every vocabulary tile in the sample or in one slice, a sample that fits
// its chunk, pieces whose offsets fit 32 bits, and a workspace with room for every block of a call and of smaller calls.
#include <stdio.h>

#include "logprob_plan.h"

using namespace estp::detail;

static int bad = 0;
static void check(bool ok, const char* what, long n, int V, int k) {
  if (!ok && bad++ < 8) printf("%s: %ld tokens, V %d, k %d\n", what, n, V, k);
}

int main() {
  const int Vs[] = {1, 255, 8192, 8193, 32767, 32768, 33000, 36097, 65536, 128256, 151936, 1000003, 1 << 22, 1 << 24};
  int listed = 0;
  for (int V : Vs)
    for (int k : {0, 1, 20, 128}) {
      for (int n = 1; n <= kBlockToks; n += n < 600 ? 1 : 97) {
        LogprobBuffers b;
        const PiecePlan p = plan_pieces(n, V);
        check(p.Vc >= kChunk && p.Vc % kChunk == 0 && int64_t(p.Vc) * 256 * 4 <= int64_t(1) << 32 &&
                  size_t(n) * size_t(p.Vc) <= piece_room(n, 64, V, k, 0).Z && int64_t(p.chunks) * kChunk >= V,
              "pieces", n, V, k);
        if (!use_quads(385, V, 0)) {
          check(carve_logprobs(piece_room(n, 64, V, k, 0), nullptr, &b) <= logprob_bytes(n, 64, V, k, 0), "room", n, V, k);
          continue;
        }
        if (n <= 384) {
          check(carve_logprobs(piece_room(n, 64, V, k, 0), nullptr, &b) <= logprob_bytes(n, 64, V, k, 0), "room", n, V, k);
          check(logprob_bytes(n, 64, V, k, 0) <= logprob_bytes(385, 64, V, k, 0), "grows", n, V, k);
        }
        if (n > kQuadToks) continue;
        // (the last block of a call of many tokens may be of any size)
        ++listed;
        const QuadPlan q = plan_quads(n, V, k);
        const int n_vt = (V + 255) / 256;
        check(q.slices >= 1 && q.slices <= q.n_main, "slices", n, V, k);
        check(q.sample + q.n_main == n_vt && q.sample <= kSampleTiles && (k == 0) == (q.sample == 0), "sample", n, V, k);
        if (k > 0) {
          check(q.step >= 2 && (q.sample - 1) * q.step < n_vt, "step", n, V, k);
          int other = 0, at = 0;
          for (int t = 0; t < n_vt; ++t)
            if (t % q.step != 0) {
              other += at + 1 + at / (q.step - 1) != t;  // the kernel's place of the at-th tile outside of the sample
              ++at;
            }
          check(other == 0 && at == q.n_main, "tiles", n, V, k);
        }
        const size_t need = carve_logprobs(quad_room(n, q, k), nullptr, &b);
        check(need <= logprob_bytes(std::max(n, 385), 64, V, k, 0), "room for quads", n, V, k);
        check(need <= logprob_bytes(100000, 64, V, k, 0), "room for a last block", n, V, k);
      }
    }
  printf("%d plans with quads, %d wrong\n", listed, bad);
  return bad != 0 || listed == 0;
}
