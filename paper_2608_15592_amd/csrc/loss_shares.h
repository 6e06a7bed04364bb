// How the vocabulary rows of a piece are shared out among the workgroups that form dX (token_loss.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

namespace estp {
namespace detail {

// Vocabulary rows [k0, k1) of a piece.
struct Depth {
  int k0, k1;
};

// Shares of a piece's vocabulary rows whose products add up to its part of dX.
struct Shares {
  int n;     // shares
  int rows;  // vocabulary rows of a share, a multiple of 64
  // of a share in a piece of `live` rows.  The last piece can be too short for all shares: one without rows is [0, 0),
  // so that the offset along k, which its transfers add to an empty resource, is 0 (of a resource shorter than that
  // offset the hardware's range check, offset >= length - scalar offset, is not known to hold).
  __host__ __device__ __forceinline__ Depth depth(int share, int live) const {
    const int k0 = share * rows;
    return k0 < live ? Depth{k0, min(live, k0 + rows)} : Depth{0, 0};
  }
};

// As many shares as give a workgroup each to the chip, while the fp32 sums of all shares (n live rows each) fit into
// `room` floats.  The same on every piece and for every kernel of a call.
__host__ __device__ __forceinline__ Shares dx_shares(int n_live, int d, int Vc, int tile_toks, int wgs, size_t room) {
  const int tiles = (n_live + tile_toks - 1) / tile_toks * ((d + 255) / 256);
  int s = tiles > 0 ? max(1, wgs / tiles) : 1;
  s = min(s, (Vc + 63) / 64);
  const size_t each = size_t(max(1, n_live)) * d, most = room / each;
  s = most < size_t(s) ? max(1, int(most)) : s;
  const int rows = ((Vc + s - 1) / s + 63) / 64 * 64;
  return {(Vc + rows - 1) / rows, rows};
}

}  // namespace detail
}  // namespace estp
