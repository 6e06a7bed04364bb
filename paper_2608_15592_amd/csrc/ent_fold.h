// The running entropy state of a token's logits in the matrix-core kernels that stream the LM head: the exponent of a weight
// and the rebased state are entropy.hip's and logprobs.hip's, the fold of a tile entropy.hip's.  (logprobs.hip has its own,
// which looks for a maximum and rebases only where a sum has grown: its logits stay in registers, a column at a time.)
#pragma once

#include "estp_common.h"

namespace estp {
namespace detail {

// Exponent of a weight, clamped to where exp2 is 0; a NaN stays one (a maximum would drop it).
__device__ __forceinline__ float exp2_arg(float x) { return x < kExp2Floor ? kExp2Floor : x; }

constexpr int kFoldBlocks = 8;  // 16-row blocks of a lane's tile

// The state relative to its log-sum-exp: m += log2 s, s = 1, t = t / s - log2 s.  (s >= 1 where a logit was seen: the
// reference never exceeds the largest, in base 2.)
__device__ __forceinline__ Ent2 rebased(Ent2 e) {
  if (e.s > 0.f) {
    const float dl = fast_log2(e.s);
    e = Ent2{e.m + dl, 1.f, e.t / e.s - dl};
  }
  return e;
}

// Fold of a finished tile into one lane's running state of one token: the lane's 32 logits z(i, r) of
// vocabulary rows 16 i + r past its first, live where 16 i + r < lim.
//
// The state (m, s, t) is kept relative to a reference m that is the running
// log-sum-exp after each tile (rebased so that s = 1).  Full tiles are then
// folded with 3 VALU ops and one exp2 per logit and no max pass; a tile whose
// logits exceed the reference by more than 2^64 in weight (or overflow) is
// refolded exactly with its own max.  The ragged last vocabulary tile always
// takes the exact, masked path.
//
// entropy_gemm_kernel holds the same steps written out: through this function its
// next-token mode kernel spilled 17 instead of 13 registers and took 1% longer
// (8192 tokens, V 151936, d 1536).  test_few_tokens_change_no_bit holds the two equal.
template <typename Z>
__device__ __forceinline__ Ent2 fold_tile(Ent2 e, bool first, bool ragged, int lim, Z&& z) {
  bool exact = ragged;
  if (!ragged) {
    if (first) {  // first tile: the tile's own max is the reference
      float mx = z(0, 0);
#pragma unroll
      for (int i = 0; i < kFoldBlocks; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, z(i, r));
      e = Ent2{mx * kLog2e, 0.f, 0.f};
    }
    float s = e.s, t = e.t;
#pragma unroll
    for (int i = 0; i < kFoldBlocks; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float dd = fmaf(z(i, r), kLog2e, -e.m);
        const float p = fast_exp2(dd);
        s += p;
        t = fmaf(p, dd, t);
      }
    if (s <= 0x1p64f) {
      e.s = s;
      e.t = t;
    } else {
      exact = true;  // overflow (or a logit far above the reference): refold exactly
    }
  }
  if (exact) {
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < kFoldBlocks; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool live = !ragged || i * 16 + r < lim;
        mx = live ? fmaxf(mx, z(i, r)) : mx;
      }
    const float mnew = fmaxf(e.m, mx * kLog2e);
    const float mref = fmaxf(mnew, -0x1p127f);  // finite for a lane with no live row yet
    const float dl = fmaxf(e.m - mnew, kExp2Floor);
    const float sc = fast_exp2(dl);
    float s = sc * e.s;
    float t = sc * (e.t + e.s * dl);
#pragma unroll
    for (int i = 0; i < kFoldBlocks; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // dead rows enter as -inf: dd clamps to the floor and adds 0 * floor
        const bool live = !ragged || i * 16 + r < lim;
        const float dd = exp2_arg(fmaf(live ? z(i, r) : -INFINITY, kLog2e, -mref));
        const float p = fast_exp2(dd);
        s += p;
        t = fmaf(p, dd, t);
      }
    e = Ent2{mnew, s, t};
  }
  return rebased(e);
}

}  // namespace detail
}  // namespace estp
