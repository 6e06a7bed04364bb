// Parts of the calls over the LM head that take one token at a time: the product of two rows, and the log-sum-exp of a
// token's partial states (token_loss.hip, distill.hip, logprobs.hip).
#pragma once

#include "estp_common.h"

namespace estp {
namespace detail {

// sum over 8 consecutive elements of a[k] b[k]
__device__ __forceinline__ float dot8(const __bf16* a, const __bf16* b, float s) {
  const bf16x8_t x = *reinterpret_cast<const bf16x8_t*>(a), y = *reinterpret_cast<const bf16x8_t*>(b);
#pragma unroll
  for (int k = 0; k < 8; ++k) s = fmaf(float(x[k]), float(y[k]), s);
  return s;
}
__device__ __forceinline__ float dot8(const float* a, const float* b, float s) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a + 4 * h), y = *reinterpret_cast<const f32x4_t*>(b + 4 * h);
#pragma unroll
    for (int k = 0; k < 4; ++k) s = fmaf(x[k], y[k], s);
  }
  return s;
}

// ln of 2^m s in natural units with one rounding (ln 2 in two parts): weights exp(z - lse) near 1, whose distance from 1
// is the gradient, have the error of lse.  (A NaN in s stays one.)
__device__ __forceinline__ float natural_lse(float m, float s) {
  constexpr float kLn2Rest = -1.904654299957768e-9f;
  const float t2 = fast_log2(s);
  return m == -INFINITY ? m + t2 : fmaf(m, kLn2, fmaf(m, kLn2Rest, kLn2 * t2));
}

// Natural log-sum-exp of token tok from its `states` partial (maximum, sum) states in base 2, state p at tok states + p;
// by one wave, the same in every lane.
__device__ __forceinline__ float lse_of_states(const float* __restrict__ part_m, const float* __restrict__ part_s,
                                               int tok, int states, int lane) {
  constexpr int kAhead = 8;  // states of a lane on their way together
  float M = -INFINITY, s = 0.f;
  for (int p0 = lane; p0 < states; p0 += 64 * kAhead) {
    float m[kAhead], ps[kAhead], top = M;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const size_t at = size_t(tok) * states + min(p0 + 64 * u, states - 1);
      m[u] = part_m[at];
      ps[u] = part_s[at];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const bool in = p0 + 64 * u < states;
      m[u] = in ? m[u] : -INFINITY;
      ps[u] = in ? ps[u] : 0.f;
      top = fmaxf(top, m[u]);
    }
    const float ref = fmaxf(top, -0x1p127f);
    s *= fast_exp2(fmaxf(M - ref, kExp2Floor));
#pragma unroll
    for (int u = 0; u < kAhead; ++u) s = fmaf(ps[u], fast_exp2(fmaxf(m[u] - ref, kExp2Floor)), s);
    M = top;
  }
  const float top = wave_max(M);
  s = wave_sum(s * fast_exp2(fmaxf(M - fmaxf(top, -0x1p127f), kExp2Floor)));
  return natural_lse(top, s);
}

}  // namespace detail
}  // namespace estp
