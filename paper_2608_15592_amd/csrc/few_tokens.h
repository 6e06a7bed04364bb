// Logits of few tokens (bf16), which one pass over W bounds, shared by logprobs.hip and distill.hip.
//
// 8 waves share the depth, an eighth each, and hold the tokens' part of it in registers, as the matrix cores take it, for
// the whole call.  W comes 16 rows at a time, of which a wave asks for its eighth in whole runs (512 bytes of a row at d
// 2048), with the policy of lines that are used once, straight into a ring of its own in LDS; it waits for nobody, and asks
// for the next rows as soon as its fragments are in registers: 96 to 128 KB are on their way to a compute unit.  The waves'
// sums of 16 rows meet in LDS, in the order of the waves, one barrier for every 32 tokens.
//
// Reading alone, 1.05 GB (d 4096, V 128256): runs of 1 KB with that policy 150 us (7.0 TB/s), with the ordinary one 167;
// 64 bytes of each of 16 rows, as the matrix cores take them, 174 (at d 1536, V 151936 68 us against 86).
#pragma once

#include <algorithm>
#include <type_traits>

#include "estp_common.h"
#include "lds_ops.h"

namespace estp {
namespace detail {
namespace few {

constexpr int kWaves = 8;
constexpr int kRows = 16;  // of a tile
constexpr int kWgs = 256;  // one on each compute unit

// Products of 32 k of a wave, and blocks of 16 tokens: what both take of the registers sets which calls come here.  A slot of
// the ring takes 8 KB for each of them: 16 and the sums' 32 KB fill the 160 KB of LDS.
inline int blocks_of(int64_t n) { return n <= 16 ? 1 : n <= 32 ? 2 : 4; }
inline bool takes(int64_t n_tok, int d, int dtype) {
  if (dtype != ESTP_BF16 || n_tok > 64 || d % (32 * kWaves) != 0) return false;
  const int steps = d / (32 * kWaves);
  return steps == 4 || steps == 6 || steps == 8 || ((steps == 10 || steps == 14 || steps == 16) && blocks_of(n_tok) <= 2);
}
__host__ __device__ __forceinline__ int tiles_of(int V) { return (V + kRows - 1) / kRows; }
inline unsigned workgroups(int tiles) { return unsigned(std::min(kWgs, (tiles + 1) / 2)); }

template <int kSteps, int kNB>
struct Rows {
  static constexpr int kTile = 1024 * kSteps;                 // bytes of a wave's part of a tile
  static constexpr bool kWide = kNB == 4 && kSteps < 8;         // room for the sums of all four blocks
  static constexpr int kSlots = kSteps > 8 ? 1 : (kWide ? 12 : 16) / kSteps;  // of the ring of a wave
  static constexpr int kRound = kWide ? 4 : kNB < 2 ? kNB : 2;  // blocks of tokens whose sums meet at a barrier
  static constexpr int kRing = kWaves * kSlots * kTile;
  static constexpr int kLds = kRing + 2 * kWaves * kRound * 1024;
  static constexpr int kPer = 4 * kSteps;  // 16-byte chunks of a row's eighth
  // Swizzle of the chunks of a row, so that 16 rows at one chunk lie in distinct banks.
  __device__ static __forceinline__ int swz(int row, int chunk) {
    return kPer % 16 == 0 ? chunk ^ row : chunk ^ (row >> 1);
  }
};

// Tiles 0 .. tiles - 1 of W's V rows.  take(row, z): 4 consecutive vocabulary rows' logits (rows past V: 0) of token 16 b +
// lane % 16, where waves 0 .. kNB - 1 take block b = wave; by the same thread for all rows that are equal modulo 16.  It ends
// with kStores vector-memory operations, always.
template <int kSteps, int kNB, int kStores, typename Take>
__device__ __forceinline__ void run(const __bf16* __restrict__ X, const __bf16* __restrict__ W, int n, int d, int V,
                                    int tiles, char* lds, Take&& take) {
  using R = Rows<kSteps, kNB>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ld = uint32_t(d) * 2u, part = ld / kWaves;  // bytes of a row, and of its eighth
  const int fr = lane & 15, fq = lane >> 4;
  bf16x8_t x[kNB][kSteps];
#pragma unroll
  for (int b = 0; b < kNB; ++b) {
    const int rows = max(0, min(16, n - 16 * b));
    const buf_rsrc_t r = make_rsrc(X + size_t(16 * b) * d, uint32_t(rows) * ld);
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      x[b][s] = __builtin_bit_cast(bf16x8_t, buf_load4(r, uint32_t(fr) * ld + wave * part + uint32_t(64 * s + 16 * fq)));
  }
  uint32_t src[kSteps];  // what lane `lane` of a transfer brings: chunk by chunk, row by row
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int c = 64 * s + lane, row = c / R::kPer;
    src[s] = uint32_t(row) * ld + wave * part + uint32_t(R::swz(row, c % R::kPer)) * 16u;
  }
  uint32_t at[kSteps];  // of a fragment in its slot
#pragma unroll
  for (int s = 0; s < kSteps; ++s) at[s] = uint32_t(fr * R::kPer + R::swz(fr, 4 * s + fq)) * 16u;
  char* ring = lds + wave * (R::kSlots * R::kTile);
  f32x4_t* sums = reinterpret_cast<f32x4_t*>(lds + R::kRing);
  auto fetch = [&](int64_t tile, int slot) {  // past the last tile an empty resource: no access
    const int64_t row = tile * kRows;
    const int rows = __builtin_amdgcn_readfirstlane(int(max(int64_t(0), min(int64_t(kRows), V - row))));
    const u32x4_t r = rsrc_words(W + size_t(rows > 0 ? row : 0) * d, uint32_t(rows) * ld);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) dma16<true>(r, src[s], 0, ring + slot * R::kTile + 1024 * s);
  };
  // two neighbours a workgroup in turn, where more than one is on its way (12 tokens, d 2048, V 128256: 84 us one by one, 80;
  // one token, d 4096: 155, and 167 with two)
  auto tile_of = [&](int i) {
    constexpr int kPair = R::kSlots > 1 ? 1 : 0;
    return ((int64_t(blockIdx.x) + int64_t(i >> kPair) * gridDim.x) << kPair) + (i & kPair);
  };
  wait_vm<0>();  // (the waits below count transfers alone)
#pragma unroll
  for (int i = 0; i < R::kSlots; ++i) fetch(tile_of(i), i);
  const bool takes = wave < kNB;
  int slot = 0, buf = 0, nth = 0;
  for (int64_t tile = tile_of(0); tile < tiles; tile = tile_of(++nth)) {
    // the tile has landed: what may be on its way is later tiles' transfers, and what take() has left since
    constexpr int kLater = (R::kSlots - 1) * kSteps;
    __builtin_amdgcn_sched_barrier(0);
    if (kStores > 0 && takes && nth >= R::kSlots)
      wait_vm<kLater + R::kSlots * kStores>();
    else
      wait_vm<kLater>();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_sched_barrier(0);
    bf16x8_t w[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) w[s] = *reinterpret_cast<const bf16x8_t*>(ring + slot * R::kTile + at[s]);
    lds_read_done();
    fetch(tile_of(nth + R::kSlots), slot);
    slot = slot + 1 == R::kSlots ? 0 : slot + 1;
    __builtin_amdgcn_sched_barrier(0);
    f32x4_t acc[kNB];
#pragma unroll
    for (int b = 0; b < kNB; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int b = 0; b < kNB; ++b) acc[b] = mfma_bf16(w[s], x[b][s], acc[b]);
#pragma unroll
    for (int b0 = 0; b0 < kNB; b0 += R::kRound, buf ^= 1) {
      f32x4_t* p = sums + buf * (kWaves * R::kRound * 64);
#pragma unroll
      for (int b = 0; b < R::kRound; ++b) p[(wave * R::kRound + b) * 64 + lane] = acc[b0 + b];
      lds_barrier();
      // (the other half is written next; this one only behind the barrier after that, with these reads done)
      if (wave >= b0 && wave < b0 + R::kRound) {
        f32x4_t z = p[(wave - b0) * 64 + lane];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) z += p[(v * R::kRound + wave - b0) * 64 + lane];
        take(tile * kRows + 4 * fq, z);
      }
    }
  }
  wait_vm<0>();  // no transfer into LDS outlives the workgroup
}

// The form of a call that takes() holds for: go(kSteps, kNB) as integral constants.
template <typename Go>
void choose(int n, int d, Go&& go) {
  const int nb = blocks_of(n);
  auto blocks = [&](auto s) {
    if (nb == 1)
      go(s, std::integral_constant<int, 1>{});
    else if (nb == 2)
      go(s, std::integral_constant<int, 2>{});
    else if constexpr (decltype(s)::value <= 8)
      go(s, std::integral_constant<int, 4>{});
  };
  switch (d / (32 * kWaves)) {
    case 4: return blocks(std::integral_constant<int, 4>{});
    case 6: return blocks(std::integral_constant<int, 6>{});
    case 8: return blocks(std::integral_constant<int, 8>{});
    case 10: return blocks(std::integral_constant<int, 10>{});
    case 14: return blocks(std::integral_constant<int, 14>{});
    default: return blocks(std::integral_constant<int, 16>{});
  }
}

}  // namespace few
}  // namespace detail
}  // namespace estp
