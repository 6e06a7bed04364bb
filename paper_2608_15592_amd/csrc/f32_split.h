// fp32 logits by the bf16 matrix cores, shared by logprobs.hip, distill.hip and token_loss.hip (whose dX and dW of a
// distillation form their products of the same parts).
//
// A number of 24 bits is the sum of three bf16 numbers, each what rounding has left of it: x = x1 + x2 + x3.  Of the nine
// products of two numbers' parts, six are formed: x1 w1, and apart from it, where rounding costs less, x1 w2, x2 w1, x2 w2,
// x1 w3 and x3 w1.  The other three are below 2^-26 of |x w|, a quarter of what rounding the product to fp32 may take.  So a
// logit is as exact as a chain of fp32 FMAs, at a sixth of the bf16 rate, 2.6 times that of v_mfma_f32 instructions.  (The
// third part of a number below 2^-110 is below the smallest normal one, 2^-126, and such parts may be taken as 0: numbers
// are held to 2^-24 of themselves or to 2^-126, whichever is more.)
//
// The tokens are few beside the vocabulary: their parts are written once (split_rows_kernel).  W is read as it is, and 16
// rows of a wave are split, 44 vector instructions, between the products of the 16 before them, 36 of 96 tokens.  The second
// part of an infinite number is NaN, the first is the number itself (as of those within 2^-8 of the largest): where the sum
// of x1 w1 is not finite, it is the result, infinite or NaN as products and sums of infinite numbers are.
#pragma once

#include <type_traits>

#include "estp_common.h"
#include "lds_ops.h"

namespace estp {
namespace detail {
namespace split {

constexpr int kWaves = 8;
constexpr int kRows = 256;  // vocabulary rows of a tile, 32 a wave
constexpr int kWgs = 256;   // persistent, one on each compute unit
constexpr int kDepth = 32;  // k of a stage
// Depth of the tokens' parts, with zeros past d.
__host__ __device__ __forceinline__ int padded(int d) { return (d + kDepth - 1) / kDepth * kDepth; }

__device__ __forceinline__ float top_half(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }
__device__ __forceinline__ float low_half(uint32_t pair) { return __uint_as_float(pair << 16); }

// (The compiler would round each number of a pair once more, by itself, for the difference.)
__device__ __forceinline__ uint32_t as_formed(uint32_t pair) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm("" : "+v"(pair));
#endif
  return pair;
}

// Three parts of two numbers each.
struct Parts {
  uint32_t p1, p2, p3;
};
__device__ __forceinline__ Parts parts_of(float a, float b) {
  Parts r;
  r.p1 = as_formed(pack_bf16(a, b));
  a -= low_half(r.p1);
  b -= top_half(r.p1);
  r.p2 = as_formed(pack_bf16(a, b));
  r.p3 = pack_bf16(a - low_half(r.p2), b - top_half(r.p2));
  return r;
}

// 8 numbers of a lane, as they are, and their parts, formed in 8 pieces.
struct Raw {
  float v[8];
};
struct Frag {
  uint32_t q[3][4];
  __device__ __forceinline__ bf16x8_t part(int p) const {
    return __builtin_bit_cast(bf16x8_t, uint4{q[p][0], q[p][1], q[p][2], q[p][3]});
  }
  __device__ __forceinline__ void piece(Raw& r, int j) {
    const int e = j / 2;
    float &a = r.v[2 * e], &b = r.v[2 * e + 1];
    const uint32_t pair = as_formed(pack_bf16(a, b));
    a -= low_half(pair);
    b -= top_half(pair);
    q[j % 2][e] = pair;
    if (j % 2) q[2][e] = pack_bf16(a, b);
  }
};

// A sum of products: that of x1 w1 and that of the others.
__device__ __forceinline__ float joined(float sum, float low) { return fabsf(sum) < INFINITY ? sum + low : sum; }
__device__ __forceinline__ f32x4_t joined(const f32x4_t& sum, const f32x4_t& low) {
  return f32x4_t{joined(sum[0], low[0]), joined(sum[1], low[1]), joined(sum[2], low[2]), joined(sum[3], low[3])};
}

// parts[p][row][padded(d)] of X's rows, below n (or *n_live).  Four numbers a thread.
static __global__ __launch_bounds__(256) void split_rows_kernel(const float* __restrict__ X, int n,
                                                                const int* __restrict__ n_live, int d,
                                                                __bf16* __restrict__ parts) {
  const int row = blockIdx.x, dp = padded(d);
  if (n_live && row >= *n_live) return;
  for (int k = 4 * (blockIdx.y * 256 + threadIdx.x); k < dp; k += 1024 * gridDim.y) {
    f32x4_t v{0.f, 0.f, 0.f, 0.f};
    if (k < d) v = *reinterpret_cast<const f32x4_t*>(X + size_t(row) * d + k);  // (d is a multiple of 8)
    const Parts lo = parts_of(v[0], v[1]), hi = parts_of(v[2], v[3]);
    const uint32_t at[3][2] = {{lo.p1, hi.p1}, {lo.p2, hi.p2}, {lo.p3, hi.p3}};
#pragma unroll
    for (int p = 0; p < 3; ++p)
      *reinterpret_cast<uint2*>(parts + (size_t(p) * n + row) * dp + k) = uint2{at[p][0], at[p][1]};
  }
}

// The same as the matrix cores take them where the rows are the depth: of 16 columns, a part and 32 rows (of `steps`) 1 KB,
// lane (column lane % 16) the rows 8 (lane / 16) .. + 7; zeros past the live rows.  A wave for 16 columns and 32 rows.
constexpr int kDeepRows = 96;  // that a wave holds in registers (loss_dw_split_kernel)
static __global__ __launch_bounds__(192) void split_columns_kernel(const float* __restrict__ X,
                                                                   const int* __restrict__ n_live, int d, int steps,
                                                                   __bf16* __restrict__ parts) {
  const int lane = threadIdx.x & 63, step = 3 * blockIdx.y + (threadIdx.x >> 6);
  const int col = 16 * blockIdx.x + (lane & 15), n = *n_live;
  if (step >= steps) return;
  uint32_t q[3][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int row = 32 * step + 8 * (lane >> 4) + 2 * e;
    const float a = row < n && col < d ? X[size_t(row) * d + col] : 0.f;
    const float b = row + 1 < n && col < d ? X[size_t(row + 1) * d + col] : 0.f;
    const Parts p = parts_of(a, b);
    q[0][e] = p.p1;
    q[1][e] = p.p2;
    q[2][e] = p.p3;
  }
#pragma unroll
  for (int p = 0; p < 3; ++p)
    *reinterpret_cast<uint4*>(parts + ((size_t(blockIdx.x) * 3 + p) * steps + step) * 512 + 8 * lane) =
        uint4{q[p][0], q[p][1], q[p][2], q[p][3]};
}

// Bytes of the parts of n rows.
inline size_t parts_bytes(size_t n, int d) { return 3 * n * size_t(padded(d)) * 2; }
inline size_t column_bytes(size_t n, int d) { return size_t((d + 15) / 16) * 3 * ((n + 31) / 32) * 1024; }

// 256 vocabulary rows x 16 kNB tokens by 8 waves, tile after tile.  Three stages of 32 k in LDS: two are on their way, 64 KB
// of W, while one is multiplied, across tile boundaries too.  kStream: each row of W is read once in the call.
template <int kNB, bool kStream>
struct Tile {
  static constexpr int kTN = 16 * kNB, kStages = 3;
  static constexpr int kLX = (3 * kNB + kWaves - 1) / kWaves;  // transfers of a wave of the tokens' parts
  static constexpr int kStageW = kRows * kDepth * 4, kStage = kStageW + 3 * 1024 * kNB;
  static constexpr int kLds = kStages * kStage + 1024;  // and what transfers past the last block bring, zeros
  static_assert(kLds <= 163840, "LDS of a compute unit");
  using Acc = f32x4_t[2][kNB];
  struct Place {
    int m0, n0;
  };

  // Tiles 0 .. count - 1 of the workgroup, at(i) their places; done(place, acc) takes the products.  acc[i][b][r]: logit of
  // vocabulary row m0 + 32 wave + 16 i + 4 (lane / 16) + r and token n0 + 16 b + lane % 16.  W has `rows` rows of d numbers;
  // parts as split_rows_kernel's of X's n rows, of which `live` are given.
  template <typename At, typename Done>
  __device__ static __forceinline__ void run(char* lds, const float* __restrict__ W, int rows,
                                             const __bf16* __restrict__ parts, int n, int live, int d, int count,
                                             At&& at, Done&& done) {
    if (count <= 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fr = lane & 15, fq = lane >> 4, dp = padded(d);
    uint32_t off_w[4], off_x;
    int kc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * (kWaves * i + wave) + lane / 8, c = (lane % 8) ^ ((row >> 1) & 7);
      off_w[i] = uint32_t(row) * uint32_t(d) * 4u + uint32_t(c) * 16u;
      kc[i] = 4 * c;
    }
    {
      const int row = lane / 4;  // of a block of 16 tokens
      off_x = uint32_t(row) * uint32_t(dp) * 2u + uint32_t((lane % 4) ^ ((row >> 2) & 3)) * 16u;
    }
    // the next stage to ask for: k of tile pf; past the last tile empty resources
    int pf = 0, pf_k = 0, pf_slot = 0;
    Place where = at(0);
    auto fetch = [&]() {
      char* to = lds + pf_slot * kStage;
      const bool some = pf < count;
      const Window w = window(some ? min(kRows, rows - where.m0) : 0, uint32_t(d) * 4u, uint32_t(pf_k) * 4u);
      const u32x4_t rw = rsrc_words(W + size_t(where.m0) * d, w.bytes);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        dma16<kStream>(rw, pf_k + kc[i] < d ? off_w[i] : kPastEnd, w.offset, to + 1024 * (kWaves * i + wave));
#pragma unroll
      for (int i = 0; i < kLX; ++i) {
        const int t = kWaves * i + wave, p = t / kNB, b = t % kNB;
        const int left = some && t < 3 * kNB ? min(16, live - where.n0 - 16 * b) : 0;
        const Window x = window(left, uint32_t(dp) * 2u, uint32_t(pf_k) * 2u);
        const u32x4_t r =
            rsrc_words(parts + (size_t(min(p, 2)) * n + (left > 0 ? where.n0 + 16 * b : 0)) * dp, x.bytes);
        dma16(r, off_x, x.offset, t < 3 * kNB ? to + kStageW + 1024 * t : lds + kStages * kStage);
      }
      pf_slot = pf_slot + 1 == kStages ? 0 : pf_slot + 1;
      pf_k += kDepth;
      if (pf_k >= dp) {
        pf_k = 0;
        ++pf;
        where = pf < count ? at(pf) : Place{0, 0};
      }
    };
    auto read = [&](int slot, int i) {
      const int row = 32 * wave + 16 * i + fr, g = (row >> 1) & 7;
      const char* p = lds + slot * kStage + row * 128;
      const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(p + ((2 * fq) ^ g) * 16);
      const f32x4_t hi = *reinterpret_cast<const f32x4_t*>(p + ((2 * fq + 1) ^ g) * 16);
      return Raw{{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
    };
    wait_vm<0>();  // (the waits below count transfers alone)
    fetch();
    fetch();
    fetch();
    arrived<2 * (4 + kLX)>();
    lds_barrier();
    int slot = 0;
    Frag first, second;
    {
      Raw r = read(0, 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) first.piece(r, j);
    }
    bf16x8_t x[3][kNB];
    auto read_x = [&](int of, int p, int b) {
      x[p][b] = *reinterpret_cast<const bf16x8_t*>(lds + of * kStage + kStageW + 1024 * (p * kNB + b) + fr * 64 +
                                                   (fq ^ ((fr >> 2) & 3)) * 16);
    };
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      read_x(0, 2, b);
      read_x(0, 1, b);
    }
    for (int tile = 0; tile < count; ++tile) {
      Acc acc, low;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int b = 0; b < kNB; ++b) acc[i][b] = low[i][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      // Products of 16 rows, one behind the other with what after(m) puts between them; the tokens' parts of lower
      // weight first, so that theirs can be read again early; products of one sum kNB apart, since each waits for the
      // one before it.
      auto products = [&](int i, const Frag& w, auto&& after) {
        constexpr int kW[6] = {0, 1, 0, 2, 1, 0}, kX[6] = {2, 1, 1, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < 6 * kNB; ++m) {
          const int t = m / kNB, b = m % kNB;
          f32x4_t& sum = t == 5 ? acc[i][b] : low[i][b];
          sum = mfma_bf16(w.part(kW[t]), x[kX[t]][b], sum);
          after(m);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      constexpr int kEvery = kNB > 1 ? 6 * kNB / 8 : 1, kPieces = kNB > 1 ? 1 : 2;  // pieces after each kEvery products
      for (int k = 0; k < dp; k += kDepth) {
        Raw other = read(slot, 1);
#pragma unroll
        for (int b = 0; b < kNB; ++b) read_x(slot, 0, b);
        __builtin_amdgcn_sched_barrier(0);
        products(0, first, [&](int m) {
#pragma unroll
          for (int j = 0; j < kPieces; ++j)
            if (m % kEvery == 0 && m / kEvery * kPieces + j < 8) second.piece(other, m / kEvery * kPieces + j);
        });
        // this wave's reads of the stage are done, and the next stage has landed (its successor may be in flight):
        // after the barrier nobody reads this stage's slot again
        arrived<4 + kLX>();
        lds_barrier();
        fetch();
        slot = slot + 1 == kStages ? 0 : slot + 1;
        Raw after = read(slot, 0);
        __builtin_amdgcn_sched_barrier(0);
        products(1, second, [&](int m) {
          if (m >= kNB && m < 2 * kNB) read_x(slot, 2, m - kNB);
          if (m >= 3 * kNB && m < 4 * kNB) read_x(slot, 1, m - 3 * kNB);
#pragma unroll
          for (int j = 0; j < kPieces; ++j)
            if (m % kEvery == 0 && m / kEvery * kPieces + j < 8) first.piece(after, m / kEvery * kPieces + j);
        });
      }
      const Place p = at(tile);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int b = 0; b < kNB; ++b) acc[i][b] = joined(acc[i][b], low[i][b]);
      done(p, acc);
    }
    wait_vm<0>();  // no transfer into LDS outlives the workgroup
  }
};

// Blocks of 16 tokens of a tile: by the products of a stage, and what a stage costs besides, as much as 3 blocks.
inline int blocks_of(int64_t n) {
  int best = 6;
  int64_t least = INT64_MAX;
  for (int nb : {6, 4, 3, 2, 1}) {
    const int64_t cost = (n + 16 * nb - 1) / (16 * nb) * (nb + 3);
    if (cost < least) {
      least = cost;
      best = nb;
    }
  }
  return best;
}
// The same of a tile whose depth is the vocabulary (dX).
inline int deep_blocks(int64_t n) {
  int best = 6;
  for (int nb : {4, 2})
    if ((n + 16 * nb - 1) / (16 * nb) * (nb + 3) < (n + 16 * best - 1) / (16 * best) * (best + 3)) best = nb;
  return best;
}
// go(kNB, kStream) as integral constants.
template <typename Go>
void choose(int64_t n, Go&& go) {
  const int nb = blocks_of(n);
  auto with = [&](auto b) { n <= 16 * nb ? go(b, std::true_type{}) : go(b, std::false_type{}); };
  switch (nb) {
    case 1: return with(std::integral_constant<int, 1>{});
    case 2: return with(std::integral_constant<int, 2>{});
    case 3: return with(std::integral_constant<int, 3>{});
    case 4: return with(std::integral_constant<int, 4>{});
    default: return with(std::integral_constant<int, 6>{});
  }
}
// Calls that the fp32 instructions do no faster: tiles for most compute units, of few tokens, which one pass over W bounds,
// for all of them more than once.  Log-sum-exps in us here and there: 33 tokens, d 2048, V 128256 (501 tiles) 229 and 323;
// 30 tokens, d 2048, V 50000 (196) 92 and 107; 200 tokens, d 2048, V 33000 (387) 237 and 506; 300 tokens, d 256, V 16384
// (256) 36 and 43; 400 tokens, d 512, V 5000 (100) 44 and 39; 100 tokens, d 2048, V 5000 (40) 94 and 61; one token, d 512,
// V 128256 51 and 56; 8 tokens, d 1024, V 65536 (256) 68 and 54.  (And 256 rows of W whose offsets fit 32 bits.)
inline bool takes(int64_t n, int d, int V) {
  const int64_t cols = 16 * blocks_of(n), tiles = ((int64_t(V) + kRows - 1) / kRows) * ((n + cols - 1) / cols);
  return d >= 64 && d <= (1 << 20) && tiles >= (n <= 16 ? 384 : 192);
}

}  // namespace split
}  // namespace detail
}  // namespace estp
