// Log-probabilities of given tokens under the LM head, with the entropy of their distributions and the most probable
// alternatives.
//
//   z_i = W x_i,  s_i = z_i / temperature,  lse_i = log sum_v exp s_i[v],  logprob_i = s_i[t_i] - lse_i
//   H_i = lse_i - sum_v exp(s_i[v] - lse_i) s_i[v]
//   top_i = the k largest z_i[v], descending, the lowest v first among equals
//
// Few tokens, and fp32 (launch_pieces): the logits of a block of tokens over a piece of the vocabulary are formed by the
// matrix cores and kept in fp32 (logits_few_kernel, where one pass over W bounds the call; logits_mfma_kernel;
// logits_split_kernel, logits_f32_kernel); logprob_select_kernel makes of each chunk of a row a partial state and its k
// largest logits; logprob_merge_kernel joins a row's chunks.
//
// Many tokens of bf16 (launch_quads): to write and read again 4 bytes a logit would cost as much as half of the products.
// So a sample of the vocabulary's tiles gives a lower bound of each token's k-th largest logit, by the two kernels above,
// and the products of all other tiles end in the partial states and in the few logits that reach the bound
// (logprob_main_kernel), which logprob_merge_kernel ranks.  8192 tokens, d 4096, V 128256, 64 alternatives: 6.4 to 6.7 ms,
// 1.28 to 1.34 PFLOP/s over all of it; 5.9 ms is what a plain product of this size takes at the card's best rate.
#include <algorithm>
#include <type_traits>

#include "ent_fold.h"
#include "estp_common.h"
#include "f32_gemm.h"
#include "f32_split.h"
#include "few_tokens.h"
#include "lm_head.h"
#include "logprob_plan.h"
#include "lse_states.h"
#include "mfma_gemm.h"
#include "top_k.h"

namespace estp {
namespace detail {

// ------------------------------------------------------------------ logits

// Z[token][v] of n_m vocabulary tiles, every `step`-th from row v0 (rows past V: 0), pitch Vc.  M side: vocabulary rows.
// A lane holds 8 consecutive vocabulary rows of a token: two 16-byte stores.  Bound by the matrix cores and the stores: a
// sample of 39 tiles, 2048 tokens, d 4096, 109 us, 1.54 PFLOP/s; of 1511 tokens, d 2048, which 240 workgroups of 256 share
// a tile each, 69.
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void logits_mfma_kernel(const __bf16* __restrict__ X,
                                                             const __bf16* __restrict__ W, int n, int d, int V,
                                                             int64_t v0, int n_m, int step, int Vc,
                                                             float* __restrict__ Z) {
  using Run = gemm::Tiles<true, true, true, kNBN, kOdd, 8 * kNBN < 48 ? 8 * kNBN : 48, kNBN == 4>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n_n = (n + Run::kBN - 1) / Run::kBN;
  const gemm::TileOrder order(n_m, n_n);
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 2u, int(V - v0)};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 2u, n};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  Run::run(
      lds, A, B, gemm::first_tile(blockIdx.x, gridDim.x), gridDim.x, n_m * n_n,
      [&](int id) {
        const gemm::TileAt t = order(id);
        return gemm::Place{256 * step * t.m, Run::kBN * t.n, 0, d, 256 * t.m};
      },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][kNBN]) {
        const int lane = gemm::fresh_lane(), fr = lane & 15, fq = lane >> 4;
        const int live = min(Run::kBN, n - at.n0);
        const buf_rsrc_t out = make_rsrc(Z + size_t(at.n0) * Vc, uint32_t(live) * uint32_t(Vc) * 4u);
        const int c0 = at.tag + 128 * wm + 8 * fq;
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          const uint32_t row = uint32_t(16 * kNBN * wn + 16 * j + fr) * uint32_t(Vc);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            buf_store16(out, (row + uint32_t(c0 + 32 * (i / 2) + 4 * (i % 2))) * 4u,
                        __builtin_bit_cast(uint4, acc[i][j]));
        }
      });
}

// Z[v / 32][token][v % 32] of few tokens and all of the vocabulary: the logits of two tiles, a workgroup's, lie together.
// Bound by the bytes of W: one token, d 4096, V 128256 155 us, 6.8 TB/s; 48 tokens, d 1536, V 151936 88 us, 5.3 TB/s, and
// 29 MB of logits besides.
template <int kSteps, int kNB>
__global__ __launch_bounds__(64 * few::kWaves, 2) void logits_few_kernel(const __bf16* __restrict__ X,
                                                                         const __bf16* __restrict__ W, int n, int d,
                                                                         int V, float* __restrict__ Z) {
  __shared__ __attribute__((aligned(16))) char lds[few::Rows<kSteps, kNB>::kLds];
  const int tok = threadIdx.x / 64 * 16 + (threadIdx.x & 15);
  few::run<kSteps, kNB, 1>(X, W, n, d, V, few::tiles_of(V), lds, [&](int64_t row, f32x4_t z) {
    const buf_rsrc_t out = make_rsrc(Z + size_t(row & ~int64_t(31)) * n, uint32_t(n) * 128u);
    buf_store16(out, uint32_t(tok) * 128u + uint32_t(row & 31) * 4u, __builtin_bit_cast(uint4, z));
  });
}

template <int kTN>
__global__ __launch_bounds__(256, 2) void logits_f32_kernel(const float* __restrict__ X, const float* __restrict__ W,
                                                            int n, int d, int V, int64_t v0, int Vc,
                                                            float* __restrict__ Z) {
  using Run = F32Tile<true, true, kTN>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int n0 = blockIdx.y * kTN, m0 = blockIdx.x * kFT;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  if (m0 >= rows) return;
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 4u, rows};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 4u, n};
  typename Run::Acc acc;
  Run::run(lds, A, B, m0, n0, 0, d, acc);
  const auto at = Run::place(m0, n0);
#pragma unroll
  for (int j = 0; j < Run::kNJ; ++j) {
    const int s = at.n + 32 * j;
    if (s >= n) continue;
#pragma unroll
    for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4_t*>(Z + size_t(s) * Vc + at.m + 32 * i + 8 * q) =
            f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
  }
}

// The same of vocabulary rows v0 .. v0 + Vc by the bf16 matrix cores.  37 tokens, d 2048, V 128256: 237 us, 4.4 TB/s of W
// (323 by the fp32 instructions); 48 columns' products, 121 GF in bf16, and the splitting of W take about as long as W.
template <int kNB, bool kStream>
__global__ __launch_bounds__(64 * split::kWaves, 2) void logits_split_kernel(const __bf16* __restrict__ parts,
                                                                             const float* __restrict__ W, int n, int d,
                                                                             int V, int64_t v0, int Vc,
                                                                             float* __restrict__ Z) {
  using Run = split::Tile<kNB, kStream>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  const int n_vt = (rows + split::kRows - 1) / split::kRows, n_tt = (n + Run::kTN - 1) / Run::kTN;
  // (the token tiles of a vocabulary tile next to each other on one XCD)
  const int first = gemm::first_tile(blockIdx.x, gridDim.x), total = n_vt * n_tt;
  Run::run(
      lds, W + size_t(v0) * d, rows, parts, n, n, d, first < total ? (total - first - 1) / int(gridDim.x) + 1 : 0,
      [&](int i) {
        const int id = first + i * int(gridDim.x);
        return typename Run::Place{id / n_tt * split::kRows, id % n_tt * Run::kTN};
      },
      [&](const typename Run::Place& at, const typename Run::Acc& acc) {
        const int lane = threadIdx.x & 63, row = at.m0 + 32 * int(threadIdx.x >> 6) + 4 * (lane >> 4);
#pragma unroll
        for (int b = 0; b < kNB; ++b) {
          const int tok = at.n0 + 16 * b + (lane & 15);
          if (tok >= n) continue;
#pragma unroll
          for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4_t*>(Z + size_t(tok) * Vc + row + 16 * i) = acc[i][b];
        }
      });
}

// ------------------------------------------------------------------ many tokens: what may be among the largest
//
// With a bound of each token's k-th largest logit from a sample of the vocabulary's tiles, the products of the other
// tiles leave behind only the logits that reach it, a quad of four rows at a time: some k V / sample of each token's V.
// They go where all would go, and a bit says of each quad whether it was written, so there is room for any number of
// them, nothing is counted across lanes, and no order depends on which workgroup runs first.

// The next fp32 number above x (of the largest, infinity; of infinity, a NaN).
__device__ __forceinline__ float next_up(float x) {
  const uint32_t u = __float_as_uint(x);
  return __uint_as_float(u >> 31 ? u - 1 : u + 1);
}

// The largest of four sums (a NaN only of four).
__device__ __forceinline__ float largest(const float (&z)[4]) {
#if defined(__HIP_DEVICE_COMPILE__)
  float m;  // (fmaxf would make each operand canonical first)
  asm("v_max3_f32 %0, %1, %2, %3\n\tv_max_f32 %0, %0, %4" : "=&v"(m) : "v"(z[0]), "v"(z[1]), "v"(z[2]), "v"(z[3]));
  return m;
#else
  return z[0];
#endif
}
// A number formed by now: what it is made of is not kept for later.
__device__ __forceinline__ uint32_t settled(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
  return v;
}

// A sum of weights past this is folded again, relative to the tile's own maximum, and the state then taken relative to its
// log-sum-exp.  H is log2 s - t / s, off by some units in the last place of log2 s: of 10 bits at most so.  (With 2^64 a mode
// some 20 bits above the first tile made H off by 2^-19.)  Rows without a mode stay below it, one refold in 1024 tiles.  2048
// tokens, d 2048, V 128256, temperature 0.7, modes up to 17 nats above the rest: H is 1.1e-7 off relative to 64 bits over all
// and 1.3e-4 in the worst row (1.5e-6 and 2.6e-3 with 2^64, a plain sum in fp32 4.4e-7 and 1.4e-3), in the same time.
constexpr float kFoldRoom = 0x1p10f;

// Workgroup (token tile, slice) takes the vocabulary tiles slice, slice + n_slices, ... of those that are not in the
// sample (every `step`-th; step 0: no sample).  Partial states 2 slice + wave row of the last 2 n_slices of `states` a token.
// kTop: quads that reach the logit of bounds[token k + k - 1], and their bits.
//
// What follows a tile's products is a branch only where a state is refolded: a quad that is not wanted is stored past the
// end of the resource.  (With a branch and a list for each, sums were moved to memory and back: 125 us a tile of d 4096,
// V 128256, and 93 without.)  Bound by the matrix cores: 2048 tokens, d 4096, the 462 tiles that are not in a sample of 39
// of V 128256: 1410 us, 1.41 PFLOP/s, where the same products end in a log-sum-exp alone at 1.58; the rest is the entropy's
// second sum, the comparisons and the stores.
template <bool kOdd, bool kTop>
__global__ __launch_bounds__(256, 1) void logprob_main_kernel(const __bf16* __restrict__ X,
                                                              const __bf16* __restrict__ W, int n, int d, int V,
                                                              float c2, int n_tt, int n_slices, int step, int n_main,
                                                              int k, const uint64_t* __restrict__ bounds, int states,
                                                              float* __restrict__ part, Quads quads) {
  using Run = gemm::Tiles<true, true, false, 8, kOdd, kTop ? 48 : 0>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const gemm::SliceAt wg = gemm::slice_of(gemm::first_tile(blockIdx.x, gridDim.x), n_tt, n_slices);
  const int tt = wg.tile, slice = wg.slice;
  if (slice >= n_slices) return;
  const gemm::Operand A{reinterpret_cast<const char*>(W), uint32_t(d) * 2u, V};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 2u, n};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  const int n_mine = (n_main - slice + n_slices - 1) / n_slices;
  const gemm::Divisor between(uint32_t(max(1, step - 1)));  // tiles between two of the sample
  Ent2 st[8];
  float from[8];  // what a logit has to reach
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    st[j] = Ent2{-INFINITY, 0.f, 0.f};
    const int tok = 256 * tt + 128 * wn + 16 * j + (threadIdx.x & 15);
    from[j] = __uint_as_float(0x7fc00000u);
    if (kTop && tok < n) {
      // a bound from the first tile, below all of these, has to be exceeded; one of NaN keeps whatever is not NaN out
      const uint64_t key = bounds[size_t(tok) * k + k - 1];
      const float z = logit_of(key);
      from[j] = z != z ? -INFINITY : id_of(key) < 256 ? next_up(z) : z;
    }
  }
  Run::run(
      lds, A, B, 0, 1, n_mine,
      [&](int i) {
        const int at = slice + i * n_slices, vt = step ? at + 1 + int(between.div(uint32_t(at))) : at;
        return gemm::Place{256 * vt, 256 * tt, 0, d, i};
      },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][8]) {
        const int lane = gemm::fresh_lane(), fr = lane & 15, fq = lane >> 4;
        const bool ragged = at.m0 + 256 > V;
        const int lim = V - (at.m0 + 128 * wm + 4 * fq);  // live rows: 16 i + r < lim
        const int place = slice + at.tag * n_slices;
        const buf_rsrc_t out = make_rsrc(quads.z + (size_t(tt) * n_main + place) * kQuadTile, kTop ? kQuadTile * 4 : 0);
        uint32_t bits[2] = {0, 0};  // byte j % 4 of bits[j / 4]: bit i
        gemm::sums_ready();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float z[8][4];
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) z[i][r] = gemm::read_sum(acc[i][j][r]);
          if constexpr (kTop) {
            const uint32_t row = uint32_t(128 * wn + 16 * j + fr) * 1024u + uint32_t(128 * wm + 4 * fq) * 4u;
            uint32_t mine = bits[j / 4];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const bool hit = largest(z[i]) >= from[j];
              mine |= hit ? 1u << (8 * (j % 4) + i) : 0u;
              buf_store16(out, (hit ? row : 0x80000000u) + 64u * i,
                          __builtin_bit_cast(uint4, f32x4_t{z[i][0], z[i][1], z[i][2], z[i][3]}));
            }
            bits[j / 4] = settled(mine);
          }
          Ent2 e = st[j];
          bool exact = ragged || at.tag == 0;
          if (!exact) {
            float s = e.s, t = e.t;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float dd = fmaf(z[i][r], c2, -e.m), p = fast_exp2(dd);
                s += p;
                t = fmaf(p, dd, t);
              }
            // (a logit of -inf makes t NaN, 0 times its exponent, which the exact path clamps; a NaN stays one there)
            exact = !(s <= kFoldRoom && t == t);
            e.s = exact ? e.s : s;
            e.t = exact ? e.t : t;
          }
          if (exact) {
            float mx = e.m;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) mx = fmaxf(mx, 16 * i + r < lim ? z[i][r] * c2 : -INFINITY);
            const float ref = fmaxf(mx, -0x1p127f);  // finite for a lane with no live row yet
            const float dl = fmaxf(e.m - ref, kExp2Floor), sc = fast_exp2(dl);
            float s = sc * e.s, t = sc * fmaf(e.s, dl, e.t);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float dd = exp2_arg(fmaf(16 * i + r < lim ? z[i][r] : -INFINITY, c2, -ref)), p = fast_exp2(dd);
                s += p;
                t = fmaf(p, dd, t);
              }
            e = rebased(Ent2{mx, s, t});
          }
          st[j] = e;
        }
        if constexpr (kTop) {
          // lane (fq, fr) takes tokens 2 fq and 2 fq + 1 of the eight blocks: a word of each, byte q from lane (q, fr)
          uint32_t word[2] = {0, 0};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t lo = __shfl(bits[0], 16 * q + fr, 64), hi = __shfl(bits[1], 16 * q + fr, 64);
            const uint32_t both = (fq & 2 ? hi : lo) >> (16 * (fq & 1));
            word[0] |= (both & 0xffu) << (8 * q);
            word[1] |= (both >> 8 & 0xffu) << (8 * q);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const size_t tok = size_t(256) * tt + 128 * wn + 16 * (2 * fq + e) + fr;  // (whole tiles have room)
            quads.bits[tok * (2 * n_main) + 2 * place + wm] = word[e];
          }
        }
      });
  const int lane = threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int tok = 256 * tt + 128 * wn + 16 * j + fr;
    // lanes l, l ^ 16, l ^ 32, l ^ 48 hold the same tokens
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1)
      st[j] = ent2_merge(st[j], Ent2{__shfl_xor(st[j].m, o, 64), __shfl_xor(st[j].s, o, 64), __shfl_xor(st[j].t, o, 64)});
    if (fq == 0 && tok < n) {
      float* p = part + 3 * (size_t(tok) * states + states - 2 * n_slices + 2 * slice + wm);
      p[0] = st[j].m;
      p[1] = st[j].s;
      p[2] = st[j].t;
    }
  }
}

// ------------------------------------------------------------------ selection

// Partial state (base 2) and the k largest logits of 256 kE columns of Z's row, chunk `chunk0 + c` of the token's.  32
// columns lie together, those of a token `of_tok` apart, and the next of the same token `of_32` on.  Column c is vocabulary
// row v0 + c, or of every `step`-th tile of 256.  One workgroup each, with its logits in registers: they are read once.
// One token's 16 chunks of 8192: 6 us, latency; 48 tokens, 19 chunks: 13.5 (29 MB, from L2 or the last cache); 2048 tokens'
// samples, 84 MB: 31, 2.7 TB/s, what the barriers of the bound and of the ranking leave.
template <int kE>
__global__ __launch_bounds__(256) void logprob_select_kernel(const float* __restrict__ Z, int of_tok, int of_32,
                                                             int live, int64_t v0, int step, float c2, int k,
                                                             int piece_chunks, int chunk0, int states, int chunks,
                                                             float* __restrict__ part, uint64_t* __restrict__ top) {
  __shared__ TopK<kMaxTop * kE> pick;
  __shared__ float wave_m[4], wave_s[4], wave_t[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tok = blockIdx.x / piece_chunks, c = blockIdx.x % piece_chunks;
  const float* row = Z + size_t(tok) * of_tok;
  const int first = 256 * kE * c + 4 * tid;  // columns first + 1024 u + e, ascending in 4 u + e
  f32x4_t z[kE / 4];
#pragma unroll
  for (int u = 0; u < kE / 4; ++u)
    z[u] = *reinterpret_cast<const f32x4_t*>(row + size_t((first + 1024 * u) >> 5) * of_32 + (first & 31));
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < kE / 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[u][e] = first + 1024 * u + e < live ? z[u][e] : -INFINITY;
      m = fmaxf(m, z[u][e]);
    }
  const float mine = m;
  m = wave_max(m);
  if (lane == 0) wave_m[wave] = m;
  if (tid == 0) pick.count = 0;
  __syncthreads();
  m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3])) * c2;
  const float ref = fmaxf(m, -0x1p127f);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int u = 0; u < kE / 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float dd = exp2_arg(fmaf(z[u][e], c2, -ref)), p = fast_exp2(dd);
      s += p;
      t = fmaf(p, dd, t);
    }
  s = wave_sum(s);
  t = wave_sum(t);
  if (lane == 0) {
    wave_s[wave] = s;
    wave_t[wave] = t;
  }
  __syncthreads();
  s = wave_s[0] + wave_s[1] + wave_s[2] + wave_s[3];
  if (tid == 0) {
    float* p = part + 3 * (size_t(tok) * states + chunk0 + c);
    p[0] = m;
    p[1] = s;
    p[2] = wave_t[0] + wave_t[1] + wave_t[2] + wave_t[3];
  }
  if (k == 0) return;
  auto id = [&](int e) {
    const int col = first + 1024 * (e / 4) + e % 4;
    return int(v0) + (col >> 8) * 256 * step + (col & 255);
  };
  const float reach = pick.bound_of(first < live ? ascending(mine) : 0u, k);
  if (reach == reach && s == s) {  // as a rule: numbers, and different ones where it matters
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (z[e / 4][e % 4] >= reach)
        pick.list[atomicAdd(&pick.count, 1)] = key_of(ascending(z[e / 4][e % 4]), id(e));
  } else {
    uint32_t up[kE], most = 0;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      up[e] = first + 1024 * (e / 4) + e % 4 < live ? ascending(z[e / 4][e % 4]) : 0;
      most = max(most, up[e]);
    }
    int which = 0;
#pragma unroll
    for (int e = kE - 1; e >= 0; --e) which = up[e] == most ? e : which;  // the lowest
    const uint64_t from = pick.bound_of(most ? key_of(most, id(which)) : uint64_t(0), k);
#pragma unroll
    for (int e = 0; e < kE; ++e)
      if (up[e] >= uint32_t(from >> 32) && key_of(up[e], id(e)) >= from && up[e])
        pick.list[atomicAdd(&pick.count, 1)] = key_of(up[e], id(e));
  }
  __syncthreads();
  uint64_t* out = top + (size_t(tok) * chunks + chunk0 + c) * k;
  const int n = pick.count;
  if (tid >= n && tid < k) out[tid] = 0;  // (fewer columns than k)
  pick.rank(n, k, [&](int r, uint64_t v) { out[r] = v; });
}

// A token's outputs from its `states` partial states and from the k largest of each of its `chunks` chunks, or (kQuads)
// from the k largest of the sample and the quads that reach them.  One workgroup each; latency: bits, then quads, then the
// ranking, each behind the other.  One token 5 us; 1511 tokens with 5 alternatives 24; 2048 with 64, some 800 quads each,
// 71 (16-byte reads far apart).
template <typename T, bool kQuads>
__global__ __launch_bounds__(256) void logprob_merge_kernel(const T* __restrict__ X, const T* __restrict__ W,
                                                            const int32_t* __restrict__ targets, int d, int V, int k,
                                                            float inv_t, int states, const float* __restrict__ part,
                                                            int chunks, const uint64_t* __restrict__ top, Quads quads,
                                                            int n_main, int step,
                                                            float* __restrict__ logprob, float* __restrict__ lse,
                                                            float* __restrict__ H, int32_t* __restrict__ top_id,
                                                            float* __restrict__ top_logprob) {
  constexpr int kCap = kQuads ? 12 * 256 : 2048;
  __shared__ TopK<kCap> pick;
  __shared__ uint64_t best[kMaxTop];
  __shared__ float wave_z[4];
  __shared__ Ent2 wave_state[4];
  __shared__ bool among;  // the given token is an alternative
  const int tok = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the given token's logit
  const int t = targets ? targets[tok] : -1;
  const bool live = t >= 0 && t < V;
  float z = 0.f;
  if (live)
    for (int i = 8 * tid; i < d; i += 2048) z = dot8(X + size_t(tok) * d + i, W + size_t(t) * d + i, z);
  z = wave_sum(z);
  Ent2 a{-INFINITY, 0.f, 0.f};
  for (int c = tid; c < states; c += 256) {
    const float* p = part + 3 * (size_t(tok) * states + c);
    a = ent2_merge(a, Ent2{p[0], p[1], p[2]});
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
    a = ent2_merge(a, Ent2{__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)});
  if (lane == 0) {
    wave_z[wave] = z;
    wave_state[wave] = a;
  }
  if (tid == 0) among = false;
  __syncthreads();
  z = wave_z[0] + wave_z[1] + wave_z[2] + wave_z[3];
  a = ent2_merge(ent2_merge(wave_state[0], wave_state[1]), ent2_merge(wave_state[2], wave_state[3]));
  const float l = natural_lse(a.m, a.s);
  if (tid < k) best[tid] = 0;
  const uint64_t* from = top + size_t(tok) * chunks * k;
  if constexpr (kQuads) {
    // A thread reads the bits of up to kWords half tiles, and lists their quads; then the threads share these out,
    // kAhead each and round.  What exceeds the bound joins the keys, which are cut to the k largest where the next round
    // could pass their end.  (Quads that do not fit their list are taken by the thread that read their bits.)
    constexpr int kWords = 4, kAhead = 2, kCodes = 1536;
    __shared__ uint32_t code[kCodes];
    __shared__ int codes;
    if (tid < k) pick.list[tid] = from[tid];
    if (tid == 0) pick.count = k;
    uint64_t bound = k > 0 ? from[k - 1] : 0;
    const int words = k > 0 ? 2 * n_main : 0;
    const uint32_t* bits = quads.bits + size_t(tok) * words;
    const float* zt = quads.z + size_t(tok / 256) * n_main * kQuadTile + tok % 256 * 256;
    for (int w0 = 0; w0 < words; w0 += 256 * kWords) {
      uint32_t left[kWords];
      int n = 0;
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        left[u] = w0 + 256 * u + tid < words ? bits[w0 + 256 * u + tid] : 0;
        n += __popc(left[u]);
      }
      if (tid == 0) codes = 0;
      __syncthreads();
      int at = n > 0 ? atomicAdd(&codes, n) : 0;
#pragma unroll
      for (int u = 0; u < kWords; ++u)
        for (; left[u] && at < kCodes; ++at) {
          const uint32_t b = __ffs(left[u]) - 1;
          code[at] = uint32_t(256 * u + tid) << 5 | b;
          left[u] &= left[u] - 1;
        }
      __syncthreads();
      const int listed = min(codes, kCodes);
      bool more = false;
#pragma unroll
      for (int u = 0; u < kWords; ++u) more |= left[u] != 0;
      for (int c0 = 0; __syncthreads_or(c0 < listed || more); c0 += 256 * kAhead) {
        f32x4_t z[kAhead];
        int row[kAhead];  // its first vocabulary row, -1: none
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int c = c0 + 256 * u + tid;
          uint32_t own = 0xffffffffu;
          if (c < listed) {
            own = code[c];
          } else if (c0 >= listed && more) {
            more = false;
#pragma unroll
            for (int w = kWords - 1; w >= 0; --w)
              if (left[w]) own = uint32_t(256 * w + tid) << 5 | uint32_t(__ffs(left[w]) - 1);
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
              if (int(own >> 5) == 256 * w + tid) left[w] &= left[w] - 1;
              more |= left[w] != 0;
            }
          }
          row[u] = -1;
          if (own != 0xffffffffu) {
            const int word = w0 + int(own >> 5), b = int(own & 31u), place = word >> 1;
            const int col = 128 * (word & 1) + 16 * (b & 7) + 4 * (b >> 3);
            z[u] = *reinterpret_cast<const f32x4_t*>(zt + size_t(place) * kQuadTile + col);
            row[u] = 256 * (place + 1 + place / (step - 1)) + col;
          }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (row[u] >= 0 && row[u] + e < V) {
              const uint64_t key = key_of(ascending(z[u][e]), row[u] + e);
              if (key > bound) pick.list[atomicAdd(&pick.count, 1)] = key;
            }
        __syncthreads();
        if (pick.count > kCap - 256 * 4 * kAhead) {
          pick.rank(pick.count, k, [&](int r, uint64_t v) { best[r] = v; });
          __syncthreads();
          if (tid < k) pick.list[tid] = best[tid];
          if (tid == 0) pick.count = k;
          bound = best[k - 1];
        }
      }
    }
    __syncthreads();
    if (k > 0) pick.rank(pick.count, k, [&](int r, uint64_t v) { best[r] = v; });
    __syncthreads();
  } else {
    // as many at a time as the list takes with those so far
    int have = 0;
    for (size_t at = 0, total = size_t(chunks) * k; at < total;) {
      const int now = int(min(total - at, size_t(kCap - have)));
      if (tid < have) pick.list[tid] = best[tid];
      for (int i = tid; i < now; i += 256) pick.list[have + i] = from[at + i];
      __syncthreads();
      pick.rank(have + now, k, [&](int r, uint64_t v) { best[r] = v; });
      __syncthreads();
      at += now;
      have = k;
    }
  }
  if (tid < k) {
    const uint64_t key = best[tid];
    const float zk = logit_of(key);
    top_id[size_t(tok) * k + tid] = id_of(key);
    top_logprob[size_t(tok) * k + tid] = fmaf(zk, inv_t, -l);
    if (live && id_of(key) == t) {  // one value of the given token, whichever output it is read from
      wave_z[0] = zk;
      among = true;
    }
  }
  __syncthreads();
  if (tid == 0) {
    if (logprob) logprob[tok] = live ? fmaf(among ? wave_z[0] : z, inv_t, -l) : 0.f;
    if (lse) lse[tok] = l;
    if (H) H[tok] = kLn2 * (fast_log2(a.s) - a.t / a.s);
  }
}

// ------------------------------------------------------------------ launches

template <typename T>
int launch_pieces(const T* X, const T* W, const int32_t* targets, int n, int d, int V, int k, float temperature,
                  void* workspace, float* logprob, float* lse, float* H, int32_t* top_id, float* top_logprob,
                  hipStream_t s) {
  const PiecePlan p = plan_pieces(n, V);
  LogprobBuffers b;
  carve_logprobs(piece_room(n, d, V, k, sizeof(T) == 4 ? ESTP_F32 : ESTP_BF16), workspace, &b);
  const float c2 = base2_of_logit(temperature), inv_t = inverse_temperature(temperature);
  const dim3 block(256);
  bool tiled = false;
  for (int64_t v0 = 0; v0 < V; v0 += p.Vc) {
    const int rows = int(std::min<int64_t>(V - v0, p.Vc));
    if constexpr (sizeof(T) == 2) {
      tiled = p.Vc >= V && few::takes(n, d, ESTP_BF16);
      if (tiled) {
        few::choose(n, d, [&](auto steps, auto nb) {
          logits_few_kernel<decltype(steps)::value, decltype(nb)::value>
              <<<dim3(few::workgroups(few::tiles_of(V))), dim3(64 * few::kWaves), 0, s>>>(X, W, n, d, V, b.Z);
        });
      } else {
        const bool odd = d % 64 != 0, narrow = n <= 384;
        auto kernel = narrow ? (odd ? logits_mfma_kernel<4, true> : logits_mfma_kernel<4, false>)
                             : (odd ? logits_mfma_kernel<8, true> : logits_mfma_kernel<8, false>);
        kernel<<<dim3(256), block, 0, s>>>(X, W, n, d, V, v0, (rows + 255) / 256, 1, p.Vc, b.Z);
      }
    } else {
      if (split::takes(n, d, V)) {
        if (v0 == 0)
          split::split_rows_kernel<<<dim3(unsigned(n)), block, 0, s>>>(X, n, nullptr, d, b.parts);
        split::choose(n, [&](auto nb, auto stream) {
          logits_split_kernel<decltype(nb)::value, decltype(stream)::value>
              <<<dim3(split::kWgs), dim3(64 * split::kWaves), 0, s>>>(b.parts, W, n, d, V, v0, p.Vc, b.Z);
        });
      } else {
        const int tile = n <= 32 ? 32 : n <= 64 ? 64 : kFT;
        auto kernel = tile == 32 ? logits_f32_kernel<32> : tile == 64 ? logits_f32_kernel<64> : logits_f32_kernel<kFT>;
        kernel<<<dim3(unsigned((rows + kFT - 1) / kFT), unsigned((n + tile - 1) / tile)), block, 0, s>>>(
            X, W, n, d, V, v0, p.Vc, b.Z);
      }
    }
    ESTP_CHECK_LAUNCH("logits_kernel");
    const int in_piece = (rows + kChunk - 1) / kChunk;
    logprob_select_kernel<kChunk / 256><<<dim3(unsigned(n) * unsigned(in_piece)), block, 0, s>>>(
        b.Z, tiled ? 32 : p.Vc, tiled ? 32 * n : 32, rows, v0, 1, c2, k, in_piece, int(v0 / kChunk), p.chunks, p.chunks, b.part, b.top);
    ESTP_CHECK_LAUNCH("logprob_select_kernel");
  }
  logprob_merge_kernel<T, false><<<dim3(unsigned(n)), block, 0, s>>>(X, W, targets, d, V, k, inv_t, p.chunks, b.part,
                                                                     p.chunks, b.top, b.quads, 0, 0, logprob, lse, H,
                                                                     top_id, top_logprob);
  ESTP_CHECK_LAUNCH("logprob_merge_kernel");
  return ESTP_OK;
}

int launch_quads(const __bf16* X, const __bf16* W, const int32_t* targets, int n, int d, int V, int k,
                 float temperature, void* workspace, float* logprob, float* lse, float* H, int32_t* top_id,
                 float* top_logprob, hipStream_t s) {
  const QuadPlan p = plan_quads(n, V, k);
  LogprobBuffers b;
  carve_logprobs(quad_room(n, p, k), workspace, &b);
  const float c2 = base2_of_logit(temperature), inv_t = inverse_temperature(temperature);
  const bool odd = d % 64 != 0;
  const dim3 block(256);
  const int states = (k > 0) + 2 * p.slices, n_tt = (n + 255) / 256;
  if (k > 0) {
    auto kernel = odd ? logits_mfma_kernel<8, true> : logits_mfma_kernel<8, false>;
    kernel<<<dim3(256), block, 0, s>>>(X, W, n, d, V, 0, p.sample, p.step, 256 * kSampleTiles, b.Z);
    ESTP_CHECK_LAUNCH("logits_kernel");
    const int live = 256 * (p.sample - 1) + std::min(256, V - 256 * p.step * (p.sample - 1));
    logprob_select_kernel<kSampleTiles><<<dim3(unsigned(n)), block, 0, s>>>(b.Z, 256 * kSampleTiles, 32, live, 0, p.step, c2,
                                                                            k, 1, 0, states, 1, b.part, b.top);
    ESTP_CHECK_LAUNCH("logprob_select_kernel");
  }
  auto main = k > 0 ? (odd ? logprob_main_kernel<true, true> : logprob_main_kernel<false, true>)
                    : (odd ? logprob_main_kernel<true, false> : logprob_main_kernel<false, false>);
  main<<<dim3(unsigned((n_tt * p.slices + 7) / 8 * 8)), block, 0, s>>>(X, W, n, d, V, c2, n_tt, p.slices, p.step,
                                                                       p.n_main, k, b.top, states, b.part, b.quads);
  ESTP_CHECK_LAUNCH("logprob_main_kernel");
  logprob_merge_kernel<__bf16, true><<<dim3(unsigned(n)), block, 0, s>>>(X, W, targets, d, V, k, inv_t, states, b.part,
                                                                         1, b.top, b.quads, p.n_main, p.step, logprob, lse,
                                                                         H, top_id, top_logprob);
  ESTP_CHECK_LAUNCH("logprob_merge_kernel");
  return ESTP_OK;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_token_logprobs_workspace_size(int64_t n_tok, int32_t d, int32_t V, int32_t k, int dtype) {
  if (n_tok < 1 || d < 1 || V < 1 || V > (1 << 24) || k < 0 || k > kMaxTop) return 0;
  return logprob_bytes(n_tok, d, V, k, dtype);
}

extern "C" int estp_token_logprobs(const void* X, const void* W, const int32_t* targets, int64_t n_tok, int32_t d,
                                   int32_t V, int32_t k, float temperature, int dtype, float* logprob, float* lse,
                                   float* H, int32_t* top_id, float* top_logprob, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_token_logprobs";
  ESTP_REQUIRE((targets != nullptr) == (logprob != nullptr), ESTP_ERR_INVALID_ARG,
               "%s: targets and logprob must be given together", fn);
  ESTP_REQUIRE(logprob || lse || H || k > 0, ESTP_ERR_INVALID_ARG, "%s: nothing to compute", fn);
  ESTP_REQUIRE(k >= 0 && k <= kMaxTop, ESTP_ERR_INVALID_ARG, "%s: k must be in [0, %d], got %d", fn, kMaxTop, k);
  ESTP_REQUIRE(k == 0 || (top_id && top_logprob), ESTP_ERR_INVALID_ARG, "%s: top_id and top_logprob must be non-null",
               fn);
  ESTP_REQUIRE(aligned(targets, 4) && aligned(logprob, 4) && aligned(lse, 4) && aligned(H, 4) && aligned(top_id, 4) &&
                   aligned(top_logprob, 4),
               ESTP_ERR_INVALID_ARG, "%s: targets and the outputs must be 4-byte aligned", fn);
  ESTP_REQUIRE(temperature >= 1e-3f && temperature <= 1e3f, ESTP_ERR_INVALID_ARG,
               "%s: temperature must be in [0.001, 1000], got %g", fn, double(temperature));
  ESTP_REQUIRE(V <= (1 << 24), ESTP_ERR_UNSUPPORTED, "%s: V = %d, at most 2^24", fn, V);
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(k <= V, ESTP_ERR_INVALID_ARG, "%s: k = %d of a vocabulary of %d", fn, k, V);
  const size_t need = estp_token_logprobs_workspace_size(n_tok, d, V, k, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool quads = use_quads(n_tok, V, dtype);
  // blocks of the same size, in whole tiles
  const int64_t most = quads ? kQuadToks : kBlockToks, blocks = (n_tok + most - 1) / most;
  const int64_t each = std::min(most, ((n_tok + blocks - 1) / blocks + 255) / 256 * 256);
  for (int64_t at = 0; at < n_tok; at += each) {
    const int n = int(std::min(each, n_tok - at));
    auto go = [&](auto launch, auto* x, auto* w) {
      return launch(x + size_t(at) * d, w, targets ? targets + at : nullptr, n, d, V, k, temperature, workspace,
                    logprob ? logprob + at : nullptr, lse ? lse + at : nullptr, H ? H + at : nullptr,
                    top_id ? top_id + at * k : nullptr, top_logprob ? top_logprob + at * k : nullptr, s);
    };
    const __bf16 *x = static_cast<const __bf16*>(X), *w = static_cast<const __bf16*>(W);
    const int rc = quads                ? go(launch_quads, x, w)
                   : dtype == ESTP_BF16 ? go(launch_pieces<__bf16>, x, w)
                                        : go(launch_pieces<float>, static_cast<const float*>(X), static_cast<const float*>(W));
    if (rc != ESTP_OK) return rc;
  }
  return ESTP_OK;
}
