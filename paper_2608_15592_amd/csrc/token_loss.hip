// LM-head loss and its gradient: softmax cross entropy of given next tokens
// over the whole vocabulary, without the n_tok x V logits.
//
//   z_i = W x_i,  lse_i = log sum_v exp z_i[v],  loss_i = lse_i - z_i[t_i]
//   G_iv = g_i (exp(z_i[v] - lse_i) - [v = t_i]),  dX = G W,  dW = G^T X
//
// Forward: lse comes from a pass over the vocabulary that keeps a maximum and a sum per token: of kernels of this file
// (bf16 up to 2048 tokens, fp32), or the entropy kernels' (entropy.hip) for more tokens, and where H or the most
// probable token are asked for too.  loss_pick_kernel forms z_i[t_i] from one row of each operand.  A token whose
// target lies outside [0, V) is ignored: loss 0, no gradient, and its row of X (padding may hold anything) is never
// multiplied into a gradient.
//
// Backward: the live tokens' rows are first gathered next to each other (loss_list_kernel, loss_gather_kernel), so that
// ignored tokens cost nothing and cannot put a NaN into dW.  Then, for one piece of the vocabulary after the other,
// three products: the piece's logits again, turned into G in their epilogue; dX += G W_piece in fp32; dW_piece = G^T X,
// written once.  G is held in the inputs' type (bf16: one rounding of each entry, 2^-8 relative, the type in which the
// matrix cores take it; of up to 64 tokens in two parts; the sums over it are fp32).  Last, loss_dx_kernel rounds dX
// once and puts it into the tokens' places.
//
// Few tokens are bounded by one pass over W for each product, many by the matrix cores: 2 n V d operations for the
// logits of the forward, and three times as many for the backward, which forms them again instead of keeping n V of
// them.  4096 tokens, d 4096, V 128256: 13.1 ms, 1.31 PFLOP/s over all of it (a library product of these logits alone
// runs at 1.48).
#include <algorithm>

#include "estp_common.h"
#include "f32_gemm.h"
#include "f32_split.h"
#include "few_tokens.h"
#include "lm_head.h"
#include "loss_shares.h"
#include "lse_states.h"
#include "mfma_gemm.h"

namespace estp {
namespace detail {

// ------------------------------------------------------------------ elementwise parts

// loss_i = lse_i - x_i . W[t_i], one wave per token, lse_i given or from `states` partial (maximum, sum) states in base
// 2, state p of token i at i states + p: then it is written too.  A sum of probabilities is at most 1, so a difference
// below 0 is rounding and is returned as 0.  (In a launch of their own the states take 7 us after a pass of 226 us over
// 61 tokens, d 4096, V 128256.)
template <typename T, bool kStates>
__global__ __launch_bounds__(256) void loss_pick_kernel(const T* __restrict__ X, const T* __restrict__ W,
                                                        const int32_t* __restrict__ targets, int n_tok, int d, int V,
                                                        const float* __restrict__ part_m,
                                                        const float* __restrict__ part_s, int states,
                                                        float* __restrict__ lse, float* __restrict__ loss) {
  const int tok = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tok >= n_tok) return;
  const int t = targets[tok];
  const bool live = t >= 0 && t < V;
  float z = 0.f;
  if (live)
    for (int k = 8 * lane; k < d; k += 512) z = dot8(X + size_t(tok) * d + k, W + size_t(t) * d + k, z);
  z = wave_sum(z);
  float l;
  if constexpr (kStates) {
    l = lse_of_states(part_m, part_s, tok, states, lane);
    if (lane == 0) lse[tok] = l;
  } else {
    l = lse[tok];
  }
  if (lane == 0) loss[tok] = !live ? 0.f : l - z < 0.f ? 0.f : l - z;
}

// The live tokens in ascending order: row[slot] = token, slot[token] = slot or -1, n_live[0] of them, n_live[1] =
// parts n_live[0] rows of G.  One workgroup takes 1024 tokens a round: latency, 5 us for up to 4096.
__global__ __launch_bounds__(1024) void loss_list_kernel(const int32_t* __restrict__ targets, int n_tok, int V,
                                                         int parts, int* __restrict__ row, int* __restrict__ slot,
                                                         int* __restrict__ n_live) {
  __shared__ int wave_total[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int base = 0;
  for (int64_t at = 0; at < n_tok; at += 1024) {
    const int64_t i = at + tid;
    const int t = i < n_tok ? targets[i] : -1;
    const bool live = t >= 0 && t < V;
    const uint64_t m = __ballot(live);
    if (lane == 0) wave_total[wave] = __popcll(m);
    __syncthreads();
    int before = base, total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      before += w < wave ? wave_total[w] : 0;
      total += wave_total[w];
    }
    const int s = before + __popcll(m & ((uint64_t(1) << lane) - 1));
    if (live) row[s] = int(i);
    if (i < n_tok) slot[i] = live ? s : -1;
    base += total;
    __syncthreads();
  }
  if (tid == 0) {
    n_live[0] = base;
    n_live[1] = parts * base;
  }
}

// Rows, targets, normalisers and weights of the live tokens, next to each other, and all of them once more where G has
// two parts.  16-byte pieces of rows.  A copy (4096 tokens of 8 KB: 13 us, 5.1 TB/s).  kList: of up to 1024 tokens, whose
// targets every workgroup counts for itself to find its token; the first does loss_list_kernel's part (the two launches
// of 1021 tokens, d 2048, take 10.8 us, this one 5.8).
template <bool kList>
__global__ __launch_bounds__(256) void loss_gather_kernel(const uint4* __restrict__ X, const int* __restrict__ row,
                                                          int* __restrict__ slot, int* __restrict__ n_live, int row16,
                                                          const int32_t* __restrict__ targets, int n_tok, int V,
                                                          int parts, const float* __restrict__ lse,
                                                          const float* __restrict__ grad, uint4* __restrict__ Xc,
                                                          int32_t* __restrict__ tc, float* __restrict__ lc,
                                                          float* __restrict__ gc) {
  const int s = blockIdx.x, tid = threadIdx.x;
  int tok;
  if constexpr (kList) {
    __shared__ int counts[16], found;
    const int lane = tid & 63, wave = tid >> 6;
    uint64_t m[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = 256 * u + tid, t = i < n_tok ? targets[i] : -1;
      m[u] = __ballot(t >= 0 && t < V);
      if (lane == 0) counts[4 * u + wave] = __popcll(m[u]);
    }
    __syncthreads();
    int n = 0, before[4];
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      if (c % 4 == wave) before[c / 4] = n;
      n += counts[c];
    }
    const int want = s < n ? s : s - n;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = 256 * u + tid, rank = before[u] + __popcll(m[u] & ((uint64_t(1) << lane) - 1));
      const bool live = (m[u] >> lane) & 1;
      if (live && rank == want) found = i;
      if (s == 0 && i < n_tok) slot[i] = live ? rank : -1;
    }
    if (s == 0 && tid == 0) {
      n_live[0] = n;
      n_live[1] = parts * n;
    }
    if (s >= parts * n) return;
    __syncthreads();
    tok = found;
  } else {
    const int n = n_live[0];
    if (s >= n_live[1]) return;
    tok = row[s < n ? s : s - n];
  }
  for (int k = tid; k < row16; k += 256) Xc[size_t(s) * row16 + k] = X[size_t(tok) * row16 + k];
  if (tid == 0) {
    tc[s] = targets[tok];
    lc[s] = lse[tok];
    gc[s] = grad ? grad[tok] : 1.f;
  }
}

// dX of every token from the partial sums of its slot (and of the second part's), rounded once; 0 for ignored tokens.
// Four columns a thread.  It reads what the products wrote: memory bounds it (684 live of 1021 tokens, d 2048, 10
// shares: 20.8 us, 2.8 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_kernel(const float* __restrict__ acc, const int* __restrict__ slot,
                                                      const int* __restrict__ n_live, int d, int Vc, int tile_toks,
                                                      int wgs, size_t room, T* __restrict__ dX) {
  const int tok = blockIdx.x, s = slot[tok], n = n_live[1], n_tokens = n_live[0];
  const Shares sh = dx_shares(n, d, Vc, tile_toks, wgs, room);
  const size_t each = size_t(n) * d;
  for (int k = 4 * (blockIdx.y * 256 + threadIdx.x); k < d; k += 1024 * gridDim.y) {
    f32x4_t v{0.f, 0.f, 0.f, 0.f};
    if (s >= 0)
      for (int r = s; r < n; r += n_tokens) {
        const float* from = acc + size_t(r) * d + k;
        constexpr int kAhead = 16;  // shares on their way together
        for (int p = 0; p < sh.n; p += kAhead) {
          f32x4_t x[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            x[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (p + u < sh.n) x[u] = *reinterpret_cast<const f32x4_t*>(from + size_t(p + u) * each);
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) v += x[u];
        }
      }
    T* o = dX + size_t(tok) * d + k;
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = T(v[q]);
  }
}

// ------------------------------------------------------------------ matrix-core products (fp32)

// Running (maximum, sum) in base 2 of every token's logits over a slice of the vocabulary tiles: slice s of n_slices
// takes tiles s, s + n_slices, ...; each wave's rows of a tile have a state of their own.  Partial states
// [n_tok, kWM n_slices].
template <int kTN>
__global__ __launch_bounds__(256, 2) void loss_lse_f32_kernel(const float* __restrict__ X, const float* __restrict__ W,
                                                              int n_tok, int d, int V, float c2, int n_slices,
                                                              float* __restrict__ part_m, float* __restrict__ part_s) {
  using Run = F32Tile<true, true, kTN>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int slice = blockIdx.x % n_slices, n0 = blockIdx.x / n_slices * kTN;
  const gemm::Operand A{reinterpret_cast<const char*>(W), uint32_t(d) * 4u, V};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 4u, n_tok};
  float m[Run::kNJ], l[Run::kNJ];
#pragma unroll
  for (int j = 0; j < Run::kNJ; ++j) {
    m[j] = -INFINITY;
    l[j] = 0.f;
  }
  for (int64_t m0 = int64_t(slice) * kFT; m0 < V; m0 += int64_t(n_slices) * kFT) {
    typename Run::Acc acc;
    Run::run(lds, A, B, int(m0), n0, 0, d, acc);
    const auto at = Run::place(int(m0), n0);
#pragma unroll
    for (int j = 0; j < Run::kNJ; ++j) {
      float mx = m[j];
#pragma unroll
      for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool live = at.m + 32 * i + 8 * (r >> 2) + (r & 3) < V;
          mx = fmaxf(mx, live ? acc[i][j][r] * c2 : -INFINITY);
        }
      const float ref = fmaxf(mx, -0x1p127f);  // finite for a lane with no live row yet
      float sum = l[j] * fast_exp2(fmaxf(m[j] - ref, kExp2Floor));
#pragma unroll
      for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool live = at.m + 32 * i + 8 * (r >> 2) + (r & 3) < V;
          sum += live ? fast_exp2(fmaf(acc[i][j][r], c2, -ref)) : 0.f;
        }
      m[j] = mx;
      l[j] = sum;
    }
  }
  const auto at = Run::place(0, n0);
#pragma unroll
  for (int j = 0; j < Run::kNJ; ++j) {
    const float mo = __shfl_xor(m[j], 32, 64), lo = __shfl_xor(l[j], 32, 64), M = fmaxf(m[j], mo);
    const float ref = fmaxf(M, -0x1p127f);
    const float s = l[j] * fast_exp2(fmaxf(m[j] - ref, kExp2Floor)) + lo * fast_exp2(fmaxf(mo - ref, kExp2Floor));
    const int tok = at.n + 32 * j;
    if ((threadIdx.x & 32) == 0 && tok < n_tok) {
      const size_t o = size_t(tok) * (Run::kWM * n_slices) + Run::kWM * slice + at.wm;
      part_m[o] = M;
      part_s[o] = s;
    }
  }
}

// G[slot][v] of vocabulary rows v0 .. v0 + Vc (columns past V: 0), pitch Vc.  M side: vocabulary rows.
template <int kTN>
__global__ __launch_bounds__(256, 2) void loss_grad_f32_kernel(const float* __restrict__ Xc,
                                                               const float* __restrict__ W,
                                                               const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                               int Vc, const int32_t* __restrict__ tc,
                                                               const float* __restrict__ lc,
                                                               const float* __restrict__ gc, float inv_t,
                                                               float* __restrict__ G) {
  using Run = F32Tile<true, true, kTN>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int n = n_live[1], n0 = blockIdx.y * kTN, m0 = blockIdx.x * kFT;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  if (n0 >= n || m0 >= rows) return;
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 4u, rows};
  const gemm::Operand B{reinterpret_cast<const char*>(Xc), uint32_t(d) * 4u, n};
  typename Run::Acc acc;
  Run::run(lds, A, B, m0, n0, 0, d, acc);
  const auto at = Run::place(m0, n0);
#pragma unroll
  for (int j = 0; j < Run::kNJ; ++j) {
    const int s = at.n + 32 * j;
    if (s >= n) continue;
    const int t = int(tc[s] - v0);
    const float l = lc[s], g = gc[s];
#pragma unroll
    for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int v = at.m + 32 * i + 8 * q;
        f32x4_t out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (z / temperature - lse first: near 0 for the weights that matter, so its product is exact to its own rounding)
          const float p = fast_exp2(fmaf(acc[i][j][4 * q + e], inv_t, -l) * kLog2e) - (v + e == t ? 1.f : 0.f);
          out[e] = v + e < rows ? g * p : 0.f;
        }
        *reinterpret_cast<f32x4_t*>(G + size_t(s) * Vc + v) = out;
      }
  }
}

// G of a distillation by the bf16 matrix cores: loss_grad_f32_kernel's, from the parts of the live rows.  90 tokens, d
// 1536, V 151936: 305 us; by the fp32 instructions 506.
template <int kNB, bool kStream>
__global__ __launch_bounds__(64 * split::kWaves, 2) void loss_grad_split_kernel(
    const __bf16* __restrict__ parts, int n_max, const float* __restrict__ W,
    const int* __restrict__ n_live, int d, int V, int64_t v0, int Vc, const float* __restrict__ lc,
    const float* __restrict__ gc, float inv_t, float* __restrict__ G) {
  using Run = split::Tile<kNB, kStream>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]);
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  const int n_vt = (rows + split::kRows - 1) / split::kRows, n_tt = (n + Run::kTN - 1) / Run::kTN;
  // (the token tiles of a vocabulary tile next to each other on one XCD)
  const int first = gemm::first_tile(blockIdx.x, gridDim.x), total = n_vt * n_tt;
  Run::run(
      lds, W + size_t(v0) * d, rows, parts, n_max, n, d, first < total ? (total - first - 1) / int(gridDim.x) + 1 : 0,
      [&](int i) {
        const int id = first + i * int(gridDim.x);
        return typename Run::Place{id / n_tt * split::kRows, id % n_tt * Run::kTN};
      },
      [&](const typename Run::Place& at, const typename Run::Acc& acc) {
        const int lane = threadIdx.x & 63, v0_of = at.m0 + 32 * int(threadIdx.x >> 6) + 4 * (lane >> 4);
#pragma unroll
        for (int b = 0; b < kNB; ++b) {
          const int s = at.n0 + 16 * b + (lane & 15);
          if (s >= n) continue;
          const float l = lc[s], g = gc[s];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int v = v0_of + 16 * i;
            f32x4_t out;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              out[e] = v + e < rows ? g * fast_exp2(fmaf(acc[i][b][e], inv_t, -l) * kLog2e) : 0.f;
            *reinterpret_cast<f32x4_t*>(G + size_t(s) * Vc + v) = out;
          }
        }
      });
}

// out[share][slot][k] (+)= G W_piece over the share's vocabulary rows, shares blockIdx.z, + gridDim.z, ...  M side:
// columns k of W.
template <int kTN>
__global__ __launch_bounds__(256, 2) void loss_dx_f32_kernel(const float* __restrict__ G, const float* __restrict__ W,
                                                             const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                             int Vc, int wgs, size_t room, bool first,
                                                             float* __restrict__ sums) {
  using Run = F32Tile<false, true, kTN>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int n = n_live[1], n0 = blockIdx.y * kTN, m0 = blockIdx.x * kFT;
  const Shares sh = dx_shares(n, d, Vc, kTN, wgs, room);
  if (n0 >= n) return;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 4u, d};
  const gemm::Operand B{reinterpret_cast<const char*>(G), uint32_t(Vc) * 4u, n};
  for (int share = blockIdx.z; share < sh.n; share += gridDim.z) {
    const Depth k = sh.depth(share, rows);
    typename Run::Acc acc;
    Run::run(lds, A, B, m0, n0, k.k0, k.k1, acc);
    float* out = sums + size_t(share) * size_t(n) * d;
    const auto at = Run::place(m0, n0);
#pragma unroll
    for (int j = 0; j < Run::kNJ; ++j)
#pragma unroll
      for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int s = at.n + 32 * j, k = at.m + 32 * i + 8 * q;
          if (s >= n || k >= d) continue;
          f32x4_t* o = reinterpret_cast<f32x4_t*>(out + size_t(s) * d + k);
          f32x4_t v{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          if (!first) v += *o;
          *o = v;
        }
  }
}

// dW[v0 + v][k] = sum over the live tokens of G[s][v] Xc[s][k].  M side: columns k of Xc, N side: vocabulary rows.
template <int kTN>
__global__ __launch_bounds__(256, 2) void loss_dw_f32_kernel(const float* __restrict__ G, const float* __restrict__ Xc,
                                                             const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                             int Vc, float* __restrict__ dW) {
  using Run = F32Tile<false, false, kTN>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int n = n_live[1], m0 = blockIdx.x * kFT, n0 = blockIdx.y * kTN;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  if (n0 >= rows) return;
  const gemm::Operand A{reinterpret_cast<const char*>(Xc), uint32_t(d) * 4u, d};
  const gemm::Operand B{reinterpret_cast<const char*>(G), uint32_t(Vc) * 4u, Vc};
  typename Run::Acc acc;
  Run::run(lds, A, B, m0, n0, 0, n, acc);
  const auto at = Run::place(m0, n0);
#pragma unroll
  for (int j = 0; j < Run::kNJ; ++j)
#pragma unroll
    for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int v = at.n + 32 * j, k = at.m + 32 * i + 8 * q;
        if (v >= rows || k >= d) continue;
        *reinterpret_cast<f32x4_t*>(dW + (size_t(v0) + v) * d + k) =
            f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      }
}

// loss_dx_f32_kernel's sums of a distillation by the bf16 matrix cores, numbers in three parts each.  Workgroup (256
// columns, 16 kNB tokens, share); a wave takes 32 columns and all of those tokens, 32 vocabulary rows a step.  W goes into
// registers as it lies, 8 rows and 2 columns a lane, a step ahead, and is split between the products of the step before.
// G's parts, which the waves share, are formed by a wave for each 16 tokens, and lie in LDS in the order of the operands,
// two steps of them: one barrier a step.  M side: columns of W, N side: tokens.  By parts and by the fp32 instructions, us:
// 12 tokens, d 2048, V 128256 173 and 195, 33 tokens 226 and 309, 200 827 and 1039, 400 1374 and 2075; 90 tokens, d 1536, V
// 151936 250 and 394, 3.7 TB/s of W and 1.1 PFLOP/s: W and the matrix cores take about 133 and 190 of it each.
template <int kNB>
__global__ __launch_bounds__(512, 2) void loss_dx_split_kernel(const float* __restrict__ G, const float* __restrict__ W,
                                                               const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                               int Vc, int n_cols, int n_tiles, int n_slices, int wgs,
                                                               size_t room, bool first, float* __restrict__ sums) {
  __shared__ __attribute__((aligned(16))) char lds[2 * 3 * 1024 * kNB];
  const gemm::SliceAt wg = gemm::slice_of(gemm::first_tile(blockIdx.x, gridDim.x), n_tiles, n_slices);
  const int all = __builtin_amdgcn_readfirstlane(n_live[1]), n0 = wg.tile / n_cols * 16 * kNB, n = min(16 * kNB, all - n0);
  if (wg.slice >= n_slices || n <= 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fq = lane >> 4;
  const int c0 = 256 * (wg.tile % n_cols) + 32 * wave;
  const Shares sh = dx_shares(all, d, Vc, 16 * kNB, wgs, room);
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  G += size_t(n0) * Vc;
  const buf_rsrc_t rg = make_rsrc(G, uint32_t(n) * uint32_t(Vc) * 4u);  // (rows past the live ones read 0)
  uint32_t off[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) off[e] = (uint32_t(8 * fq + e) * uint32_t(d) + uint32_t(c0 + 2 * fr)) * 4u;
  for (int share = wg.slice; share < sh.n; share += n_slices) {
    const Depth depth = sh.depth(share, rows);
    const int steps = (depth.k1 - depth.k0 + 63) / 64 * 2;  // (of rows past the share's nothing but zeros)
    // (columns past d hold the next row's numbers, or 0; they are not stored)
    auto load_w = [&](int t, split::Raw (&raw)[2]) {
      const int at = depth.k0 + 32 * t, left = c0 < d ? max(0, min(32, depth.k1 - at)) : 0;
      const buf_rsrc_t r = make_rsrc(W + size_t(v0 + (left > 0 ? at : 0)) * d, uint32_t(left) * uint32_t(d) * 4u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const f32x2_t w = buf_load2<kNonTemporal>(r, off[e]);
        raw[0].v[e] = w[0];
        raw[1].v[e] = w[1];
      }
    };
    f32x4_t g[2];
    auto load_g = [&](int t) {
      if (wave >= kNB || t >= steps) return;
      const uint32_t o = (uint32_t(16 * wave + fr) * uint32_t(Vc) + uint32_t(depth.k0 + 32 * t + 8 * fq)) * 4u;
      g[0] = buf_load4(rg, o);
      g[1] = buf_load4(rg, o + 16u);
    };
    auto keep_g = [&](int t) {
      if (wave >= kNB || t >= steps) return;
      split::Raw r{{g[0][0], g[0][1], g[0][2], g[0][3], g[1][0], g[1][1], g[1][2], g[1][3]}};
      const int left = depth.k1 - depth.k0 - 32 * t;
      if (left < 32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = 8 * fq + e < left ? r.v[e] : 0.f;
      }
      split::Frag f;
#pragma unroll
      for (int j = 0; j < 8; ++j) f.piece(r, j);
#pragma unroll
      for (int p = 0; p < 3; ++p)
        *reinterpret_cast<bf16x8_t*>(lds + (t & 1) * (3 * 1024 * kNB) + (3 * wave + p) * 1024 + 16 * lane) = f.part(p);
    };
    f32x4_t acc[2][kNB], low[2][kNB];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < kNB; ++b) acc[i][b] = low[i][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    split::Raw even[2], odd[2];
    split::Frag here[2], next[2];
    load_g(0);
    load_w(0, even);
    load_w(1, odd);
    keep_g(0);
    load_g(1);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) here[i].piece(even[i], j);
    lds_barrier();
    // step t from `w`; `later` are the rows of step t + 1, and those of t + 2 come into `free`
    auto step = [&](int t, const split::Frag (&w)[2], split::Frag (&then)[2], split::Raw (&later)[2],
                    split::Raw (&free)[2]) {
      load_w(t + 2, free);
      keep_g(t + 1);
      load_g(t + 2);
      const char* from = lds + (t & 1) * (3 * 1024 * kNB) + 16 * lane;
      bf16x8_t x[2][3];
      auto read = [&](int b) {
#pragma unroll
        for (int p = 0; p < 3; ++p) x[b & 1][p] = *reinterpret_cast<const bf16x8_t*>(from + (3 * b + p) * 1024);
      };
      read(0);
      __builtin_amdgcn_sched_barrier(0);
      constexpr int kEvery = 12 * kNB / 16;
#pragma unroll
      for (int m = 0; m < 12 * kNB; ++m) {
        constexpr int kW[6] = {2, 0, 1, 0, 1, 0}, kX[6] = {0, 2, 1, 1, 0, 0};
        const int b = m / 12, s = m % 12 / 2, i = m % 2;
        if (m % 12 == 0 && b + 1 < kNB) read(b + 1);
        f32x4_t& sum = s == 5 ? acc[i][b] : low[i][b];
        sum = mfma_bf16(w[i].part(kW[s]), x[b & 1][kX[s]], sum);
        if (m % kEvery == 0 && m / kEvery < 16) then[m / kEvery / 8].piece(later[m / kEvery / 8], m / kEvery % 8);
        __builtin_amdgcn_sched_barrier(0);
      }
      lds_barrier();
    };
    for (int t = 0; t < steps; t += 2) {
      step(t, here, next, odd, even);
      step(t + 1, next, here, even, odd);
    }
    float* out = sums + (size_t(share) * size_t(all) + n0) * d;
    const int c = c0 + 8 * fq;
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int s = 16 * b + fr;
      if (s >= n || c >= d) continue;  // (d is a multiple of 8)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4_t v;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r = 2 * h + q / 2, i = q % 2;
          v[q] = split::joined(acc[i][b][r], low[i][b][r]);
        }
        f32x4_t* o = reinterpret_cast<f32x4_t*>(out + size_t(s) * d + c + 4 * h);
        if (!first) v += *o;
        *o = v;
      }
    }
  }
}

// dW of up to 96 rows of a distillation by the bf16 matrix cores: G^T X of numbers in three parts each, six products,
// as the logits of f32_split.h and as exact.  A wave holds the parts of G's 64 columns v, all rows deep, in registers,
// and goes along X's columns, 16 at a time, whose parts split_columns_kernel laid out in the order of the operands; the
// next ones are on their way meanwhile.  No barrier.  M side: X's columns, N side: vocabulary rows.  A wave has up to a
// quarter of the columns, so that what runs at a time writes all parts of a row; G is split once more for each share.
// Results pass LDS, 64 columns at a time, so that 256 bytes of a row leave together, non-temporal.  90 tokens, d 1536,
// V 151936 (933 MB of dW): about 250 us, 495 with the fp32 instructions' tiles; 471 with
// ordinary 64-byte runs and no loads ahead, 376 with these, 326 non-temporal.  12 tokens, d 2048, V 128256 (1.05 GB):
// 229, 4.6 TB/s of stores; 442 in runs of 64 bytes, 265 where the shares of a row are far apart in the grid.
template <int kSteps>
__global__ __launch_bounds__(256, 2) void loss_dw_split_kernel(const float* __restrict__ G,
                                                               const __bf16* __restrict__ columns,
                                                               const int* __restrict__ n_live, int d, int V,
                                                               int64_t v0, int Vc, float* __restrict__ dW) {
  const int lane = threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]);
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc))), v = 256 * blockIdx.y + 64 * int(threadIdx.x >> 6) + fr;
  if (v - fr >= rows) return;
  const buf_rsrc_t rg = make_rsrc(G, uint32_t(n) * uint32_t(Vc) * 4u);  // (rows past the live ones read 0)
  bf16x8_t g[4][kSteps][3];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      uint32_t q[3][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t at = uint32_t(32 * s + 8 * fq + 2 * e) * uint32_t(Vc) + uint32_t(min(v + 16 * j, Vc - 1));
        const split::Parts p = split::parts_of(buf_load1(rg, 4u * at), buf_load1(rg, 4u * (at + uint32_t(Vc))));
        q[0][e] = p.p1;
        q[1][e] = p.p2;
        q[2][e] = p.p3;
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) g[j][s][p] = __builtin_bit_cast(bf16x8_t, uint4{q[p][0], q[p][1], q[p][2], q[p][3]});
    }
  // a wave's 64 rows of 64 columns, which leave it in whole runs of a row
  constexpr int kPitch = 68;
  __shared__ __attribute__((aligned(16))) float lds[4 * 64 * kPitch];
  float* mine = lds + (threadIdx.x >> 6) * (64 * kPitch);
  const int blocks = (d + 15) / 16, per = ((blocks + 3) / 4 + int(gridDim.x) - 1) / int(gridDim.x) * 4;
  const int first = per * int(blockIdx.x), last = min(blocks, first + per);
  bf16x8_t x[kSteps][3], ahead[kSteps][3];
  const auto load = [&](int c) {
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        ahead[s][p] = *reinterpret_cast<const bf16x8_t*>(columns + ((size_t(c) * 3 + p) * kSteps + s) * 512 + 8 * lane);
  };
  load(min(first, blocks - 1));
  for (int c = first; c < last; ++c) {
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int s = 0; s < kSteps; ++s) x[s][p] = ahead[s][p];
    load(min(c + 1, blocks - 1));
    f32x4_t acc[4], low[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = low[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr int kX[6] = {2, 0, 1, 0, 1, 0}, kG[6] = {0, 2, 1, 1, 0, 0};
#pragma unroll
    for (int t = 0; t < 6; ++t)
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f32x4_t& sum = t == 5 ? acc[j] : low[j];
          sum = mfma_bf16(x[s][kX[t]], g[j][s][kG[t]], sum);
        }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4_t*>(mine + (16 * j + fr) * kPitch + 16 * (c & 3) + 4 * fq) = split::joined(acc[j], low[j]);
    if ((c & 3) != 3 && c + 1 < last) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int col = 16 * (c & ~3) + 4 * fr;
#pragma unroll 4
    for (int i = 0; i < 16; ++i)
      if (v - fr + 4 * i + fq < rows && col < min(d, 16 * (c + 1)))
        __builtin_nontemporal_store(*reinterpret_cast<const f32x4_t*>(mine + (4 * i + fq) * kPitch + 4 * fr),
                                    reinterpret_cast<f32x4_t*>(dW + (size_t(v0) + v - fr + 4 * i + fq) * d + col));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// The same of any number of rows.  Workgroup (128 vocabulary rows, 16 kNB columns of X); a wave takes 32 vocabulary rows and
// all of those columns, 32 tokens a step.  As loss_dx_split_kernel, with G, whose columns are split on the way, in the place
// of W, and X's parts as split_columns_kernel laid them out, through LDS, in the place of G's.  The column tiles of 128
// vocabulary rows run next to each other on one XCD, into whose L2 G's columns so come once.  M side: X's columns, N side:
// vocabulary rows.  Two workgroups share a compute unit, so that one's first loads and stores lie beside the other's
// products: with one of 8 waves 657, 974, 1603 and 788 us where it takes 574 (128 tokens, d 2048, V 128256), 848 (200), 1384
// (400, 0.9 PFLOP/s of the parts) and 741 (1000, d 1024, V 65536); 711, 1082, 1981 and 1144 by the fp32 instructions.
template <int kNB>
__global__ __launch_bounds__(256, 2) void loss_dw_split_many_kernel(const float* __restrict__ G,
                                                                    const __bf16* __restrict__ columns, int all_steps,
                                                                    const int* __restrict__ n_live, int d, int V,
                                                                    int64_t v0, int Vc, int n_cols,
                                                                    float* __restrict__ dW) {
  __shared__ __attribute__((aligned(16))) char lds[2 * 3 * 1024 * kNB];
  const int id = gemm::first_tile(blockIdx.x, gridDim.x), rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  const int m0 = 128 * (id / n_cols), first = kNB * (id % n_cols);  // block of 16 columns
  if (m0 >= rows) return;
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]), steps = (n + 63) / 64 * 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fq = lane >> 4;
  const int v = m0 + 32 * wave + 2 * fr;
  uint32_t off[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) off[e] = (uint32_t(8 * fq + e) * uint32_t(Vc) + uint32_t(v)) * 4u;
  auto load_g = [&](int t, split::Raw (&raw)[2]) {
    const int left = max(0, min(32, n - 32 * t));
    const buf_rsrc_t r = make_rsrc(G + size_t(left > 0 ? 32 * t : 0) * Vc, uint32_t(left) * uint32_t(Vc) * 4u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const f32x2_t g = buf_load2(r, off[e]);
      raw[0].v[e] = g[0];
      raw[1].v[e] = g[1];
    }
  };
  constexpr int kBring = (3 * kNB + 3) / 4;  // pieces of 1 KB of a step that a wave brings
  bf16x8_t x[kBring];
  const int pieces = 3 * min(kNB, (d + 15) / 16 - first);
  auto load_x = [&](int t) {
#pragma unroll
    for (int u = 0; u < kBring; ++u)
      if (wave + 4 * u < pieces && t < all_steps)
        x[u] = *reinterpret_cast<const bf16x8_t*>(columns + ((size_t(first) * 3 + wave + 4 * u) * all_steps + t) * 512 +
                                                  8 * lane);
  };
  auto keep_x = [&](int t) {
#pragma unroll
    for (int u = 0; u < kBring; ++u)
      if (wave + 4 * u < 3 * kNB && t < steps)
        *reinterpret_cast<uint4*>(lds + (t & 1) * (3 * 1024 * kNB) + (wave + 4 * u) * 1024 + 16 * lane) =
            wave + 4 * u < pieces && t < all_steps ? __builtin_bit_cast(uint4, x[u]) : uint4{0, 0, 0, 0};
  };
  f32x4_t acc[2][kNB], low[2][kNB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int b = 0; b < kNB; ++b) acc[i][b] = low[i][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  split::Raw even[2], odd[2];
  split::Frag here[2], next[2];
  load_x(0);
  load_g(0, even);
  load_g(1, odd);
  keep_x(0);
  load_x(1);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) here[i].piece(even[i], j);
  lds_barrier();
  auto step = [&](int t, const split::Frag (&g)[2], split::Frag (&then)[2], split::Raw (&later)[2],
                  split::Raw (&free)[2]) {
    load_g(t + 2, free);
    keep_x(t + 1);
    load_x(t + 2);
    const char* from = lds + (t & 1) * (3 * 1024 * kNB) + 16 * lane;
    bf16x8_t xs[2][3];
    auto read = [&](int b) {
#pragma unroll
      for (int p = 0; p < 3; ++p) xs[b & 1][p] = *reinterpret_cast<const bf16x8_t*>(from + (3 * b + p) * 1024);
    };
    read(0);
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kEvery = 12 * kNB / 16;
#pragma unroll
    for (int m = 0; m < 12 * kNB; ++m) {
      constexpr int kG[6] = {2, 0, 1, 0, 1, 0}, kX[6] = {0, 2, 1, 1, 0, 0};
      const int b = m / 12, s = m % 12 / 2, i = m % 2;
      if (m % 12 == 0 && b + 1 < kNB) read(b + 1);
      f32x4_t& sum = s == 5 ? acc[i][b] : low[i][b];
      sum = mfma_bf16(xs[b & 1][kX[s]], g[i].part(kG[s]), sum);
      if (m % kEvery == 0 && m / kEvery < 16) then[m / kEvery / 8].piece(later[m / kEvery / 8], m / kEvery % 8);
      __builtin_amdgcn_sched_barrier(0);
    }
    lds_barrier();
  };
  for (int t = 0; t < steps; t += 2) {
    step(t, here, next, odd, even);
    step(t + 1, next, here, even, odd);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int k = 16 * (first + b) + 4 * fq;
      if (v + i >= rows || k >= d) continue;  // (d is a multiple of 8)
      *reinterpret_cast<f32x4_t*>(dW + (size_t(v0) + v + i) * d + k) = split::joined(acc[i][b], low[i][b]);
    }
}

// ------------------------------------------------------------------ matrix-core products (bf16)

// Of 16 columns of Xc's live rows (at most 128) and 32 rows 1 KB, as the matrix cores take them where the rows are the
// depth; zeros past the live rows.  One workgroup a block of columns.
__global__ __launch_bounds__(256) void loss_columns_kernel(const __bf16* __restrict__ Xc, const int* __restrict__ n_live,
                                                           int d, int steps, __bf16* __restrict__ columns) {
  const int lane = threadIdx.x & 63, step = threadIdx.x >> 6, n = n_live[1];
  if (step >= steps) return;
  bf16x8_t x;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int row = 32 * step + 8 * (lane >> 4) + e;
    x[e] = row < n ? Xc[size_t(row) * d + 16 * blockIdx.x + (lane & 15)] : __bf16(0.f);
  }
  *reinterpret_cast<bf16x8_t*>(columns + (size_t(blockIdx.x) * steps + step) * 512 + 8 * lane) = x;
}

// dW of up to 64 tokens of a distillation, whose G has two parts: at most 128 rows deep.  A wave holds G's 64 columns v,
// four a lane, all rows deep, in registers, and goes along X's columns, 16 at a time, from loss_columns_kernel; the next
// ones are on their way meanwhile.  No barrier.  M side: X's columns, N side: vocabulary rows.  Results pass LDS, 128
// columns at a time, so that 256 bytes of a row leave together, non-temporal: its stores bound it.  12 tokens, d 2048, V
// 128256 (525 MB): 105 us, 5.0 TB/s (with the tiles of larger calls 195; 163 where the shares of a row are far apart in the
// grid, since what is written at a time then lies in one part of each row); 64 tokens, d 4096 238; 16 tokens, d 64, V 1000 4.
template <int kSteps>
__global__ __launch_bounds__(256, 2) void loss_dw_few_kernel(const __bf16* __restrict__ G,
                                                             const __bf16* __restrict__ columns,
                                                             const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                             int Vc, __bf16* __restrict__ dW) {
  constexpr int kPitch = 132;  // (four rows on, eight banks on)
  __shared__ __attribute__((aligned(16))) __bf16 lds[4 * 64 * kPitch];
  const int lane = threadIdx.x & 63, fr = lane & 15, fq = lane >> 4;
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]);
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc))), v = 256 * blockIdx.y + 64 * int(threadIdx.x >> 6);
  if (v >= rows) return;
  __bf16* mine = lds + (threadIdx.x >> 6) * (64 * kPitch);
  const buf_rsrc_t rg = make_rsrc(G, uint32_t(n) * uint32_t(Vc) * 2u);  // (rows past the live ones read 0)
  bf16x8_t g[4][kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t at = uint32_t(32 * s + 8 * fq + e) * uint32_t(Vc) + uint32_t(v + 4 * fr);
      const bf16x4_t four = __builtin_bit_cast(bf16x4_t, buf_load2(rg, 2u * at));
#pragma unroll
      for (int j = 0; j < 4; ++j) g[j][s][e] = four[j];
    }
  const int blocks = d / 16, per = ((blocks + 7) / 8 + int(gridDim.x) - 1) / int(gridDim.x) * 8;  // (d a multiple of 32)
  const int first = per * int(blockIdx.x), last = min(blocks, first + per);
  bf16x8_t x[kSteps], ahead[kSteps];
  const auto load = [&](int c) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      ahead[s] = *reinterpret_cast<const bf16x8_t*>(columns + (size_t(c) * kSteps + s) * 512 + 8 * lane);
  };
  load(min(first, blocks - 1));
  for (int c = first; c < last; ++c) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) x[s] = ahead[s];
    load(min(c + 1, blocks - 1));
    f32x4_t acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = mfma_bf16(x[s], g[j][s], acc[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint2*>(mine + (4 * fr + j) * kPitch + 16 * (c & 7) + 4 * fq) =
          uint2{pack_bf16(acc[j][0], acc[j][1]), pack_bf16(acc[j][2], acc[j][3])};
    if ((c & 7) != 7 && c + 1 < last) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int col = 16 * (c & ~7) + 8 * fr;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int row = 4 * i + fq;
      const uint2* from = reinterpret_cast<const uint2*>(mine + row * kPitch + 8 * fr);
      const uint2 lo = from[0], hi = from[1];
      if (v + row < rows && col < 16 * (c + 1))
        __builtin_nontemporal_store(u32x4_t{lo.x, lo.y, hi.x, hi.y},
                                    reinterpret_cast<u32x4_t*>(dW + (size_t(v0) + v + row) * d + col));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Running (reference, sum) in base 2 of every token's logits, for calls of few tokens: workgroup (token tile, slice)
// takes the vocabulary tiles slice, slice + n_slices, ..., so that any number of token tiles fills the chip.  The
// first tile's maximum is the reference; later tiles add to the sum with one FMA, exponential and addition a logit,
// and move the reference only where a sum would pass 2^64.  Partial states [n_tok, 2 n_slices], a wave's 128 rows each.
// 61 tokens, d 4096, V 128256: 217 us, 4.8 TB/s of W; 1021 tokens, d 2048: 404 us, 1.33 PFLOP/s; 4096 tokens, d 4096:
// 2716 us, 1.58 PFLOP/s.  (The sums leave the matrix cores' registers column by column, read_sum: with all of them at once,
// some went through memory, and the three took 217, 450 and 2820 us.)
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void loss_lse_mfma_kernel(const __bf16* __restrict__ X,
                                                               const __bf16* __restrict__ W, int n_tok, int d, int V,
                                                               float c2, int n_tt, int n_slices,
                                                               float* __restrict__ part_m,
                                                               float* __restrict__ part_s) {
  using Run = gemm::Tiles<true, true, false, kNBN, kOdd, 0>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const gemm::SliceAt at_slice = gemm::slice_of(gemm::first_tile(blockIdx.x, gridDim.x), n_tt, n_slices);
  const int tt = at_slice.tile, slice = at_slice.slice;
  if (slice >= n_slices) return;
  const gemm::Operand A{reinterpret_cast<const char*>(W), uint32_t(d) * 2u, V};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 2u, n_tok};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  const int n_vt = (V + 255) / 256, n_mine = (n_vt - slice + n_slices - 1) / n_slices;
  float m[kNBN], l[kNBN];
#pragma unroll
  for (int j = 0; j < kNBN; ++j) {
    m[j] = -INFINITY;
    l[j] = 0.f;
  }
  Run::run(
      lds, A, B, 0, 1, n_mine,
      [&](int i) { return gemm::Place{256 * (slice + i * n_slices), Run::kBN * tt, 0, d, i}; },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][kNBN]) {
        const int fq = gemm::fresh_lane() >> 4;
        const int lim = V - (at.m0 + 128 * wm + 4 * fq);  // live rows: 16 i + r < lim
        const bool ragged = at.m0 + 256 > V;
        gemm::sums_ready();
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          float z[8][4];
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) z[i][r] = gemm::read_sum(acc[i][j][r]);
          bool exact = ragged || at.tag == 0;
          if (!exact) {
            float s = l[j];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) s += fast_exp2(fmaf(z[i][r], c2, -m[j]));
            exact = !(s <= 0x1p64f);  // (a NaN takes the exact path and stays one)
            l[j] = exact ? l[j] : s;
          }
          if (exact) {
            float mx = m[j];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) mx = fmaxf(mx, 16 * i + r < lim ? z[i][r] * c2 : -INFINITY);
            const float ref = fmaxf(mx, -0x1p127f);  // finite for a lane with no live row yet
            float s = l[j] * fast_exp2(fmaxf(m[j] - ref, kExp2Floor));
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                s += 16 * i + r < lim ? fast_exp2(fmaf(z[i][r], c2, -ref)) : 0.f;
            m[j] = mx;
            l[j] = s;
          }
        }
      });
  // lanes l, l ^ 16, l ^ 32, l ^ 48 hold the same tokens
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kNBN; ++j) {
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1) {
      const float mo = __shfl_xor(m[j], o, 64), lo = __shfl_xor(l[j], o, 64), M = fmaxf(m[j], mo);
      const float ref = fmaxf(M, -0x1p127f);
      l[j] = l[j] * fast_exp2(fmaxf(m[j] - ref, kExp2Floor)) + lo * fast_exp2(fmaxf(mo - ref, kExp2Floor));
      m[j] = M;
    }
    const int tok = Run::kBN * tt + 16 * kNBN * wn + 16 * j + (lane & 15);
    if (lane < 16 && tok < n_tok) {
      const size_t o = size_t(tok) * (2 * n_slices) + 2 * slice + wm;
      part_m[o] = m[j];
      part_s[o] = l[j];
    }
  }
}

// G of a piece: products of W's rows (M side) and the live tokens (N side), turned into G as they leave the matrix
// cores.  A lane holds 8 consecutive vocabulary rows of a token: one 16-byte store.  Bound by the matrix cores, with
// the exponentials between two tiles (4096 tokens, d 4096, 32768 vocabulary rows, 1.1 TFLOP: 735 us, 1.50 PFLOP/s;
// 684 live tokens, d 2048, all of 128256: 353 us, 1.02 PFLOP/s, a ninth of it on columns that no token has; 766 of 1021
// live 417).
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void loss_grad_mfma_kernel(const __bf16* __restrict__ Xc,
                                                                const __bf16* __restrict__ W,
                                                                const int* __restrict__ n_live, int d, int V,
                                                                int64_t v0, int Vc, const int32_t* __restrict__ tc,
                                                                const float* __restrict__ lc,
                                                                const float* __restrict__ gc, float c2,
                                                                __bf16* __restrict__ G) {
  using Run = gemm::Tiles<true, true, true, kNBN, kOdd, 4 * kNBN>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]), n_tokens = __builtin_amdgcn_readfirstlane(n_live[0]);
  const int rows = __builtin_amdgcn_readfirstlane(int(min(int64_t(V) - v0, int64_t(Vc))));
  const int n_m = (rows + 255) / 256, n_n = (n + Run::kBN - 1) / Run::kBN;
  const gemm::TileOrder order(n_m, n_n);
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 2u, rows};
  const gemm::Operand B{reinterpret_cast<const char*>(Xc), uint32_t(d) * 2u, n};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  Run::run(
      lds, A, B, gemm::first_tile(blockIdx.x, gridDim.x), gridDim.x, n_m * n_n,
      [&](int id) {
        const gemm::TileAt t = order(id);
        return gemm::Place{256 * t.m, Run::kBN * t.n, 0, d, 0};
      },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][kNBN]) {
        const int m0 = at.m0, n0 = at.n0, lane = gemm::fresh_lane(), fr = lane & 15, fq = lane >> 4;
        const int live = min(Run::kBN, n - n0);
        const buf_rsrc_t out =
            make_rsrc(reinterpret_cast<const char*>(G) + size_t(n0) * Vc * 2, uint32_t(live) * uint32_t(Vc) * 2u);
        const int c0 = m0 + 128 * wm + 8 * fq;  // the lane's first column of G
        const bool ragged = m0 + 256 > rows;
        float lse_of[kNBN], g_of[kNBN];  // of the lane's tokens, all on their way before the first is needed
        int t_of[kNBN];
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          const int s = min(n0 + 16 * kNBN * wn + 16 * j + fr, n - 1);
          lse_of[j] = lc[s];
          g_of[j] = gc[s];
          t_of[j] = tc[s];
        }
        __builtin_amdgcn_sched_barrier(0);
        gemm::sums_ready();
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          const int sl = 16 * kNBN * wn + 16 * j + fr;
          const float l2 = lse_of[j] * kLog2e, g = g_of[j];
          const int rel = int(t_of[j] - v0) - c0;  // the target is column rel of the lane's 128, 8 of every 32
          float p[4][8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              p[i / 2][4 * (i % 2) + r] = g * fast_exp2(fmaf(gemm::read_sum(acc[i][j][r]), c2, -l2));
          if (__any(rel >= 0 && rel < 128 && (rel & 31) < 8)) {  // seldom: one tile in V / 256 holds a token's target
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int e = 0; e < 8; ++e) p[q][e] = rel == 32 * q + e ? p[q][e] - g : p[q][e];
          }
          if (ragged) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int e = 0; e < 8; ++e) p[q][e] = c0 + 32 * q + e < rows ? p[q][e] : 0.f;
          }
          if (kNBN == 4 && n > n_tokens) {  // two parts: the second is what the rounding of the first leaves
            const bool second = n0 + sl >= n_tokens;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int e = 0; e < 8; ++e) p[q][e] -= second ? float(__bf16(p[q][e])) : 0.f;
          }
#pragma unroll
          for (int q = 0; q < 4; ++q)
            buf_store16(out, uint32_t(sl) * uint32_t(Vc) * 2u + uint32_t(c0 + 32 * q) * 2u,
                        uint4{pack_bf16(p[q][0], p[q][1]), pack_bf16(p[q][2], p[q][3]), pack_bf16(p[q][4], p[q][5]),
                              pack_bf16(p[q][6], p[q][7])});
        }
      });
}

// G of a distillation of few tokens, with W in whole runs (few_tokens.h); the same numbers as above.
template <int kSteps, int kNB>
__global__ __launch_bounds__(64 * few::kWaves, 2) void loss_grad_few_kernel(const __bf16* __restrict__ Xc,
                                                                            const __bf16* __restrict__ W,
                                                                            const int* __restrict__ n_live, int d,
                                                                            int V, int64_t v0, int Vc,
                                                                            const float* __restrict__ lc,
                                                                            const float* __restrict__ gc, float c2,
                                                                            __bf16* __restrict__ G) {
  __shared__ __attribute__((aligned(16))) char lds[few::Rows<kSteps, kNB>::kLds];
  const int n = __builtin_amdgcn_readfirstlane(n_live[0]);  // of two parts each
  const int rows = __builtin_amdgcn_readfirstlane(int(min(int64_t(V) - v0, int64_t(Vc))));
  const int s = threadIdx.x / 64 * 16 + (threadIdx.x & 15);
  const bool live = s < n;
  const float l2 = live ? lc[s] * kLog2e : 0.f, g = live ? gc[s] : 0.f;
  const buf_rsrc_t out = make_rsrc(G, uint32_t(2 * n) * uint32_t(Vc) * 2u);
  const uint32_t base = uint32_t(s) * uint32_t(Vc) * 2u, part = uint32_t(n) * uint32_t(Vc) * 2u;
  // (whole tiles of 256: what follows reads columns past the last row, where G is 0)
  few::run<kSteps, kNB, 2>(Xc, W + size_t(v0) * d, n, d, rows, (rows + 255) / 256 * 16, lds,
                           [&](int64_t row, f32x4_t z) {
    float p[4];
    uint32_t q[2], left[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = row + e < rows ? g * fast_exp2(fmaf(z[e], c2, -l2)) : 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      q[e] = pack_bf16(p[2 * e], p[2 * e + 1]);
      left[e] = pack_bf16(p[2 * e] - __uint_as_float(q[e] << 16), p[2 * e + 1] - __uint_as_float(q[e] & 0xffff0000u));
    }
    const uint32_t off = base + uint32_t(row) * 2u;
    buf_store8(out, live ? off : kPastEnd, q[0], q[1]);
    buf_store8(out, live ? off + part : kPastEnd, left[0], left[1]);
  });
}

// out[share][slot][k] (+)= G W_piece over the share's vocabulary rows.  M side: columns k of W (transposed reads), N
// side: slots.  The matrix cores bound it (the sizes above: 870 us, 1.26 PFLOP/s, and 388 us, 0.93 PFLOP/s).
template <int kNBN>
__global__ __launch_bounds__(256, 1) void loss_dx_mfma_kernel(const __bf16* __restrict__ G,
                                                              const __bf16* __restrict__ W,
                                                              const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                              int Vc, size_t room, bool first,
                                                              float* __restrict__ out) {
  using Run = gemm::Tiles<false, true, false, kNBN, false, 8 * kNBN < 48 ? 8 * kNBN : 48>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]);
  const int rows = __builtin_amdgcn_readfirstlane(int(min(int64_t(V) - v0, int64_t(Vc))));
  const int n_m = (d + 255) / 256, n_n = (n + Run::kBN - 1) / Run::kBN;
  const gemm::TileOrder order(n_m, n_n);
  const gemm::Divisor share_tiles(max(1, n_m * n_n));
  const Shares sh = dx_shares(n, d, Vc, Run::kBN, gridDim.x, room);
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 2u, d};
  const gemm::Operand B{reinterpret_cast<const char*>(G), uint32_t(Vc) * 2u, n};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  const int tiles = n_m * n_n;
  Run::run(
      lds, A, B, gemm::first_tile(blockIdx.x, gridDim.x), gridDim.x, tiles * sh.n,
      [&](int id) {
        const int share = int(share_tiles.div(uint32_t(id)));
        const gemm::TileAt t = order(id - share * tiles);
        const Depth k = sh.depth(share, rows);
        return gemm::Place{256 * t.m, Run::kBN * t.n, k.k0, k.k1, share};
      },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][kNBN]) {
        const int m0 = at.m0, n0 = at.n0, lane = gemm::fresh_lane(), fr = lane & 15, fq = lane >> 4;
        const int live = min(Run::kBN, n - n0);
        float* sums = out + (size_t(at.tag) * n + n0) * d;
        const buf_rsrc_t o = make_rsrc(sums, uint32_t(live) * uint32_t(d) * 4u);
        const buf_rsrc_t was = make_rsrc(sums, first ? 0u : uint32_t(live) * uint32_t(d) * 4u);  // (empty: reads 0)
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          const uint32_t row = uint32_t(16 * kNBN * wn + 16 * j + fr) * uint32_t(d);
          const int c0 = m0 + 128 * wm + 4 * fq;
          f32x4_t v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            v[i] = buf_load4(was, c0 + 16 * i < d ? (row + uint32_t(c0 + 16 * i)) * 4u : kPastEnd);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            buf_store16(o, c0 + 16 * i < d ? (row + uint32_t(c0 + 16 * i)) * 4u : kPastEnd,
                        __builtin_bit_cast(uint4, v[i] + acc[i][j]));
        }
      });
}

// dW of a piece: G^T Xc.  M side: columns k of Xc, N side: vocabulary rows; both transposed reads, the tokens are
// the depth.  The matrix cores bound it where there are many (the sizes above: 870 us, 1.26 PFLOP/s); of 684, which are
// 11 stages a tile, its first stage and its stores are a good part (443 us, 0.81 PFLOP/s).
//
// kStream: dW of few tokens is bound by its stores, and one that the last cache does not hold drives W out of it, which
// the next loss of the same W reads first.  It is stored with the non-temporal policy: loss and gradient of 8, 64 and 128
// tokens at d 2048, V 128256, over and over, take 495, 581 and 586 us so against 538, 595 and 599, of 16 at d 4096 891
// against 955; with an update of W from dW after each 785, 870 and 867 against 807, 869 and 868, and 1440 against 1484.
// (The kernel itself is slower so: 211 us of 128 tokens against 178, and 700 MB leave L2 for a dW of 525.)  With more
// tokens the stores are spread over the products (256: 736 against 720, 512: 1086 against 1072), and a dW that the cache
// holds is read from there by whoever uses it (16 at d 1024, V 32000: 106 against 101).
template <bool kStream>
__global__ __launch_bounds__(256, 1) void loss_dw_mfma_kernel(const __bf16* __restrict__ G,
                                                              const __bf16* __restrict__ Xc,
                                                              const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                              int Vc, __bf16* __restrict__ dW) {
  using Run = gemm::Tiles<false, false, true, 8, false, 32>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n = __builtin_amdgcn_readfirstlane(n_live[1]);
  const int rows = __builtin_amdgcn_readfirstlane(int(min(int64_t(V) - v0, int64_t(Vc))));
  const int n_m = (d + 255) / 256, n_n = (rows + 255) / 256;
  const gemm::TileOrder order(n_m, n_n);
  const gemm::Operand A{reinterpret_cast<const char*>(Xc), uint32_t(d) * 2u, d};
  const gemm::Operand B{reinterpret_cast<const char*>(G), uint32_t(Vc) * 2u, Vc};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  Run::run(
      lds, A, B, gemm::first_tile(blockIdx.x, gridDim.x), gridDim.x, n_m * n_n,
      [&](int id) {
        const gemm::TileAt t = order(id);
        return gemm::Place{256 * t.m, 256 * t.n, 0, n, 0};
      },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][8]) {
        const int m0 = at.m0, n0 = at.n0, lane = gemm::fresh_lane(), fr = lane & 15, fq = lane >> 4;
        const int live = min(256, rows - n0);
        const buf_rsrc_t o = make_rsrc(dW + (size_t(v0) + n0) * d, uint32_t(live) * uint32_t(d) * 2u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t row = uint32_t(128 * wn + 16 * j + fr) * uint32_t(d);
          const int c0 = m0 + 128 * wm + 8 * fq;  // (of every 32: d is a multiple of 32, all 8 are live or none)
#pragma unroll
          for (int i = 0; i < 8; i += 2)
            buf_store16<kStream ? kNonTemporal : 0>(o, c0 + 16 * i < d ? (row + uint32_t(c0 + 16 * i)) * 2u : kPastEnd,
                        uint4{pack_bf16(acc[i][j][0], acc[i][j][1]), pack_bf16(acc[i][j][2], acc[i][j][3]),
                              pack_bf16(acc[i + 1][j][0], acc[i + 1][j][1]),
                              pack_bf16(acc[i + 1][j][2], acc[i + 1][j][3])});
        }
      });
}

// ------------------------------------------------------------------ plan and workspace

// Rows of G of a token: of few tokens of bf16, whose products would leave half of a tile's columns empty, what the
// rounding of G leaves is a row of its own, so that dX and dW are rounded once: their error is that of one rounding,
// and 1.4 times that (of one token up to 1.7 times) otherwise.  d 2048, V 128256: 30 tokens 428 us with one part, 477
// with two; 64 tokens 453 and 521.
inline int g_parts(int64_t n_tok, int dtype) { return dtype == ESTP_BF16 && n_tok <= 64 ? 2 : 1; }
// How a backward call is cut: Vc vocabulary rows a piece (a multiple of 256), n_split sums of dX in the workspace,
// products of tile_toks tokens.
struct LossPlan {
  int parts;  // of G
  int Vc;
  int n_split;
  int tile_toks;
};

// Tokens of a bf16 tile: 256 read LDS less often, 128 leave fewer columns empty.  d 2048, V 128256, forward and
// backward in us, 128 against 256: 64 tokens 135 and 451, 163 and 497; 200 tokens 148 and 569, 154 and 582; 384
// tokens 203 and 725, 234 and 771; 512 tokens 260 and 889, 242 and 838; 1021 tokens 490 and 1581, 455 and 1438.  The
// sides change at 384 tokens, three tiles of 128, at other shapes too: 384 and 385 tokens, d 4096, V 128256, 387 and
// 1350, 419 and 1420, then 463 and 1548, 420 and 1454; d 1536, V 151936, 186 and 649, 210 and 676, then 225 and 750, 210
// and 695.
inline int bf16_tile_toks(int64_t n_tok) { return n_tok <= 384 ? 128 : 256; }
// The rule of loss_dw_mfma_kernel's kStream.
inline bool stream_dw(int64_t n_tok, int d, int V) {
  constexpr size_t kLastCache = size_t(256) << 20;  // bytes
  return n_tok <= 128 && size_t(V) * d * 2 > kLastCache;
}

// Tokens of a fp32 tile: the narrowest that takes them all, up to 128.  d 2048, V 128256, forward and backward in us:
// 16 tokens 253 and 771 with 32, 379 and 941 with 64, 518 and 1322 with 128; 50 tokens 360 and 1072 with 64, 504 and
// 1434 with 128; 100 tokens 508 and 1676 with 128, 738 and 1780 with 64.
//
// Where 128-wide tiles are fewer than kFewTiles, which leaves compute units idle, 32-wide ones share the work out (of
// dW, whose columns are vocabulary rows, by its own tiles).  Forward and backward in us with 32 against 128: 128
// tokens, d 64, V 1000 (8 tiles) 11.7 and 24.6, 11.9 and 38.5; 128 tokens, d 1024, V 16384 (128) 49 and 144, 75 and
// 176; 400 tokens, d 2048, V 5000 (160) 122 and 315, 141 and 326, V 8000 (252) 161 and 430, 142 and 400.
constexpr size_t kFewTiles = 192;
inline int f32_tile_toks(int64_t n_tok, int V) {
  const size_t tiles = size_t((n_tok + kFT - 1) / kFT) * ((size_t(V) + kFT - 1) / kFT);
  return n_tok <= 32 || tiles < kFewTiles ? 32 : n_tok <= 64 ? 64 : kFT;
}

inline LossPlan plan_loss(int64_t n_tok, int d, int V, int dtype, bool teacher) {
  const size_t es = dtype == ESTP_F32 ? 4 : 2;
  const int64_t tok_pad = (n_tok + 255) / 256 * 256;
  const int64_t v_pad = (int64_t(V) + 255) / 256 * 256;
  int64_t vc = int64_t((size_t(256) << 20) / (es * size_t(tok_pad))) / 256 * 256;
  vc = std::min(std::max<int64_t>(vc, 8192), v_pad);
  // G of 256 MiB or 8192 rows.  4096 tokens: d 4096 the same for 128 to 512 MiB and 1 % slower for 64; d 2048 5.40 ms,
  // 5.33 for 64 and 5.39 for 512.
  LossPlan p;
  p.parts = g_parts(n_tok, dtype);
  p.Vc = int(vc);
  p.tile_toks = dtype == ESTP_F32 ? f32_tile_toks(n_tok, V) : bf16_tile_toks(n_tok);
  // (dX of a distillation, 90 tokens, d 1536, V 151936: 96 columns 372 us, 128 481)
  if (teacher && dtype == ESTP_F32 && p.tile_toks == kFT && (n_tok + 95) / 96 * 96 < (n_tok + kFT - 1) / kFT * kFT)
    p.tile_toks = 96;
  if (teacher && dtype == ESTP_F32 && split::takes(n_tok, d, V)) p.tile_toks = 16 * split::deep_blocks(n_tok);
  const int64_t tiles = (n_tok + p.tile_toks - 1) / p.tile_toks * ((d + 255) / 256);
  p.n_split = int(std::min<int64_t>(std::max<int64_t>(1, 256 / tiles), (vc + 63) / 64));
  return p;
}

// Rows of G, its elements and the floats of dX's sums.
struct LossRoom {
  size_t rows, G, sums;
};
inline LossRoom loss_need(const LossPlan& p, int64_t n_tok, int d) {
  const size_t rows = size_t(p.parts) * size_t(n_tok);
  return {rows, rows * size_t(p.Vc), size_t(p.n_split) * rows * size_t(d)};
}
// At least what every call of n_tok tokens or fewer needs, which can be more than this one: parts, pieces and shares
// follow the token count in steps.  A workspace of a larger call so serves a smaller one.
inline LossRoom loss_room(int64_t n_tok, int d, int V, int dtype) {
  const size_t n = size_t(n_tok), es = dtype == ESTP_F32 ? 4 : 2, v_pad = (size_t(V) + 255) / 256 * 256;
  LossRoom r;
  r.rows = dtype == ESTP_F32 ? n : n <= 64 ? 2 * n : std::max<size_t>(n, 2 * 64);
  // a piece is all of the vocabulary, or 256 MiB of G, or 8192 rows
  r.G = std::min(r.rows * v_pad, std::max((size_t(256) << 20) / es, 8192 * r.rows));
  // t tiles of tokens have at most wide / t shares, and of at least 64 rows each
  const size_t wide = std::max<size_t>(1, 256 / ((size_t(d) + 255) / 256)), tile = dtype == ESTP_F32 ? kFT : 256;
  r.sums = std::max(r.rows, std::min(r.rows * std::min(wide, v_pad / 64), tile * wide)) * size_t(d);
  return r;
}

struct LossBuffers {
  int *row, *slot, *n_live;
  int32_t* tc;
  float *lc, *gc, *acc;
  char *Xc, *G;
  size_t room;   // floats of acc
  size_t bytes;
};

inline LossBuffers carve_loss(const LossRoom& r, int64_t n_tok, int d, int dtype, void* ws) {
  const size_t es = dtype == ESTP_F32 ? 4 : 2;
  Carver c(ws);
  LossBuffers b;
  b.row = c.take<int>(size_t(n_tok));
  b.slot = c.take<int>(size_t(n_tok));
  b.n_live = c.take<int>(2);
  b.tc = c.take<int32_t>(r.rows);
  b.lc = c.take<float>(r.rows);
  b.gc = c.take<float>(r.rows);
  b.Xc = c.take<char>(r.rows * d * es);
  b.G = c.take<char>(r.G * es);
  b.room = r.sums;
  b.acc = c.take<float>(b.room);
  b.bytes = c.bytes();
  return b;
}

template <typename T>
int launch_loss_backward(const void* X, const void* W, const int32_t* targets, const float* lse, const float* grad,
                         int n, int d, int V, int dtype, const Distillation* teacher, void* dX, void* dW,
                         void* workspace, hipStream_t s) {
  const LossPlan p = plan_loss(n, d, V, dtype, teacher != nullptr);
  const LossBuffers b = carve_loss(loss_need(p, n, d), n, d, dtype, workspace);
  constexpr int kWgs = 256;  // of the persistent kernels: one on each compute unit
  const T *Wt = static_cast<const T*>(W), *Xc = reinterpret_cast<const T*>(b.Xc);
  T* G = reinterpret_cast<T*>(b.G);
  const bool by_parts = sizeof(T) == 4 && teacher && split::takes(n, d, V);
  __bf16* parts = reinterpret_cast<__bf16*>(static_cast<char*>(workspace) + b.bytes);
  const float inv_t = teacher ? inverse_temperature(teacher->temperature) : 1.f;
  const float c2 = teacher ? base2_of_logit(teacher->temperature) : kLog2e;
  if (n > 1024)
    loss_list_kernel<<<dim3(1), dim3(1024), 0, s>>>(targets, n, V, p.parts, b.row, b.slot, b.n_live);
  auto gather = n > 1024 ? loss_gather_kernel<false> : loss_gather_kernel<true>;
  gather<<<dim3(unsigned(p.parts * n)), dim3(256), 0, s>>>(
      static_cast<const uint4*>(X), b.row, b.slot, b.n_live, int(size_t(d) * sizeof(T) / 16), targets, n, V, p.parts,
      lse, grad, reinterpret_cast<uint4*>(b.Xc), b.tc, b.lc, b.gc);
  ESTP_CHECK_LAUNCH("loss_gather_kernel");
  const dim3 block(256);
  for (int64_t v0 = 0; v0 < V; v0 += p.Vc) {
    if constexpr (sizeof(T) == 2) {
      const dim3 grid(kWgs);
      const bool odd = d % 64 != 0;
      auto grad_kernel = p.tile_toks == 128 ? (odd ? loss_grad_mfma_kernel<4, true> : loss_grad_mfma_kernel<4, false>)
                                            : (odd ? loss_grad_mfma_kernel<8, true> : loss_grad_mfma_kernel<8, false>);
      // (its 32-bit offsets: 128 rows of a piece of 2^19 columns at most, 2^27 bytes)
      if (teacher && p.parts == 2 && few::takes(n, d, dtype))
        few::choose(n, d, [&](auto steps, auto nb) {
          loss_grad_few_kernel<decltype(steps)::value, decltype(nb)::value>
              <<<dim3(few::workgroups(p.Vc / 16)), dim3(64 * few::kWaves), 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.lc,
                                                                                   b.gc, c2, G);
        });
      else
        grad_kernel<<<grid, block, 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.tc, b.lc, b.gc, c2, G);
      ESTP_CHECK_LAUNCH("loss_grad_mfma_kernel");
      if (teacher) {
        const int rc = launch_teacher_entries(*teacher, n, V, dtype, b.slot, b.n_live, v0, p.Vc, G, s);
        if (rc != ESTP_OK) return rc;
      }
      if (dX) {
        auto dx_kernel = p.tile_toks == 128 ? loss_dx_mfma_kernel<4> : loss_dx_mfma_kernel<8>;
        dx_kernel<<<grid, block, 0, s>>>(G, Wt, b.n_live, d, V, v0, p.Vc, b.room, v0 == 0, b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_mfma_kernel");
      }
      if (dW) {
        if (teacher && p.parts == 2) {
          const int steps = (2 * n + 31) / 32;
          __bf16* columns = parts;
          if (v0 == 0)
            loss_columns_kernel<<<dim3(unsigned(d / 16)), block, 0, s>>>(Xc, b.n_live, d, steps, columns);
          auto kernel = steps == 1   ? loss_dw_few_kernel<1>
                        : steps == 2 ? loss_dw_few_kernel<2>
                        : steps == 3 ? loss_dw_few_kernel<3>
                                     : loss_dw_few_kernel<4>;
          const unsigned along = unsigned(std::max(1, std::min(4, d / 256)));  // of the columns: shares of 256 at least
          kernel<<<dim3(along, unsigned((p.Vc + 255) / 256)), block, 0, s>>>(G, columns, b.n_live, d, V, v0, p.Vc,
                                                                             static_cast<T*>(dW));
          ESTP_CHECK_LAUNCH("loss_dw_few_kernel");
          continue;
        }
        auto dw_kernel = stream_dw(n, d, V) ? loss_dw_mfma_kernel<true> : loss_dw_mfma_kernel<false>;
        dw_kernel<<<grid, block, 0, s>>>(G, Xc, b.n_live, d, V, v0, p.Vc, static_cast<T*>(dW));
        ESTP_CHECK_LAUNCH("loss_dw_mfma_kernel");
      }
    } else {
      const unsigned n_tt = unsigned((n + p.tile_toks - 1) / p.tile_toks), n_dt = unsigned((d + kFT - 1) / kFT);
      const unsigned n_vt = unsigned((p.Vc + kFT - 1) / kFT);
      if (by_parts) {
        if (v0 == 0) split::split_rows_kernel<<<dim3(unsigned(n)), block, 0, s>>>(Xc, n, b.n_live, d, parts);
        split::choose(n, [&](auto nb, auto stream) {
          loss_grad_split_kernel<decltype(nb)::value, decltype(stream)::value>
              <<<dim3(split::kWgs), dim3(64 * split::kWaves), 0, s>>>(parts, n, Wt, b.n_live, d, V, v0, p.Vc, b.lc,
                                                                      b.gc, inv_t, G);
        });
      } else {
        auto grad_kernel = p.tile_toks == 32   ? loss_grad_f32_kernel<32>
                           : p.tile_toks == 64 ? loss_grad_f32_kernel<64>
                           : p.tile_toks == 96 ? loss_grad_f32_kernel<96>
                                               : loss_grad_f32_kernel<kFT>;
        grad_kernel<<<dim3(n_vt, n_tt), block, 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.tc, b.lc, b.gc, inv_t, G);
      }
      ESTP_CHECK_LAUNCH("loss_grad_f32_kernel");
      if (teacher) {
        const int rc = launch_teacher_entries(*teacher, n, V, dtype, b.slot, b.n_live, v0, p.Vc, G, s);
        if (rc != ESTP_OK) return rc;
      }
      if (dX && by_parts) {
        const int n_cols = (d + 255) / 256, n_tiles = n_cols * int(n_tt);
        const int slices = int(std::min<int64_t>(std::max(1, kWgs / n_tiles), (p.Vc + 63) / 64));
        auto kernel = p.tile_toks == 32   ? loss_dx_split_kernel<2>
                      : p.tile_toks == 64 ? loss_dx_split_kernel<4>
                                          : loss_dx_split_kernel<6>;
        kernel<<<dim3(unsigned((int64_t(n_tiles) * slices + 7) / 8 * 8)), dim3(512), 0, s>>>(
            G, Wt, b.n_live, d, V, v0, p.Vc, n_cols, n_tiles, slices, kWgs, b.room, v0 == 0, b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_split_kernel");
      } else if (dX) {
        // (a workgroup for every share there could be, up to a million in all: past that, a loop over the shares)
        const int64_t most = std::max<int64_t>(1, (int64_t(1) << 20) / (int64_t(n_dt) * n_tt));
        const unsigned shares = unsigned(std::min({int64_t(kWgs), int64_t((p.Vc + 63) / 64), most}));
        auto dx_kernel = p.tile_toks == 32   ? loss_dx_f32_kernel<32>
                         : p.tile_toks == 64 ? loss_dx_f32_kernel<64>
                         : p.tile_toks == 96 ? loss_dx_f32_kernel<96>
                                             : loss_dx_f32_kernel<kFT>;
        dx_kernel<<<dim3(n_dt, n_tt, shares), block, 0, s>>>(G, Wt, b.n_live, d, V, v0, p.Vc, kWgs, b.room, v0 == 0,
                                                             b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_f32_kernel");
      }
      if (dW) {
        if (by_parts) {
          const int steps = (n + 31) / 32;
          __bf16* columns = parts + split::parts_bytes(size_t(n), d) / 2;
          if (v0 == 0)
            split::split_columns_kernel<<<dim3(unsigned((d + 15) / 16), unsigned((steps + 2) / 3)), dim3(192), 0, s>>>(
                Xc, b.n_live, d, steps, columns);
          if (n > split::kDeepRows) {
            const int nb = split::deep_blocks(d), n_cols = (d + 16 * nb - 1) / (16 * nb);
            auto kernel = nb == 2   ? loss_dw_split_many_kernel<2>
                          : nb == 4 ? loss_dw_split_many_kernel<4>
                                    : loss_dw_split_many_kernel<6>;
            kernel<<<dim3(unsigned((int64_t(p.Vc / 128) * n_cols + 7) / 8 * 8)), block, 0, s>>>(
                G, columns, steps, b.n_live, d, V, v0, p.Vc, n_cols, static_cast<T*>(dW));
            ESTP_CHECK_LAUNCH("loss_dw_split_many_kernel");
            continue;
          }
          auto kernel = steps == 1   ? loss_dw_split_kernel<1>
                        : steps == 2 ? loss_dw_split_kernel<2>
                                     : loss_dw_split_kernel<3>;
          const unsigned along = unsigned(std::max(1, std::min(4, d / 128)));  // of the columns: shares of 128 at least
          kernel<<<dim3(along, unsigned((p.Vc + 255) / 256)), block, 0, s>>>(G, columns, b.n_live, d, V, v0, p.Vc,
                                                                             static_cast<T*>(dW));
          ESTP_CHECK_LAUNCH("loss_dw_split_kernel");
          continue;
        }
        const bool few = size_t(n_dt) * n_vt < kFewTiles;
        auto dw_kernel = few ? loss_dw_f32_kernel<32> : loss_dw_f32_kernel<kFT>;
        dw_kernel<<<dim3(n_dt, few ? unsigned(p.Vc / 32) : n_vt), block, 0, s>>>(G, Xc, b.n_live, d, V, v0, p.Vc,
                                                                                 static_cast<T*>(dW));
        ESTP_CHECK_LAUNCH("loss_dw_f32_kernel");
      }
    }
  }
  if (dX) {
    const unsigned of_token = unsigned(std::min((d + 1023) / 1024, std::max(1, 2048 / n)));  // few tokens: workgroups
    loss_dx_kernel<T><<<dim3(n, of_token), block, 0, s>>>(
        b.acc, b.slot, b.n_live, d, p.Vc, p.tile_toks, kWgs, b.room, static_cast<T*>(dX));
    ESTP_CHECK_LAUNCH("loss_dx_kernel");
  }
  return ESTP_OK;
}

size_t lm_head_backward_bytes(int64_t n_tok, int d, int V, int dtype, bool teacher) {
  const size_t loss = carve_loss(loss_room(n_tok, d, V, dtype), n_tok, d, dtype, nullptr).bytes;
  if (!teacher) return loss;
  // the parts of fp32 tokens, and columns as the operands of dW
  return loss + (dtype == ESTP_F32 ? split::parts_bytes(size_t(n_tok), d) + split::column_bytes(size_t(n_tok), d)
                                   : size_t(d / 16 + 1) * 4096);
}

int launch_lm_head_backward(const void* X, const void* W, const int32_t* targets, const float* lse, const float* grad,
                            int n, int d, int V, int dtype, const Distillation* teacher, void* dX, void* dW,
                            void* workspace, hipStream_t s) {
  auto launch = dtype == ESTP_F32 ? launch_loss_backward<float> : launch_loss_backward<__bf16>;
  return launch(X, W, targets, lse, grad, n, d, V, dtype, teacher, dX, dW, workspace, s);
}

// How a call that wants no more than lse is cut: tiles of `tile` tokens, the vocabulary tiles in `slices`, `states`
// partial states a token.
struct LsePlan {
  int tile, slices, states;
};
// bf16: a workgroup on every compute unit, tiles as in the backward.  fp32: two workgroups for every compute unit (four
// of the smaller ones).
//
// bf16 calls of more than 8 tiles, whose number does not divide 256, would so leave compute units idle (5 tiles of 52
// at 13 tiles): they take up to four rounds of workgroups, as many slices as make the longest sum of a compute unit's
// tiles shortest, with half a tile for a workgroup's first transfers.
static LsePlan plan_lse(int64_t n_tok, int V, int dtype) {
  LsePlan p;
  const bool f32 = dtype == ESTP_F32;
  p.tile = f32 ? f32_tile_toks(n_tok, V) : bf16_tile_toks(n_tok);
  const int64_t rows = f32 ? kFT : 256, n_vt = (int64_t(V) + rows - 1) / rows, n_tt = (n_tok + p.tile - 1) / p.tile;
  const int64_t fill = !f32 ? 256 : p.tile < kFT ? 1024 : 512;
  p.slices = int(std::min(n_vt, std::max<int64_t>(f32 ? 4 : 1, fill / n_tt)));
  if (!f32 && n_tt > 8) {
    int64_t best = INT64_MAX;
    for (int64_t c = p.slices; c <= std::min(n_vt, std::max<int64_t>(p.slices, 1024 / n_tt)); ++c) {
      const int64_t cost = (n_tt * c + 255) / 256 * (2 * ((n_vt + c - 1) / c) + 1);
      if (cost < best) {
        best = cost;
        p.slices = int(c);
      }
    }
  }
  p.states = p.slices * (f32 && p.tile < kFT ? 4 : 2);
  return p;
}
// At least the partial states of every call of n_tok tokens or fewer, up to `most` (plan_lse gives few tokens more
// slices): a workspace of a larger call serves a smaller one.  slices n_tok is at most fill tile (four times that of
// more than 8 tiles), or 4 n_tok, or n_vt n_tok.
static size_t lse_room(int64_t n_tok, int V, int dtype, bool few) {
  const bool f32 = dtype == ESTP_F32;
  const int64_t rows = f32 ? kFT : 256, n_vt = (int64_t(V) + rows - 1) / rows;
  if (f32) return size_t(4 * std::min(n_vt * n_tok, std::max<int64_t>(4 * n_tok, 1024 * 64)));
  if (few) return size_t(2 * std::min<int64_t>(n_vt * n_tok, 256 * 256));
  return size_t(2 * std::min<int64_t>(n_vt * n_tok, std::max<int64_t>(n_tok, 1024 * 256)));
}

size_t lse_states_bytes(int64_t n_tok, int V, int dtype, bool few) {
  Carver c(nullptr);
  for (int i = 0; i < 2; ++i) c.take<float>(lse_room(n_tok, V, dtype, few));
  return c.bytes();
}

int launch_lse_states(const char* fn, const void* X, const void* W, int n, int d, int V, int dtype, float c2,
                      void* workspace, hipStream_t s, LseStates* out) {
  const LsePlan p = plan_lse(n, V, dtype);
  Carver c(workspace);
  out->m = c.take<float>(size_t(p.states) * size_t(n));
  out->s = c.take<float>(size_t(p.states) * size_t(n));
  out->states = p.states;
  const int n_tt = int((int64_t(n) + p.tile - 1) / p.tile);
  const size_t wgs = size_t(n_tt) * size_t(p.slices);
  ESTP_REQUIRE(fits_launch(wgs + 7, 256), ESTP_ERR_UNSUPPORTED, "%s: n_tok = %d needs %zu workgroups", fn, n, wgs);
  if (dtype == ESTP_F32) {
    auto kernel = p.tile == 32   ? loss_lse_f32_kernel<32>
                  : p.tile == 64 ? loss_lse_f32_kernel<64>
                                 : loss_lse_f32_kernel<kFT>;
    kernel<<<dim3(unsigned(wgs)), dim3(256), 0, s>>>(static_cast<const float*>(X), static_cast<const float*>(W), n, d,
                                                     V, c2, p.slices, out->m, out->s);
  } else {
    auto kernel = p.tile == 128 ? (d % 64 ? loss_lse_mfma_kernel<4, true> : loss_lse_mfma_kernel<4, false>)
                                : (d % 64 ? loss_lse_mfma_kernel<8, true> : loss_lse_mfma_kernel<8, false>);
    kernel<<<dim3(unsigned((wgs + 7) / 8 * 8)), dim3(256), 0, s>>>(static_cast<const __bf16*>(X),
                                                                   static_cast<const __bf16*>(W), n, d, V, c2, n_tt,
                                                                   p.slices, out->m, out->s);
  }
  ESTP_CHECK_LAUNCH("loss_lse_kernel");
  return ESTP_OK;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

namespace {

// bf16 calls of more tokens run the entropy kernel, whose 16 slices then fill the chip.  d 2048, V 128256, here against
// there: 128 tokens 137 and 154 us, 1021 tokens 451 and 626, 2048 tokens 870 and 1220, 2500 tokens 1077 and 991, 4096
// tokens 1735 and 1544; d 4096 2048 tokens 1568 and 2304, 2304 tokens 1767 and 1629; d 1536, V 151936, 782 and 1149, 888
// and 802.  (Figures of a form of loss_lse_mfma_kernel that was a tenth slower; since then it is the faster one of 4096
// tokens at d 4096 too, 2716 and 2882, but the entropy kernel's sums keep one order for any number of tokens, so losses
// keep their last bits, and it forms H and the mode too.)  fp32: the entropy kernel runs on the vector units.
bool own_lse(int64_t n_tok, int dtype) { return dtype == ESTP_F32 || n_tok <= 2048; }

}  // namespace

extern "C" size_t estp_token_loss_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  const size_t entropy = estp_token_entropy_workspace_size(n_tok, d, V, dtype);
  if (entropy == 0) return 0;
  return std::max(entropy, lse_states_bytes(n_tok, V, dtype, true));
}

extern "C" int estp_token_loss(const void* X, const void* W, const int32_t* targets, int64_t n_tok, int32_t d,
                               int32_t V, int dtype, float* loss, float* lse, float* H, int32_t* vocab_argmax,
                               void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_token_loss";
  ESTP_REQUIRE(targets && loss && lse, ESTP_ERR_INVALID_ARG, "%s: targets, loss and lse must be non-null", fn);
  ESTP_REQUIRE(aligned(targets, 4) && aligned(loss, 4) && aligned(lse, 4) && aligned(H, 4) && aligned(vocab_argmax, 4),
               ESTP_ERR_INVALID_ARG, "%s: targets and the outputs must be 4-byte aligned", fn);
  ESTP_REQUIRE(V <= INT32_MAX - 65536, ESTP_ERR_UNSUPPORTED, "%s: V = %d, at most 2^31 - 65537", fn, V);
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  const size_t need = estp_token_loss_workspace_size(n_tok, d, V, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  ESTP_REQUIRE(fits_launch(size_t(n_tok + 3) / 4, 256), ESTP_ERR_UNSUPPORTED,
               "%s: n_tok = %lld needs more workgroups than one launch holds", fn, (long long)n_tok);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int n = int(n_tok);
  const dim3 grid(unsigned((n_tok + 3) / 4)), block(256);
  if (own_lse(n_tok, dtype) && !H && !vocab_argmax) {
    // maximum and sum alone
    LseStates p;
    const int rc = launch_lse_states(fn, X, W, n, d, V, dtype, kLog2e, workspace, s, &p);
    if (rc != ESTP_OK) return rc;
    if (dtype == ESTP_F32)
      loss_pick_kernel<float, true><<<grid, block, 0, s>>>(static_cast<const float*>(X), static_cast<const float*>(W),
                                                           targets, n, d, V, p.m, p.s, p.states, lse, loss);
    else
      loss_pick_kernel<__bf16, true><<<grid, block, 0, s>>>(static_cast<const __bf16*>(X),
                                                            static_cast<const __bf16*>(W), targets, n, d, V, p.m, p.s,
                                                            p.states, lse, loss);
  } else {
    const int rc = launch_token_entropy(X, W, n, d, V, dtype, H, vocab_argmax, lse, workspace, s);
    if (rc != ESTP_OK) return rc;
    if (dtype == ESTP_F32)
      loss_pick_kernel<float, false><<<grid, block, 0, s>>>(static_cast<const float*>(X), static_cast<const float*>(W),
                                                            targets, n, d, V, nullptr, nullptr, 0, lse, loss);
    else
      loss_pick_kernel<__bf16, false><<<grid, block, 0, s>>>(static_cast<const __bf16*>(X),
                                                             static_cast<const __bf16*>(W), targets, n, d, V, nullptr,
                                                             nullptr, 0, lse, loss);
  }
  ESTP_CHECK_LAUNCH("loss_pick_kernel");
  return ESTP_OK;
}

extern "C" size_t estp_token_loss_backward_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  if (n_tok < 1 || d < 1 || V < 1) return 0;
  return lm_head_backward_bytes(n_tok, d, V, dtype, false);
}

extern "C" int estp_token_loss_backward(const void* X, const void* W, const int32_t* targets, const float* lse,
                                        const float* grad, int64_t n_tok, int32_t d, int32_t V, int dtype, void* dX,
                                        void* dW, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_token_loss_backward";
  ESTP_REQUIRE(targets && lse, ESTP_ERR_INVALID_ARG, "%s: targets and lse must be non-null", fn);
  ESTP_REQUIRE(dX || dW, ESTP_ERR_INVALID_ARG, "%s: dX and dW are both null", fn);
  ESTP_REQUIRE(aligned(targets, 4) && aligned(lse, 4) && aligned(grad, 4), ESTP_ERR_INVALID_ARG,
               "%s: targets, lse and grad must be 4-byte aligned", fn);
  ESTP_REQUIRE(aligned(dX, 16) && aligned(dW, 16), ESTP_ERR_INVALID_ARG, "%s: dX and dW must be 16-byte aligned", fn);
  ESTP_REQUIRE(V <= INT32_MAX - 65536, ESTP_ERR_UNSUPPORTED, "%s: V = %d, at most 2^31 - 65537", fn, V);
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(n_tok <= (int64_t(1) << 22), ESTP_ERR_UNSUPPORTED, "%s: n_tok = %lld, at most 4194304", fn,
               (long long)n_tok);
  ESTP_REQUIRE(d <= (1 << 20), ESTP_ERR_UNSUPPORTED, "%s: d = %d, at most 1048576", fn, d);
  ESTP_REQUIRE(n_tok * d <= (int64_t(1) << 36), ESTP_ERR_UNSUPPORTED, "%s: n_tok d = %lld, at most 2^36", fn,
               (long long)n_tok * d);
  const size_t need = estp_token_loss_backward_workspace_size(n_tok, d, V, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return launch_lm_head_backward(X, W, targets, lse, grad, int(n_tok), d, V, dtype, nullptr, dX, dW, workspace, s);
}
