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
#include "lm_head.h"
#include "loss_shares.h"
#include "mfma_gemm.h"

namespace estp {
namespace detail {

// ------------------------------------------------------------------ elementwise parts

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
    // in natural units with one rounding (ln 2 in two parts): weights exp(z - lse) near 1, whose distance from 1 is the
    // gradient, have the error of lse
    constexpr float kLn2Rest = -1.904654299957768e-9f;
    const float t2 = fast_log2(s);
    l = top == -INFINITY ? top + t2 : fmaf(top, kLn2, fmaf(top, kLn2Rest, kLn2 * t2));  // (a NaN in s stays one)
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
//
// C[m][n] = sum_k A(m, k) B(n, k) over 128 x kTN tiles on v_mfma_f32_32x32x2_f32 (without packed instructions the
// vector units reach half its rate), 4 waves of 64 x 64, or of 32 x kTN for the 64 and 32 columns of few tokens.
// Operands lie in memory with k contiguous or strided and reach LDS as they lie, 32 k a stage, two stages of at most 32
// KB, so two or more workgroups share a compute unit.  A lane of a step gives row lane % 32 at one of two k; any order
// of the k will do if both sides keep it: of 8 k, step i takes k = i and 4 + i, so that a lane's four values are one
// 16-byte read where k is contiguous.  kFSum terms at a time are summed before they enter the total, which keeps the
// rounding of long sums small (3 tokens, d 2048: dW off by 2e-7, by 2e-6 with one chain of sums) for 64 additions in
// 256 products.
//
// 400 tokens, d 2048, V 128256 (a product of 210 GFLOP, 153 TFLOP/s at most, a fifth of it on columns that no token
// has): logits 2.15 ms, dX 2.14, dW 1.80 (117 TFLOP/s).  16 tokens, which one pass over the 1.05 GB of W or dW bounds:
// logits 244 us (4.3 TB/s), dX 222, dW 354.
constexpr int kFT = 128, kFK = 32, kFPart = kFT * kFK * 4;
constexpr int kFSum = 128;

template <bool kAK, bool kBK, int kTN>
struct F32Tile {
  static constexpr int kWM = kTN == kFT ? 2 : 4;            // waves along the rows
  static constexpr int kMI = kFT / 32 / kWM, kNJ = kTN == kFT ? 2 : kTN / 32;  // 32 x 32 blocks of a wave
  static constexpr int kPartB = kTN * kFK * 4, kStage = kFPart + kPartB, kLds = 2 * kStage, kLB = kTN / 32;
  using Acc = f32x16_t[kMI][kNJ];
  // What a lane holds: columns n + 32 j, and of each 32 rows from m + 32 i the four runs of four at 8 q.
  struct At {
    int m, n, wm;
  };
  __device__ static __forceinline__ At place(int m0, int n0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave % kWM;
    return {m0 + 32 * kMI * wm + 4 * (lane >> 5), n0 + 32 * kNJ * (wave / kWM) + (lane & 31), wm};
  }
  // byte offset in the source of what lane `lane` of transfer i brings of a part of kRows rows; *kc: its first k where
  // k is contiguous
  template <bool kK, int kRows>
  __device__ static __forceinline__ uint32_t source(int i, int wave, int lane, uint32_t ld, int* kc) {
    const int at = 64 * (4 * i + wave) + lane;
    if (kK) {
      const int row = at / 8, c = (at % 8) ^ (row & 7);
      *kc = 4 * c;
      return uint32_t(row) * ld + uint32_t(c) * 16u;
    }
    *kc = 0;
    return uint32_t(at / (kRows / 4)) * ld + uint32_t(at % (kRows / 4)) * 16u;
  }
  // rows 32 block + lane % 32 at k = 8 g + 4 (lane / 32) .. + 3 of a part in LDS
  template <bool kK, int kRows>
  __device__ static __forceinline__ f32x4_t read(const char* part, int row, int g, int half) {
    if (kK) return *reinterpret_cast<const f32x4_t*>(part + row * 128 + ((2 * g + half) ^ (row & 7)) * 16);
    f32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = *reinterpret_cast<const float*>(part + ((8 * g + 4 * half + i) * kRows + row) * 4);
    return v;
  }
  // acc[i][j] = the product over k in [k0, k1) of the wave's 32 x 32 blocks (mfma32_f32's layout)
  __device__ static __forceinline__ void run(char* lds, const gemm::Operand& A, const gemm::Operand& B, int m0, int n0,
                                             int k0, int k1, Acc& acc) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % kWM, wn = wave / kWM, half = lane >> 5, row = lane & 31;
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
      for (int j = 0; j < kNJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    if (k0 >= k1) return;
    uint32_t off_a[4], off_b[kLB];
    int kc_a[4], kc_b[kLB];
#pragma unroll
    for (int i = 0; i < 4; ++i) off_a[i] = source<kAK, kFT>(i, wave, lane, A.ld, &kc_a[i]);
#pragma unroll
    for (int i = 0; i < kLB; ++i) off_b[i] = source<kBK, kTN>(i, wave, lane, B.ld, &kc_b[i]);
    auto part = [&](auto contig, auto n_parts, const gemm::Operand& o, int r0, int rows, int k, const uint32_t* off,
                    const int* kc, char* dst) {
      constexpr bool kContig = decltype(contig)::value;
      const int left = k1 - k;
      const u32x4_t r = kContig ? rsrc_words(o.base + size_t(r0) * o.ld, uint32_t(min(rows, o.rows - r0)) * o.ld)
                                : rsrc_words(o.base + size_t(k) * o.ld + size_t(r0) * 4,
                                             uint32_t(min(kFK, left)) * o.ld - uint32_t(r0) * 4u);
      const uint32_t soff = kContig ? uint32_t(k) * 4u : 0u;
#pragma unroll
      for (int i = 0; i < decltype(n_parts)::value; ++i)
        dma16(r, kContig && kc[i] >= left ? kPastEnd : off[i], soff, dst + 1024 * (4 * i + wave));
    };
    auto stage = [&](int k, int buf) {
      part(std::bool_constant<kAK>{}, std::integral_constant<int, 4>{}, A, m0, kFT, k, off_a, kc_a, lds + buf * kStage);
      part(std::bool_constant<kBK>{}, std::integral_constant<int, kLB>{}, B, n0, kTN, k, off_b, kc_b,
           lds + buf * kStage + kFPart);
    };
    lds_barrier();  // the last tile's stages are read
    stage(k0, 0);
    int buf = 0;
    Acc part_sum;
    auto clear = [&]() {
#pragma unroll
      for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) part_sum[i][j][r] = 0.f;
    };
    auto add = [&]() {
#pragma unroll
      for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNJ; ++j) acc[i][j] += part_sum[i][j];
    };
    clear();
    int left_in_sum = kFSum;
    for (int k = k0; k < k1; k += kFK, buf ^= 1) {
      if (left_in_sum == 0) {
        add();
        clear();
        left_in_sum = kFSum;
      }
      left_in_sum -= kFK;
      arrived<0>();
      lds_barrier();  // every wave's transfers of the stage have landed, and its reads of the other are done
      if (k + kFK < k1) stage(k + kFK, buf ^ 1);
      const char *pa = lds + buf * kStage, *pb = pa + kFPart;
#pragma unroll
      for (int g = 0; g < kFK / 8; ++g) {
        f32x4_t a[kMI], b[kNJ];
#pragma unroll
        for (int i = 0; i < kMI; ++i) a[i] = read<kAK, kFT>(pa, 32 * (kMI * wm + i) + row, g, half);
#pragma unroll
        for (int j = 0; j < kNJ; ++j) b[j] = read<kBK, kTN>(pb, 32 * (kNJ * wn + j) + row, g, half);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < kMI; ++i)
#pragma unroll
            for (int j = 0; j < kNJ; ++j) part_sum[i][j] = mfma32_f32(a[i][q], b[j][q], part_sum[i][j]);
      }
    }
    add();
  }
};

// Running (maximum, sum) in base 2 of every token's logits over a slice of the vocabulary tiles: slice s of n_slices
// takes tiles s, s + n_slices, ...; each wave's rows of a tile have a state of their own.  Partial states
// [n_tok, kWM n_slices].
template <int kTN>
__global__ __launch_bounds__(256, 2) void loss_lse_f32_kernel(const float* __restrict__ X, const float* __restrict__ W,
                                                              int n_tok, int d, int V, int n_slices,
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
          mx = fmaxf(mx, live ? acc[i][j][r] * kLog2e : -INFINITY);
        }
      const float ref = fmaxf(mx, -0x1p127f);  // finite for a lane with no live row yet
      float sum = l[j] * fast_exp2(fmaxf(m[j] - ref, kExp2Floor));
#pragma unroll
      for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool live = at.m + 32 * i + 8 * (r >> 2) + (r & 3) < V;
          sum += live ? fast_exp2(fmaf(acc[i][j][r], kLog2e, -ref)) : 0.f;
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
                                                               const float* __restrict__ gc, float* __restrict__ G) {
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
          // (z - lse first: near 0 for the weights that matter, so its product is exact to its own rounding)
          const float p = fast_exp2((acc[i][j][4 * q + e] - l) * kLog2e) - (v + e == t ? 1.f : 0.f);
          out[e] = v + e < rows ? g * p : 0.f;
        }
        *reinterpret_cast<f32x4_t*>(G + size_t(s) * Vc + v) = out;
      }
  }
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

// ------------------------------------------------------------------ matrix-core products (bf16)

// Stores of 16 bytes at a byte offset of a buffer resource; past its end nothing is written.
template <int kAux = 0>
__device__ __forceinline__ void buf_store16(buf_rsrc_t r, uint32_t off, uint4 v) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{v.x, v.y, v.z, v.w}, r, off, 0, kAux);
#endif
}

// Running (reference, sum) in base 2 of every token's logits, for calls of few tokens: workgroup (token tile, slice)
// takes the vocabulary tiles slice, slice + n_slices, ..., so that any number of token tiles fills the chip.  The
// first tile's maximum is the reference; later tiles add to the sum with one FMA, exponential and addition a logit,
// and move the reference only where a sum would pass 2^64.  Partial states [n_tok, 2 n_slices], a wave's 128 rows each.
// 61 tokens, d 4096, V 128256: 217 us, 4.8 TB/s of W; 1021 tokens, d 2048: 450 us, 1.19 PFLOP/s.
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void loss_lse_mfma_kernel(const __bf16* __restrict__ X,
                                                               const __bf16* __restrict__ W, int n_tok, int d, int V,
                                                               int n_tt, int n_slices, float* __restrict__ part_m,
                                                               float* __restrict__ part_s) {
  using Run = gemm::Tiles<true, true, false, kNBN, kOdd, 0>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  // token tiles of a slice, which stream the same rows of W, next to each other on one XCD
  const int wg = gemm::first_tile(blockIdx.x, gridDim.x), tt = wg % n_tt, slice = wg / n_tt;
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
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          bool exact = ragged || at.tag == 0;
          if (!exact) {
            float s = l[j];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) s += fast_exp2(fmaf(acc[i][j][r], kLog2e, -m[j]));
            exact = !(s <= 0x1p64f);  // (a NaN takes the exact path and stays one)
            l[j] = exact ? l[j] : s;
          }
          if (exact) {
            float mx = m[j];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) mx = fmaxf(mx, 16 * i + r < lim ? acc[i][j][r] * kLog2e : -INFINITY);
            const float ref = fmaxf(mx, -0x1p127f);  // finite for a lane with no live row yet
            float s = l[j] * fast_exp2(fmaxf(m[j] - ref, kExp2Floor));
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                s += 16 * i + r < lim ? fast_exp2(fmaf(acc[i][j][r], kLog2e, -ref)) : 0.f;
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
// the exponentials between two tiles (4096 tokens, d 4096, 32768 vocabulary rows, 1.1 TFLOP: 830 us, 1.32 PFLOP/s;
// 684 live tokens, d 2048, all of 128256: 353 us, 1.02 PFLOP/s, a ninth of it on columns that no token has).
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void loss_grad_mfma_kernel(const __bf16* __restrict__ Xc,
                                                                const __bf16* __restrict__ W,
                                                                const int* __restrict__ n_live, int d, int V,
                                                                int64_t v0, int Vc, const int32_t* __restrict__ tc,
                                                                const float* __restrict__ lc,
                                                                const float* __restrict__ gc, __bf16* __restrict__ G) {
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
              p[i / 2][4 * (i % 2) + r] = g * fast_exp2(fmaf(acc[i][j][r], kLog2e, -l2));
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

inline LossPlan plan_loss(int64_t n_tok, int d, int V, int dtype) {
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
                         int n, int d, int V, int dtype, void* dX, void* dW, void* workspace, hipStream_t s) {
  const LossPlan p = plan_loss(n, d, V, dtype);
  const LossBuffers b = carve_loss(loss_need(p, n, d), n, d, dtype, workspace);
  constexpr int kWgs = 256;  // of the persistent kernels: one on each compute unit
  const T *Wt = static_cast<const T*>(W), *Xc = reinterpret_cast<const T*>(b.Xc);
  T* G = reinterpret_cast<T*>(b.G);
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
      grad_kernel<<<grid, block, 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.tc, b.lc, b.gc, G);
      ESTP_CHECK_LAUNCH("loss_grad_mfma_kernel");
      if (dX) {
        auto dx_kernel = p.tile_toks == 128 ? loss_dx_mfma_kernel<4> : loss_dx_mfma_kernel<8>;
        dx_kernel<<<grid, block, 0, s>>>(G, Wt, b.n_live, d, V, v0, p.Vc, b.room, v0 == 0, b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_mfma_kernel");
      }
      if (dW) {
        auto dw_kernel = stream_dw(n, d, V) ? loss_dw_mfma_kernel<true> : loss_dw_mfma_kernel<false>;
        dw_kernel<<<grid, block, 0, s>>>(G, Xc, b.n_live, d, V, v0, p.Vc, static_cast<T*>(dW));
        ESTP_CHECK_LAUNCH("loss_dw_mfma_kernel");
      }
    } else {
      const unsigned n_tt = unsigned((n + p.tile_toks - 1) / p.tile_toks), n_dt = unsigned((d + kFT - 1) / kFT);
      const unsigned n_vt = unsigned((p.Vc + kFT - 1) / kFT);
      auto grad_kernel = p.tile_toks == 32   ? loss_grad_f32_kernel<32>
                         : p.tile_toks == 64 ? loss_grad_f32_kernel<64>
                                             : loss_grad_f32_kernel<kFT>;
      grad_kernel<<<dim3(n_vt, n_tt), block, 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.tc, b.lc, b.gc, G);
      ESTP_CHECK_LAUNCH("loss_grad_f32_kernel");
      if (dX) {
        // (a workgroup for every share there could be, up to a million in all: past that, a loop over the shares)
        const int64_t most = std::max<int64_t>(1, (int64_t(1) << 20) / (int64_t(n_dt) * n_tt));
        const unsigned shares = unsigned(std::min({int64_t(kWgs), int64_t((p.Vc + 63) / 64), most}));
        auto dx_kernel = p.tile_toks == 32   ? loss_dx_f32_kernel<32>
                         : p.tile_toks == 64 ? loss_dx_f32_kernel<64>
                                             : loss_dx_f32_kernel<kFT>;
        dx_kernel<<<dim3(n_dt, n_tt, shares), block, 0, s>>>(G, Wt, b.n_live, d, V, v0, p.Vc, kWgs, b.room, v0 == 0,
                                                             b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_f32_kernel");
      }
      if (dW) {
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

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

namespace {

// How a call that wants no more than lse is cut: tiles of `tile` tokens, the vocabulary tiles in `slices`, `states`
// partial states a token.
struct LsePlan {
  int tile, slices, states;
};
// bf16: a workgroup on every compute unit, tiles as in the backward.  fp32: two workgroups for every compute unit (four
// of the smaller ones).
LsePlan plan_lse(int64_t n_tok, int V, int dtype) {
  LsePlan p;
  const bool f32 = dtype == ESTP_F32;
  p.tile = f32 ? f32_tile_toks(n_tok, V) : bf16_tile_toks(n_tok);
  const int64_t rows = f32 ? kFT : 256, n_vt = (int64_t(V) + rows - 1) / rows, n_tt = (n_tok + p.tile - 1) / p.tile;
  const int64_t fill = !f32 ? 256 : p.tile < kFT ? 1024 : 512;
  p.slices = int(std::min(n_vt, std::max<int64_t>(f32 ? 4 : 1, fill / n_tt)));
  p.states = p.slices * (f32 && p.tile < kFT ? 4 : 2);
  return p;
}
// At least the partial states of every call of n_tok tokens or fewer (plan_lse gives few tokens more slices): a workspace
// of a larger call serves a smaller one.  slices n_tok is at most fill tile, or 4 n_tok, or n_vt n_tok.
size_t lse_room(int64_t n_tok, int V, int dtype) {
  const bool f32 = dtype == ESTP_F32;
  const int64_t rows = f32 ? kFT : 256, n_vt = (int64_t(V) + rows - 1) / rows;
  if (f32) return size_t(4 * std::min(n_vt * n_tok, std::max<int64_t>(4 * n_tok, 1024 * 64)));
  return size_t(2 * std::min<int64_t>(n_vt * n_tok, 256 * 256));
}
// bf16 calls of more tokens run the entropy kernel, whose 16 slices then fill the chip.  d 2048, V 128256, here against
// there: 128 tokens 137 and 154 us, 1021 tokens 451 and 626, 2048 tokens 870 and 1220, 2500 tokens 1077 and 991, 4096
// tokens 1735 and 1544; d 4096 2048 tokens 1568 and 2304, 2304 tokens 1767 and 1629; d 1536, V 151936, 782 and 1149, 888
// and 802.  (Its sums keep one order for any number of tokens, and it forms H and the mode too.)  fp32:
// the entropy kernel runs on the vector units.
bool own_lse(int64_t n_tok, int dtype) { return dtype == ESTP_F32 || n_tok <= 2048; }

}  // namespace

extern "C" size_t estp_token_loss_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  const size_t entropy = estp_token_entropy_workspace_size(n_tok, d, V, dtype);
  if (entropy == 0) return 0;
  Carver c(nullptr);
  for (int i = 0; i < 2; ++i) c.take<float>(lse_room(n_tok, V, dtype));
  return std::max(entropy, c.bytes());
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
    const LsePlan p = plan_lse(n_tok, V, dtype);
    Carver c(workspace);
    float* pm = c.take<float>(size_t(p.states) * size_t(n_tok));
    float* ps = c.take<float>(size_t(p.states) * size_t(n_tok));
    const int n_tt = int((n_tok + p.tile - 1) / p.tile);
    const size_t wgs = size_t(n_tt) * size_t(p.slices);
    ESTP_REQUIRE(fits_launch(wgs + 7, 256), ESTP_ERR_UNSUPPORTED, "%s: n_tok = %d needs %zu workgroups", fn, n, wgs);
    if (dtype == ESTP_F32) {
      auto kernel = p.tile == 32   ? loss_lse_f32_kernel<32>
                    : p.tile == 64 ? loss_lse_f32_kernel<64>
                                   : loss_lse_f32_kernel<kFT>;
      kernel<<<dim3(unsigned(wgs)), dim3(256), 0, s>>>(static_cast<const float*>(X), static_cast<const float*>(W), n, d,
                                                       V, p.slices, pm, ps);
    } else {
      auto kernel = p.tile == 128 ? (d % 64 ? loss_lse_mfma_kernel<4, true> : loss_lse_mfma_kernel<4, false>)
                                  : (d % 64 ? loss_lse_mfma_kernel<8, true> : loss_lse_mfma_kernel<8, false>);
      kernel<<<dim3(unsigned((wgs + 7) / 8 * 8)), dim3(256), 0, s>>>(static_cast<const __bf16*>(X),
                                                                     static_cast<const __bf16*>(W), n, d, V, n_tt,
                                                                     p.slices, pm, ps);
    }
    ESTP_CHECK_LAUNCH("loss_lse_kernel");
    if (dtype == ESTP_F32)
      loss_pick_kernel<float, true><<<grid, block, 0, s>>>(static_cast<const float*>(X), static_cast<const float*>(W),
                                                           targets, n, d, V, pm, ps, p.states, lse, loss);
    else
      loss_pick_kernel<__bf16, true><<<grid, block, 0, s>>>(static_cast<const __bf16*>(X),
                                                            static_cast<const __bf16*>(W), targets, n, d, V, pm, ps,
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
  return carve_loss(loss_room(n_tok, d, V, dtype), n_tok, d, dtype, nullptr).bytes;
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
  const int n = int(n_tok);
  auto launch = dtype == ESTP_F32 ? launch_loss_backward<float> : launch_loss_backward<__bf16>;
  return launch(X, W, targets, lse, grad, n, d, V, dtype, dX, dW, workspace, s);
}
