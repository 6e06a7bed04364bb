// LM-head loss and its gradient: softmax cross entropy of given next tokens
// over the whole vocabulary, without the n_tok x V logits.
//
//   z_i = W x_i,  lse_i = log sum_v exp z_i[v],  loss_i = lse_i - z_i[t_i]
//   G_iv = g_i (exp(z_i[v] - lse_i) - [v = t_i]),  dX = G W,  dW = G^T X
//
// Forward: lse comes from the entropy kernels (entropy.hip), whose running
// maximum and sum it is; loss_pick_kernel forms z_i[t_i] from one row of each
// operand.  A token whose target lies outside [0, V) is ignored: loss 0, no
// gradient, and its row of X (padding may hold anything) is never multiplied.
//
// Backward: the live tokens' rows are first gathered next to each other
// (loss_list_kernel, loss_gather_kernel), so that ignored tokens cost nothing
// and cannot put a NaN into dW.  Then, for one piece of the vocabulary after
// the other, three products: the piece's logits again, turned into G in their
// epilogue; dX += G W_piece in fp32; dW_piece = G^T X, written once.  G is held
// in the inputs' type (bf16: one rounding of each entry, 2^-8 relative, the
// type in which the matrix cores take it; the sums over it are fp32).  Last,
// loss_dx_kernel rounds dX once and puts it into the tokens' places.
#include <algorithm>

#include "estp_common.h"
#include "lm_head.h"
#include "mfma_gemm.h"

namespace estp {
namespace detail {

// ------------------------------------------------------------------ elementwise parts

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ float to_f32<__bf16>(__bf16 v) {
  return float(v);
}

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

// loss_i = lse_i - x_i . W[t_i], one wave per token.  A sum of probabilities is at most 1, so a
// difference below 0 is rounding and is returned as 0.
template <typename T>
__global__ __launch_bounds__(256) void loss_pick_kernel(const T* __restrict__ X, const T* __restrict__ W,
                                                        const int32_t* __restrict__ targets, int n_tok, int d, int V,
                                                        const float* __restrict__ lse, float* __restrict__ loss) {
  const int tok = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tok >= n_tok) return;
  const int t = targets[tok];
  if (t < 0 || t >= V) {
    if (lane == 0) loss[tok] = 0.f;
    return;
  }
  float s = 0.f;
  for (int k = 8 * lane; k < d; k += 512) s = dot8(X + size_t(tok) * d + k, W + size_t(t) * d + k, s);
  s = wave_sum(s);
  const float l = lse[tok] - s;
  if (lane == 0) loss[tok] = l < 0.f ? 0.f : l;
}

// The live tokens in ascending order: row[slot] = token, slot[token] = slot or -1, n_live[0].  One
// workgroup; each thread counts a contiguous run of tokens.
__global__ __launch_bounds__(1024) void loss_list_kernel(const int32_t* __restrict__ targets, int n_tok, int V,
                                                         int* __restrict__ row, int* __restrict__ slot,
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
  if (tid == 0) n_live[0] = base;
}

// Rows, targets, normalisers and weights of the live tokens, next to each other.  16-byte pieces of rows.
__global__ __launch_bounds__(256) void loss_gather_kernel(const uint4* __restrict__ X, const int* __restrict__ row,
                                                          const int* __restrict__ n_live, int row16,
                                                          const int32_t* __restrict__ targets,
                                                          const float* __restrict__ lse, const float* __restrict__ grad,
                                                          uint4* __restrict__ Xc, int32_t* __restrict__ tc,
                                                          float* __restrict__ lc, float* __restrict__ gc) {
  const int s = blockIdx.x;
  if (s >= n_live[0]) return;
  const int tok = row[s];
  for (int k = threadIdx.x; k < row16; k += 256) Xc[size_t(s) * row16 + k] = X[size_t(tok) * row16 + k];
  if (threadIdx.x == 0) {
    tc[s] = targets[tok];
    lc[s] = lse[tok];
    gc[s] = grad ? grad[tok] : 1.f;
  }
}

// Shares of a piece's vocabulary rows whose products add up to its part of dX: as many as give a workgroup each to
// the chip, while the fp32 sums of all shares (n live rows each) fit into `room` floats.  The same on every piece
// and for every kernel of a call.
struct Shares {
  int n;     // shares
  int rows;  // vocabulary rows of a share, a multiple of 256
};
__device__ __forceinline__ Shares dx_shares(int n_live, int d, int Vc, int tile_toks, int wgs, size_t room) {
  const int tiles = (n_live + tile_toks - 1) / tile_toks * ((d + 255) / 256);
  int s = tiles > 0 ? max(1, wgs / tiles) : 1;
  s = min(s, (Vc + 511) / 512);
  const size_t each = size_t(max(1, n_live)) * d;
  s = int(min(size_t(s), max(size_t(1), room / each)));
  const int rows = ((Vc + s - 1) / s + 255) / 256 * 256;
  return {(Vc + rows - 1) / rows, rows};
}

// dX of every token from the partial sums of its slot, rounded once; 0 for ignored tokens.
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_kernel(const float* __restrict__ acc, const int* __restrict__ slot,
                                                      const int* __restrict__ n_live, int d, int Vc, int tile_toks,
                                                      int wgs, size_t room, T* __restrict__ dX) {
  const int tok = blockIdx.x, s = slot[tok], n = n_live[0];
  const Shares sh = dx_shares(n, d, Vc, tile_toks, wgs, room);
  const size_t each = size_t(n) * d;
  for (int k = 4 * threadIdx.x; k < d; k += 1024) {
    f32x4_t v{0.f, 0.f, 0.f, 0.f};
    if (s >= 0)
      for (int p = 0; p < sh.n; ++p) v += *reinterpret_cast<const f32x4_t*>(acc + p * each + size_t(s) * d + k);
    T* o = dX + size_t(tok) * d + k;
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = T(v[q]);
  }
}

// ------------------------------------------------------------------ vector-unit products
//
// C[m][n] = sum_k A(m, k) B(n, k) over 128 x 128 tiles, 8 x 8 of them a thread, 16 deep stages held k-major in
// LDS (double-buffered, the next stage loaded into registers meanwhile).  An operand lies in memory with k
// contiguous (A[m * ld + k]) or with its rows contiguous (A[k * ld + m]).
constexpr int kPT = 128, kPK = 16, kPPitch = 132;

// 128 rows x 16 k of one operand: two groups of 4 elements a thread.
template <typename T, bool kKContig>
struct PieceLoad {
  float v[2][4];
  // element (r, k) for r < rows, k < depth; elsewhere 0
  __device__ __forceinline__ void load(const T* p, size_t ld, int rows, int depth, int tid) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = tid + 256 * i;
      const int r = kKContig ? q >> 2 : 4 * (q & 31), k = kKContig ? 4 * (q & 3) : q >> 5;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int rr = kKContig ? r : r + j, kk = kKContig ? k + j : k;
        v[i][j] = rr < rows && kk < depth ? to_f32<T>(p[kKContig ? size_t(rr) * ld + kk : size_t(kk) * ld + rr]) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void store(float (*lds)[kPPitch], int tid) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int q = tid + 256 * i;
      const int r = kKContig ? q >> 2 : 4 * (q & 31), k = kKContig ? 4 * (q & 3) : q >> 5;
#pragma unroll
      for (int j = 0; j < 4; ++j) lds[kKContig ? k + j : k][kKContig ? r : r + j] = v[i][j];
    }
  }
};

// acc[i][j] += the product of the tile at rows m0, columns n0 over k in [k0, k1): rows 4 rv .. + 3 and 64 + 4 rv .. + 3,
// columns 4 ct .. + 3 and 64 + 4 ct .. + 3 with rv = tid / 16, ct = tid % 16.
template <typename TA, typename TB, bool kAK, bool kBK>
__device__ __forceinline__ void tile_product(const TA* A, size_t lda, int M, const TB* B, size_t ldb, int N, int m0,
                                             int n0, int k0, int k1, float (&acc)[8][8]) {
  __shared__ __attribute__((aligned(16))) float as[2][kPK][kPPitch];
  __shared__ __attribute__((aligned(16))) float bs[2][kPK][kPPitch];
  const int tid = threadIdx.x, rv = tid >> 4, ct = tid & 15;
  PieceLoad<TA, kAK> la;
  PieceLoad<TB, kBK> lb;
  auto load = [&](int k) {
    la.load(A + (kAK ? size_t(m0) * lda + k : size_t(k) * lda + m0), lda, M - m0, k1 - k, tid);
    lb.load(B + (kBK ? size_t(n0) * ldb + k : size_t(k) * ldb + n0), ldb, N - n0, k1 - k, tid);
  };
  if (k0 >= k1) return;
  load(k0);
  la.store(as[0], tid);
  lb.store(bs[0], tid);
  __syncthreads();
  int buf = 0;
  for (int k = k0; k < k1; k += kPK, buf ^= 1) {
    const bool more = k + kPK < k1;
    if (more) load(k + kPK);
#pragma unroll
    for (int q = 0; q < kPK; ++q) {
      float a[8], b[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(&as[buf][q][64 * h + 4 * rv]);
        const f32x4_t y = *reinterpret_cast<const f32x4_t*>(&bs[buf][q][64 * h + 4 * ct]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          a[4 * h + j] = x[j];
          b[4 * h + j] = y[j];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
    }
    if (more) {
      la.store(as[buf ^ 1], tid);
      lb.store(bs[buf ^ 1], tid);
    }
    __syncthreads();
  }
}
__device__ __forceinline__ int tile_at(int group, int i) { return (i < 4 ? 4 * group + i : 64 + 4 * group + i - 4); }

// G[slot][v] of vocabulary rows v0 .. v0 + Vc (columns past V: 0), pitch Vc.
template <typename T>
__global__ __launch_bounds__(256) void loss_grad_kernel(const T* __restrict__ Xc, const T* __restrict__ W,
                                                        const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                        int Vc, const int32_t* __restrict__ tc,
                                                        const float* __restrict__ lc, const float* __restrict__ gc,
                                                        T* __restrict__ G) {
  const int n = n_live[0], m0 = blockIdx.y * kPT, c0 = blockIdx.x * kPT;
  if (m0 >= n) return;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  float acc[8][8] = {};
  tile_product<T, T, true, true>(Xc, d, n, W + size_t(v0) * d, d, rows, m0, c0, 0, d, acc);
  const int rv = threadIdx.x >> 4, ct = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = m0 + tile_at(rv, i);
    if (s >= n) continue;
    const int t = int(tc[s] - v0);
    const float l2 = lc[s] * kLog2e, g = gc[s];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = c0 + tile_at(ct, j);
      if (c >= Vc) continue;
      const float p = fast_exp2(fmaf(acc[i][j], kLog2e, -l2)) - (c == t ? 1.f : 0.f);
      G[size_t(s) * Vc + c] = T(c < rows ? g * p : 0.f);
    }
  }
}

// out[s][k] (+)= sum over the blockIdx.z-th share of the piece's vocabulary rows of G[s][v] W[v0 + v][k]
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_piece_kernel(const T* __restrict__ G, const T* __restrict__ W,
                                                            const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                            int Vc, int wgs, size_t room, bool first,
                                                            float* __restrict__ out) {
  const int n = n_live[0], m0 = blockIdx.y * kPT, n0 = blockIdx.x * kPT;
  const Shares sh = dx_shares(n, d, Vc, kPT, wgs, room);
  if (m0 >= n || int(blockIdx.z) >= sh.n) return;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  const int k0 = min(rows, int(blockIdx.z) * sh.rows), k1 = min(rows, k0 + sh.rows);
  float acc[8][8] = {};
  tile_product<T, T, true, false>(G, Vc, n, W + size_t(v0) * d, d, d, m0, n0, k0, k1, acc);
  out += size_t(blockIdx.z) * size_t(n) * d;
  const int rv = threadIdx.x >> 4, ct = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int s = m0 + tile_at(rv, i), k = n0 + tile_at(ct, j);
      if (s >= n || k >= d) continue;
      float* o = out + size_t(s) * d + k;
      *o = first ? acc[i][j] : *o + acc[i][j];
    }
}

// dW[v0 + v][k] = sum over the live tokens of G[s][v] Xc[s][k]
template <typename T>
__global__ __launch_bounds__(256) void loss_dw_kernel(const T* __restrict__ G, const T* __restrict__ Xc,
                                                      const int* __restrict__ n_live, int d, int V, int64_t v0, int Vc,
                                                      T* __restrict__ dW) {
  const int n = n_live[0], m0 = blockIdx.y * kPT, n0 = blockIdx.x * kPT;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  if (m0 >= rows) return;
  float acc[8][8] = {};
  tile_product<T, T, false, false>(G, Vc, rows, Xc, d, d, m0, n0, 0, n, acc);
  const int rv = threadIdx.x >> 4, ct = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int v = m0 + tile_at(rv, i), k = n0 + tile_at(ct, j);
      if (v < rows && k < d) dW[(size_t(v0) + v) * d + k] = T(acc[i][j]);
    }
}

// ------------------------------------------------------------------ matrix-core products (bf16)

// Stores of 8 and 16 bytes at a byte offset of a buffer resource; past its end nothing is written.
__device__ __forceinline__ void buf_store8(buf_rsrc_t r, uint32_t off, uint2 v) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{v.x, v.y}, r, off, 0, 0);
#endif
}
__device__ __forceinline__ void buf_store16(buf_rsrc_t r, uint32_t off, uint4 v) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{v.x, v.y, v.z, v.w}, r, off, 0, 0);
#endif
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2_t{__bf16(lo), __bf16(hi)});
}

// G of a piece: products of W's rows (M side) and the live tokens (N side), turned into G as they leave the matrix
// cores.  A lane holds 8 consecutive vocabulary rows of a token: one 16-byte store.
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void loss_grad_mfma_kernel(const __bf16* __restrict__ Xc,
                                                                const __bf16* __restrict__ W,
                                                                const int* __restrict__ n_live, int d, int V,
                                                                int64_t v0, int Vc, const int32_t* __restrict__ tc,
                                                                const float* __restrict__ lc,
                                                                const float* __restrict__ gc, __bf16* __restrict__ G) {
  using Run = gemm::Tiles<true, true, true, kNBN, kOdd>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n = __builtin_amdgcn_readfirstlane(n_live[0]);
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
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          const int sl = 16 * kNBN * wn + 16 * j + fr, s = min(n0 + sl, n - 1);
          const float l2 = lc[s] * kLog2e, g = gc[s];
          const int rel = int(tc[s] - v0) - c0;  // the target is column rel of the lane's 128, 8 of every 32
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
#pragma unroll
          for (int q = 0; q < 4; ++q)
            buf_store16(out, uint32_t(sl) * uint32_t(Vc) * 2u + uint32_t(c0 + 32 * q) * 2u,
                        uint4{pack_bf16(p[q][0], p[q][1]), pack_bf16(p[q][2], p[q][3]), pack_bf16(p[q][4], p[q][5]),
                              pack_bf16(p[q][6], p[q][7])});
        }
      });
}

// out[share][slot][k] (+)= G W_piece over the share's vocabulary rows.  M side: columns k of W (transposed reads), N
// side: slots.
template <int kNBN>
__global__ __launch_bounds__(256, 1) void loss_dx_mfma_kernel(const __bf16* __restrict__ G,
                                                              const __bf16* __restrict__ W,
                                                              const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                              int Vc, size_t room, bool first,
                                                              float* __restrict__ out) {
  using Run = gemm::Tiles<false, true, false, kNBN, false>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n = __builtin_amdgcn_readfirstlane(n_live[0]);
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
        return gemm::Place{256 * t.m, Run::kBN * t.n, min(rows, share * sh.rows), min(rows, (share + 1) * sh.rows),
                           share};
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
// the depth.
__global__ __launch_bounds__(256, 1) void loss_dw_mfma_kernel(const __bf16* __restrict__ G,
                                                              const __bf16* __restrict__ Xc,
                                                              const int* __restrict__ n_live, int d, int V, int64_t v0,
                                                              int Vc, __bf16* __restrict__ dW) {
  using Run = gemm::Tiles<false, false, false, 8, false>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int n = __builtin_amdgcn_readfirstlane(n_live[0]);
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
          const int c0 = m0 + 128 * wm + 4 * fq;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            buf_store8(o, c0 + 16 * i < d ? (row + uint32_t(c0 + 16 * i)) * 2u : kPastEnd,
                       uint2{pack_bf16(acc[i][j][0], acc[i][j][1]), pack_bf16(acc[i][j][2], acc[i][j][3])});
        }
      });
}

// ------------------------------------------------------------------ plan and workspace

// How a backward call is cut: Vc vocabulary rows a piece (a multiple of 256), n_split sums of dX in the workspace,
// products of tile_toks tokens.
struct LossPlan {
  int Vc;
  int n_split;
  int tile_toks;
};

inline LossPlan plan_loss(int64_t n_tok, int d, int V, int dtype) {
  const size_t es = dtype == ESTP_F32 ? 4 : 2;
  const int64_t tok_pad = (n_tok + 255) / 256 * 256;
  const int64_t v_pad = (int64_t(V) + 255) / 256 * 256;
  int64_t vc = int64_t((size_t(256) << 20) / (es * size_t(tok_pad))) / 256 * 256;
  vc = std::min(std::max<int64_t>(vc, 8192), v_pad);
  LossPlan p;
  p.Vc = int(vc);
  p.tile_toks = dtype == ESTP_F32 ? kPT : n_tok <= 128 ? 128 : 256;
  const int64_t tiles = (n_tok + p.tile_toks - 1) / p.tile_toks * ((d + 255) / 256);
  p.n_split = int(std::min<int64_t>(std::max<int64_t>(1, 256 / tiles), (vc + 511) / 512));
  return p;
}

struct LossBuffers {
  int *row, *slot, *n_live;
  int32_t* tc;
  float *lc, *gc, *acc;
  char *Xc, *G;
  size_t room;   // floats of acc
  size_t bytes;
};

inline LossBuffers carve_loss(const LossPlan& p, int64_t n_tok, int d, int dtype, void* ws) {
  const size_t es = dtype == ESTP_F32 ? 4 : 2;
  Carver c(ws);
  LossBuffers b;
  b.row = c.take<int>(size_t(n_tok));
  b.slot = c.take<int>(size_t(n_tok));
  b.n_live = c.take<int>(1);
  b.tc = c.take<int32_t>(size_t(n_tok));
  b.lc = c.take<float>(size_t(n_tok));
  b.gc = c.take<float>(size_t(n_tok));
  b.Xc = c.take<char>(size_t(n_tok) * d * es);
  b.G = c.take<char>(size_t(n_tok) * p.Vc * es);
  b.room = size_t(p.n_split) * size_t(n_tok) * d;
  b.acc = c.take<float>(b.room);
  b.bytes = c.bytes();
  return b;
}

template <typename T>
int launch_loss_backward(const void* X, const void* W, const int32_t* targets, const float* lse, const float* grad,
                         int n, int d, int V, int dtype, void* dX, void* dW, void* workspace, hipStream_t s) {
  const LossPlan p = plan_loss(n, d, V, dtype);
  const LossBuffers b = carve_loss(p, n, d, dtype, workspace);
  constexpr int kWgs = 256;  // of the persistent kernels: one on each compute unit
  const T *Wt = static_cast<const T*>(W), *Xc = reinterpret_cast<const T*>(b.Xc);
  T* G = reinterpret_cast<T*>(b.G);
  loss_list_kernel<<<dim3(1), dim3(1024), 0, s>>>(targets, n, V, b.row, b.slot, b.n_live);
  loss_gather_kernel<<<dim3(n), dim3(256), 0, s>>>(static_cast<const uint4*>(X), b.row, b.n_live,
                                                   int(size_t(d) * sizeof(T) / 16), targets, lse, grad,
                                                   reinterpret_cast<uint4*>(b.Xc), b.tc, b.lc, b.gc);
  ESTP_CHECK_LAUNCH("loss_gather_kernel");
  const dim3 block(256);
  for (int64_t v0 = 0; v0 < V; v0 += p.Vc) {
    if constexpr (sizeof(T) == 2) {
      const dim3 grid(kWgs);
      auto grad_kernel = p.tile_toks == 128 ? (d % 64 ? loss_grad_mfma_kernel<4, true> : loss_grad_mfma_kernel<4, false>)
                                            : (d % 64 ? loss_grad_mfma_kernel<8, true> : loss_grad_mfma_kernel<8, false>);
      grad_kernel<<<grid, block, 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.tc, b.lc, b.gc, G);
      ESTP_CHECK_LAUNCH("loss_grad_mfma_kernel");
      if (dX) {
        auto dx_kernel = p.tile_toks == 128 ? loss_dx_mfma_kernel<4> : loss_dx_mfma_kernel<8>;
        dx_kernel<<<grid, block, 0, s>>>(G, Wt, b.n_live, d, V, v0, p.Vc, b.room, v0 == 0, b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_mfma_kernel");
      }
      if (dW) {
        loss_dw_mfma_kernel<<<grid, block, 0, s>>>(G, Xc, b.n_live, d, V, v0, p.Vc, static_cast<T*>(dW));
        ESTP_CHECK_LAUNCH("loss_dw_mfma_kernel");
      }
    } else {
      const unsigned n_tt = unsigned((n + kPT - 1) / kPT), n_dt = unsigned((d + kPT - 1) / kPT);
      const unsigned n_vt = unsigned((p.Vc + kPT - 1) / kPT);
      loss_grad_kernel<T><<<dim3(n_vt, n_tt), block, 0, s>>>(Xc, Wt, b.n_live, d, V, v0, p.Vc, b.tc, b.lc, b.gc, G);
      ESTP_CHECK_LAUNCH("loss_grad_kernel");
      if (dX) {
        const unsigned shares = unsigned(std::min<int64_t>(kWgs, (p.Vc + 511) / 512));
        loss_dx_piece_kernel<T><<<dim3(n_dt, n_tt, shares), block, 0, s>>>(G, Wt, b.n_live, d, V, v0, p.Vc, kWgs,
                                                                           b.room, v0 == 0, b.acc);
        ESTP_CHECK_LAUNCH("loss_dx_piece_kernel");
      }
      if (dW) {
        loss_dw_kernel<T><<<dim3(n_dt, n_vt), block, 0, s>>>(G, Xc, b.n_live, d, V, v0, p.Vc, static_cast<T*>(dW));
        ESTP_CHECK_LAUNCH("loss_dw_kernel");
      }
    }
  }
  if (dX) {
    loss_dx_kernel<T><<<dim3(n), block, 0, s>>>(b.acc, b.slot, b.n_live, d, p.Vc, p.tile_toks, kWgs, b.room,
                                                static_cast<T*>(dX));
    ESTP_CHECK_LAUNCH("loss_dx_kernel");
  }
  return ESTP_OK;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_token_loss_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  return estp_token_entropy_workspace_size(n_tok, d, V, dtype);
}

extern "C" int estp_token_loss(const void* X, const void* W, const int32_t* targets, int64_t n_tok, int32_t d,
                               int32_t V, int dtype, float* loss, float* lse, float* H, int32_t* vocab_argmax,
                               void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_token_loss";
  ESTP_REQUIRE(targets && loss && lse, ESTP_ERR_INVALID_ARG, "%s: targets, loss and lse must be non-null", fn);
  ESTP_REQUIRE(aligned(targets, 4) && aligned(loss, 4) && aligned(lse, 4) && aligned(H, 4) && aligned(vocab_argmax, 4),
               ESTP_ERR_INVALID_ARG, "%s: targets and the outputs must be 4-byte aligned", fn);
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  const size_t need = estp_token_loss_workspace_size(n_tok, d, V, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int n = int(n_tok);
  const int rc = launch_token_entropy(X, W, n, d, V, dtype, H, vocab_argmax, lse, workspace, s);
  if (rc != ESTP_OK) return rc;
  const dim3 grid(unsigned((n_tok + 3) / 4)), block(256);
  if (dtype == ESTP_F32)
    loss_pick_kernel<float><<<grid, block, 0, s>>>(static_cast<const float*>(X), static_cast<const float*>(W), targets,
                                                   n, d, V, lse, loss);
  else
    loss_pick_kernel<__bf16><<<grid, block, 0, s>>>(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W),
                                                    targets, n, d, V, lse, loss);
  ESTP_CHECK_LAUNCH("loss_pick_kernel");
  return ESTP_OK;
}

extern "C" size_t estp_token_loss_backward_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  if (n_tok < 1 || d < 1 || V < 1) return 0;
  return carve_loss(plan_loss(n_tok, d, V, dtype), n_tok, d, dtype, nullptr).bytes;
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
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(n_tok <= (int64_t(1) << 22), ESTP_ERR_UNSUPPORTED, "%s: n_tok = %lld, at most 4194304", fn,
               (long long)n_tok);
  ESTP_REQUIRE(d <= (1 << 20), ESTP_ERR_UNSUPPORTED, "%s: d = %d, at most 1048576", fn, d);
  const size_t need = estp_token_loss_backward_workspace_size(n_tok, d, V, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int n = int(n_tok);
  return dtype == ESTP_F32 ? launch_loss_backward<float>(X, W, targets, lse, grad, n, d, V, dtype, dX, dW, workspace, s)
                           : launch_loss_backward<__bf16>(X, W, targets, lse, grad, n, d, V, dtype, dX, dW, workspace, s);
}
