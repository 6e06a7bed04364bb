// fp32 matrix-core product tiles, shared by the calls that stream the LM head (token_loss.hip, logprobs.hip).
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
#pragma once

#include "estp_common.h"
#include "lds_ops.h"
#include "mfma_gemm.h"

namespace estp {
namespace detail {

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

}  // namespace detail
}  // namespace estp
