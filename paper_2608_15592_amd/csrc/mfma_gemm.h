// bf16 matrix-core product tiles for the LM-head gradient: C[m][n] = sum_k A(m, k) B(n, k) with fp32
// accumulation, over 256 x kBN tiles that a persistent workgroup takes one after the other.
//
// An operand lies in memory either with k contiguous (a row of A or B per m or n) or with k strided (a row per
// k, m or n contiguous).  Both reach LDS as they lie, 16-byte pieces straight from memory: a stage is 64 deep,
// [rows][64 k] of 128 bytes a row, or [64 k][rows].  The matrix-core step v_mfma_f32_16x16x32_bf16 takes 8
// consecutive k of one row per lane, which the first form gives with one 16-byte read, and the second with two
// transposing reads (ds_read_b64_tr_b16: the 16 lanes of a group read 4 x 16 elements, k-major, and each gets 4 k
// of one column).  So no operand is ever transposed in memory: dX and dW read W, X and G as they are.
//
// Waves, ring, barriers and the spacing of reads and transfers between the MFMAs are entropy_gemm_kernel's: 4
// waves of 128 x kBN / 2, one per SIMD, five 32 KB slots that hold A and B parts of the stages in turn, one barrier a
// stage, transfers issued two and a half stages ahead and across tile boundaries.  The matrix cores bound it: 256 x 256
// tiles at a depth of 4096 reach 1.25 to 1.3 PFLOP/s with what follows a tile (library products of these shapes 1.15 to
// 1.48); at a depth of 704, 11 stages, 0.8.
#pragma once

#include <type_traits>

#include "estp_common.h"
#include "lds_ops.h"

namespace estp {
namespace detail {
// Stores of 16 bytes at a byte offset of a buffer resource; past its end nothing is written.
template <int kAux = 0>
__device__ __forceinline__ void buf_store16(buf_rsrc_t r, uint32_t off, uint4 v) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{v.x, v.y, v.z, v.w}, r, off, 0, kAux);
#endif
}

template <int kAux = 0>
__device__ __forceinline__ void buf_store8(buf_rsrc_t r, uint32_t off, uint32_t lo, uint32_t hi) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{lo, hi}, r, off, 0, kAux);
#endif
}

namespace gemm {

constexpr int kWaves = 4;
constexpr int kBM = 256;
constexpr int kDepth = 64;              // k of a stage
constexpr int kSlots = 5;
constexpr int kSlotBytes = 32768;
constexpr int kNBM = 8;                 // 16-row blocks of a wave, M side

// An operand in memory: element (row, k) at base + row * ld + 2 k (k contiguous) or base + k * ld + 2 row.
struct Operand {
  const char* base;
  uint32_t ld;   // bytes
  int rows;      // live rows; past them a k-contiguous operand reads 0, a k-strided one whatever lies there
};

// x / d for uniform 32-bit numbers on the scalar unit: the product with ceil(2^32 / d) is at most one too high.
struct Divisor {
  uint32_t d, magic;
  __device__ __forceinline__ explicit Divisor(uint32_t v)
      : d(v), magic(uint32_t(__builtin_amdgcn_readfirstlane(int(v <= 1 ? 0u : (0xffffffffu / v) + 1u)))) {}
  __device__ __forceinline__ uint32_t div(uint32_t x) const {
    const uint32_t q = __umulhi(x, magic);
    const uint32_t fixed = q * d > x ? q - 1 : q;
    return d == 1 ? x : fixed;
  }
};
// Tiles of n_m x n_n, in groups of 8 columns: 32 consecutive ids, which one XCD works on at a time, cover 4 x 8
// tiles and share their operands in its L2.  No branch: it runs in the middle of the products.
struct TileAt {
  int m, n;
};
struct TileOrder {
  int n_n, full;     // full: columns in whole groups
  Divisor per, tail;  // tiles of a group; columns of the last, smaller group
  uint32_t n_group;  // tiles of one whole group
  __device__ __forceinline__ TileOrder(int n_m, int n_n_)
      : n_n(n_n_),
        full(n_n_ & ~7),
        per(uint32_t(8 * n_m)),
        tail(uint32_t(max(1, n_n_ & 7))),
        n_group(uint32_t(8 * n_m)) {}
  __device__ __forceinline__ TileAt operator()(int id) const {
    const uint32_t g = per.div(uint32_t(id)), rem = uint32_t(id) - g * n_group;
    const bool whole = int(8 * g) < full;
    const uint32_t t = tail.div(rem);
    const uint32_t m = whole ? rem >> 3 : t, c = whole ? rem & 7u : rem - t * tail.d;
    return {int(m), int(8 * g + c)};
  }
};
// A tile: its first row on either side, its depth [k0, k1), [0, 0) if it is empty, and what the caller adds.
struct Place {
  int m0, n0, k0, k1, tag;
};
// A sum where the matrix cores left it, copied to a register that the vector units read: here, and not before.  (Left to
// the compiler, all 256 sums of a lane are copied at the end of the products, and what has no room goes to memory.)  The
// first of them follows sums_ready().
__device__ __forceinline__ float read_sum(float a) {
#if defined(__HIP_DEVICE_COMPILE__)
  float v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
  return v;
#else
  return a;
#endif
}
// The last products are done: 18 wait states, which the compiler does not count for reads it cannot see.
__device__ __forceinline__ void sums_ready() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
#endif
}
// This lane's number, formed anew: what done() derives from it is not kept in registers through the products.
__device__ __forceinline__ int fresh_lane() {
  int lane = threadIdx.x & 63;
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(lane));
#endif
  return lane;
}
// Token tile and vocabulary slice of workgroup id `wg` of n_tt x n_slices, in groups of 8 token tiles: the 32 consecutive
// ids that one XCD works on at a time stream 4 slices of W past 8 tiles of tokens.  slice >= n_slices: none.
struct SliceAt {
  int tile, slice;
};
__device__ __forceinline__ SliceAt slice_of(int wg, int n_tt, int n_slices) {
  const int whole = n_tt & ~7, cols = n_tt & 7;
  if (wg < whole * n_slices) {
    const int group = wg / (8 * n_slices), r = wg - group * 8 * n_slices;
    return {8 * group + (r & 7), r >> 3};
  }
  const int r = wg - whole * n_slices;
  return cols ? SliceAt{whole + r % cols, r / cols} : SliceAt{0, n_slices};
}
// First tile id of a workgroup; it goes on in steps of the grid (a multiple of 8).
__device__ __forceinline__ int first_tile(int wg, int grid) { return (wg & 7) * (grid >> 3) + (wg >> 3); }

// kAK, kBK: k contiguous (else strided).  kPairA: block i of a wave holds rows 32 (i / 2) + 4 (i % 2) + 8 (m / 4) + m
// % 4, so that the results of a block pair in a lane are 8 consecutive m (a strided A then has 2-way bank conflicts,
// which its reads have room for). kNBN: 16-row blocks of a wave, N side.  kOdd: the depth may be an odd multiple of
// 32 (both k contiguous).  kStores: vector-memory operations that done() leaves in flight at least (it ends with so
// many stores, always): the stage after it need not wait for them.
template <bool kAK, bool kBK, bool kPairA, int kNBN, bool kOdd, int kStores, bool kStreamA = false>
struct Tiles {
  static constexpr int kBN = 32 * kNBN;
  static constexpr int kLA = 8;              // transfers of a wave per part
  static constexpr int kLB = kNBN;
  static constexpr int kReadsA = kAK ? kNBM : 2 * kNBM, kReadsB = kBK ? kNBN : 2 * kNBN;
  static constexpr int kReads = kReadsA + kReadsB;
  static constexpr int kMfma = kNBM * kNBN;
  static constexpr int kReadEvery = kMfma / kReads;
  static constexpr int kDmaEvery = kMfma / (kLA + kLB);
  static_assert(kReadEvery >= 1 && kDmaEvery >= 1, "reads and transfers fit behind the products of a step");

  // chunk (16 bytes) swizzles: 16 rows a k-contiguous read touches, or 8 k-rows a transposing one does, lie in
  // distinct banks
  __device__ static __forceinline__ int swz_k(bool pair, int row) {
    return pair ? ((row >> 1) & 1) | ((row >> 2) & 6) : (row >> 1) & 7;
  }
  __device__ static __forceinline__ int swz_s(int k) { return 2 * ((k & 3) | ((k >> 1) & 4)); }

  // byte offset in a part's source of what lane `lane` of transfer i brings, and its 16-byte chunk along k
  template <bool kK, bool kPair, int kRows>
  __device__ static __forceinline__ uint32_t source(int i, int wave, int lane, uint32_t ld, int* chunk_k) {
    if (kK) {
      const int row = 8 * (kWaves * i + wave) + lane / 8, c = (lane % 8) ^ swz_k(kPair, row);
      *chunk_k = c;
      return uint32_t(row) * ld + uint32_t(c) * 16u;
    }
    constexpr int kChunks = kRows / 8;  // of a k-row
    const int at = 64 * (kWaves * i + wave) + lane, k = at / kChunks, c = (at % kChunks) ^ swz_s(k);
    return uint32_t(k) * ld + uint32_t(c) * 16u;
  }

  struct Frags {
    bf16x8_t a[kNBM], b[kNBN];
  };

  // Runs tile ids first, first + step, ... < total: at(id) places a tile, done(place, acc) takes its products
  // (acc[i][j][r]: row 16 i + 4 (lane / 16) + r of the wave's 128 rows, or as kPairA says; column
  // 16 j + lane % 16 of its kBN / 2 columns).
  template <typename At, typename Done>
  __device__ static __forceinline__ void run(char* lds, const Operand& A, const Operand& B, int first, int step,
                                             int total, At&& at, Done&& done) {
    if (first >= total) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;

    uint32_t off_a[kLA], off_b[kLB];
    int kc_a[kLA], kc_b[kLB];
#pragma unroll
    for (int i = 0; i < kLA; ++i) off_a[i] = source<kAK, kPairA, kBM>(i, wave, lane, A.ld, &kc_a[i]);
#pragma unroll
    for (int i = 0; i < kLB; ++i) off_b[i] = source<kBK, false, kBN>(i, wave, lane, B.ld, &kc_b[i]);

    // ---- prefetch: parts A, B of the stages in order; past the last tile an empty resource (no access).  pf is the
    // stage the next parts belong to, nx the tile after pf's: selects between the two keep the loop body one block,
    // nx is formed anew, with a branch, at the top of a stage.
    const Place none{0, 0, 0, 0, 0};
    int nx_id = first + step, pf_slot = 0;
    Place pf = at(first), nx = nx_id < total ? at(nx_id) : none;
    bool nx_used = false;
    struct Part {
      u32x4_t rsrc;
      uint32_t soff;
      char* dst;
      int depth;  // k the stage holds (kOdd)
    };
    auto place = [&](const Operand& o, bool contig, int r0, int rows) {
      Part p;
      p.dst = lds + pf_slot * kSlotBytes + 1024 * wave;
      pf_slot = pf_slot + 1 == kSlots ? 0 : pf_slot + 1;
      const int left = pf.k1 - pf.k0;  // never negative
      p.depth = left;
      if (contig) {
        const uint32_t bytes = uint32_t(min(rows, o.rows - r0)) * o.ld;
        p.rsrc = rsrc_words(o.base + size_t(r0) * o.ld, left > 0 ? bytes : 0u);
        p.soff = uint32_t(pf.k0) * 2u;
      } else {
        const uint32_t bytes = uint32_t(min(kDepth, left)) * o.ld - uint32_t(r0) * 2u;
        p.rsrc = rsrc_words(o.base + size_t(pf.k0) * o.ld + size_t(r0) * 2, left > 0 ? bytes : 0u);
        p.soff = 0;
      }
      return p;
    };
    auto next_a = [&]() { return place(A, kAK, pf.m0, kBM); };
    auto next_b = [&]() {
      const Part p = place(B, kBK, pf.n0, kBN);
      // (as masks that the compiler cannot see through: it would make a branch of four selects, and spill around it)
      const int wrap = __builtin_amdgcn_readfirstlane(-int(pf.k0 + kDepth >= pf.k1));
      pf.k0 += (kDepth & ~wrap) + ((nx.k0 - pf.k0) & wrap);
      pf.k1 += (nx.k1 - pf.k1) & wrap;
      pf.m0 += (nx.m0 - pf.m0) & wrap;
      pf.n0 += (nx.n0 - pf.n0) & wrap;
      nx_used = wrap != 0;
      return p;
    };
    auto refill = [&]() {
      if (nx_used) {
        nx_id += step;
        nx = nx_id < total ? at(nx_id) : none;
        nx_used = false;
      }
    };
    auto dma_a = [&](const Part& p, int i) {
      const uint32_t o = kOdd && kAK && 8 * kc_a[i] >= p.depth ? kPastEnd : off_a[i];
      dma16<kStreamA>(p.rsrc, o, p.soff, p.dst + 1024 * kWaves * i);
    };
    auto dma_b = [&](const Part& p, int i) {
      const uint32_t o = kOdd && kBK && 8 * kc_b[i] >= p.depth ? kPastEnd : off_b[i];
      dma16(p.rsrc, o, p.soff, p.dst + 1024 * kWaves * i);
    };

    // ---- fragment reads of the 32-deep step u of a stage
    const int fr = lane & 15, fq = lane >> 4;
    uint32_t ra[2], rb[2];  // k contiguous: offset of block 0 for each step; k strided: [0] for both
    {
      const int row = 128 * wm + (kPairA ? 8 * (fr >> 2) + (fr & 3) : fr);
      const int k = 8 * fq + (fr >> 2), g = swz_s(k) >> 1;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        ra[u] = kAK ? row * 128 + ((4 * u + fq) ^ swz_k(kPairA, row)) * 16
                    : kPairA ? k * (2 * kBM) + ((8 * wm + ((fr >> 1) & 1)) ^ g) * 32 + (fr & 1) * 16
                             : k * (2 * kBM) + ((8 * wm) ^ g) * 32 + (fr & 3) * 8;
      const int rowb = 16 * kNBN * wn + fr;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        rb[u] = kBK ? rowb * 128 + ((4 * u + fq) ^ swz_k(false, rowb)) * 16
                    : k * (2 * kBN) + ((kNBN * wn) ^ g) * 32 + (fr & 3) * 8;
    }
    s16x4_t half[2];  // first half of a transposed fragment until the second is read
    auto read = [&](Frags& f, int slot_a, int slot_b, int u, int q) {
      if (q < kReadsA) {
        const char* s = lds + slot_a * kSlotBytes;
        if (kAK) {
          f.a[q] = *reinterpret_cast<const bf16x8_t*>(s + ra[u] +
                                                      (kPairA ? 4096 * (q / 2) + 512 * (q % 2) : 2048 * q));
        } else {
          const int i = q / 2;  // block
          const char* p = s + (kPairA ? (ra[0] ^ (uint32_t(i / 2) << 6)) + 8 * (i % 2) : ra[0] ^ (uint32_t(i) << 5)) +
                          (32 * u + 4 * (q % 2)) * (2 * kBM);
          if (q % 2 == 0)
            half[0] = read_tr(p);
          else
            f.a[q / 2] = join_tr(half[0], read_tr(p));
        }
      } else {
        q -= kReadsA;
        const char* s = lds + slot_b * kSlotBytes;
        if (kBK) {
          f.b[q] = *reinterpret_cast<const bf16x8_t*>(s + rb[u] + 2048 * q);
        } else {
          const char* p = s + (rb[0] ^ (uint32_t(q / 2) << 5)) + (32 * u + 4 * (q % 2)) * (2 * kBN);
          if (q % 2 == 0)
            half[1] = read_tr(p);
          else
            f.b[q / 2] = join_tr(half[1], read_tr(p));
        }
      }
    };

    // ---- prologue: A0 B0 A1 B1 A2 in flight, stage 0 landed
    {
      Part p = next_a();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < kLA; ++i) dma_a(p, i);
        p = next_b();
#pragma unroll
        for (int i = 0; i < kLB; ++i) dma_b(p, i);
        refill();
        p = next_a();
      }
#pragma unroll
      for (int i = 0; i < kLA; ++i) dma_a(p, i);
    }
    wait_vm<2 * kLA + kLB>();
    lds_barrier();
    Frags f[2];
#pragma unroll
    for (int q = 0; q < kReads; ++q) read(f[0], 0, 1, 0, q);
    int sa = 0;  // slot of the current stage's A part; B in the next one

    for (int id = first; id < total; id += step) {
      const Place p = at(id);
      f32x4_t acc[kNBM][kNBN];
#pragma unroll
      for (int i = 0; i < kNBM; ++i)
#pragma unroll
        for (int j = 0; j < kNBN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      // at least one stage, also of an empty depth.  The compiler must not know that: of a loop that surely runs it
      // keeps the sums in other registers than the products' own, and spills (145 registers of the dW kernel; 10 so).
      const int nk = __builtin_amdgcn_readfirstlane(max(1, (p.k1 - p.k0 + kDepth - 1) / kDepth));
      auto stage = [&](auto behind) {  // behind: operations issued after the next stage's parts that may stay in flight
        const int sb = sa + 1 == kSlots ? 0 : sa + 1;
        const int sa_next = sb + 1 == kSlots ? 0 : sb + 1;
        const int sb_next = sa_next + 1 == kSlots ? 0 : sa_next + 1;
        refill();
        Part pb, pa;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Frags& cur = f[u];
          Frags& nxt = f[u ^ 1];
          if (u == 1) {
            // this wave's reads of the stage are done, and the next stage has landed (only its successor's A
            // part may be in flight): after the barrier nobody reads this stage's slots again
            __builtin_amdgcn_sched_barrier(0);
            wait_vm<decltype(behind)::value>();
            lds_barrier();
          }
#pragma unroll
          for (int i = 0; i < kNBM; ++i)
#pragma unroll
            for (int j = 0; j < kNBN; ++j) {
              const int m = i * kNBN + j;
              acc[i][j] = mfma_bf16(cur.a[i], cur.b[j], acc[i][j]);
              if (u == 0 && m == kMfma / 8) pb = next_b();
              if (u == 0 && m == kMfma / 2) pa = next_a();
              if (m % kReadEvery == 0 && m / kReadEvery < kReads) {
                if (u == 1)
                  read(nxt, sa_next, sb_next, 0, m / kReadEvery);
                else
                  read(nxt, sa, sb, 1, m / kReadEvery);
              }
              if (u == 1 && m % kDmaEvery == kDmaEvery - 1 && m / kDmaEvery < kLA + kLB) {
                const int t = m / kDmaEvery;
                if (t < kLB)
                  dma_b(pb, t);
                else
                  dma_a(pa, t - kLB);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
        }
        sa = sa_next;
      };
      // (the first stage of a tile leaves the last tile's stores behind as well)
      if (id == first)
        stage(std::integral_constant<int, kLA>{});
      else
        stage(std::integral_constant<int, kLA + kStores>{});
      for (int ks = 1; ks < nk; ++ks) stage(std::integral_constant<int, kLA>{});
      done(p, acc);
      // the next tile's first fragments, again: done() has the registers to itself
      const int sb = sa + 1 == kSlots ? 0 : sa + 1;
#pragma unroll
      for (int q = 0; q < kReads; ++q) read(f[0], sa, sb, 0, q);
    }
    wait_vm<0>();  // no transfer into LDS outlives the workgroup
  }
};

}  // namespace gemm
}  // namespace detail
}  // namespace estp
