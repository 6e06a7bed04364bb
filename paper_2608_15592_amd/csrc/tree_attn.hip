// Attention of drafted tokens over a cache, and the weight each cached token
// receives from it.
//
// Sequence b holds lens[b] cached tokens in slots [0, lens[b]) of its KV heads
// and T = cu_q[b + 1] - cu_q[b] <= 64 drafted ones in the slots after them.
// Drafted row t sees every cached slot and the drafted slots whose bit its mask
// has.  Query head h reads KV head h / G, G = Hq / Hkv, so the T G rows of a KV
// head share its keys and are handled together: row r is token r / G, head
// r % G of the group.
//
//   s_rj = scale q_r . k_j,  lse_r = log sum_j exp s_rj,  O_r = sum_j exp(s_rj - lse_r) v_j
//   acc_j += sum_r w_r exp(s_rj - lse_r)
//
// A row that sees nothing has lse -inf and O 0, and adds nothing.
//
// An item is one (sequence, KV head) and up to 16, 32 or 64 rows of it; its keys come in chunks.  All chunks of all
// items form one line, cut into equal shares, one for each workgroup of a grid that fills the chip once: lengths may
// differ as they like, and no workgroup is empty.  A share's piece of an item is a segment, worked off in one pass with
// the running maximum and sum of the softmax (base 2); tree_join joins an item's segments.  The account takes the rows'
// normalisers, so it comes last: from scores that the first kernel kept where the rows are few (in the launch of the
// join), else from scores formed again.  No atomics: bitwise reproducible.
//
// The cache is read once; that bounds calls of few rows (4.4 to 4.9 TB/s by the counters; a copy moves 4.9 on this card).
// Calls of many rows spend their time on the exponentials and what goes with them, each score twice (256 rows of 64, 8
// sequences of 8000, bf16: vector instructions in flight 55 % of the attention's cycles, matrix ones 28 %).
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <vector>

#include "estp_common.h"
#include "lds_ops.h"

namespace estp {
namespace detail {

constexpr int kMaxTree = 64;  // drafted tokens of a sequence: the bits of a mask
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

struct TreeShape {
  int B, max_q, n_q, Hq, Hkv, cap, max_kv;
  int item_shift, items;  // 2^item_shift rows of an item; items of a (sequence, KV head) at most
  int G;                  // Hq / Hkv, at most 32768
  uint32_t over_G;        // ceil(2^31 / G)
  __device__ __forceinline__ int item_rows() const { return 1 << item_shift; }
  __device__ __forceinline__ int most_rows() const { return max_q * G; }  // of a (sequence, KV head)
  // r / G for a row number (below 65536): r (G over_G - 2^31) stays below 2^31
  __device__ __forceinline__ int token(int r) const { return int(__umulhi(uint32_t(2 * r), over_G)); }
};
inline TreeShape tree_shape(int B, int max_q, int64_t n_q, int Hq, int Hkv, int64_t cap, int max_kv, int item_shift,
                            int items) {
  const int G = Hq / Hkv;
  return {B, max_q, int(n_q), Hq, Hkv, int(cap), max_kv, item_shift, items, G,
          uint32_t(((uint64_t(1) << 31) + uint64_t(G) - 1) / uint64_t(G))};
}

// One sequence as the kernels see it: counts out of range (invalid input) never become an access out of range.
struct TreeSeq {
  int q0, T, len, keys;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeShape& sh, const int* lens, const int* cu_q, int b) {
  TreeSeq q;
  q.q0 = max(0, min(cu_q[b], sh.n_q));
  q.T = max(0, min(max(0, min(cu_q[b + 1], sh.n_q)) - q.q0, sh.max_q));
  q.len = max(0, min(lens[b], sh.max_kv));
  q.keys = min(q.len + q.T, sh.max_kv);
  return q;
}
// The mask of drafted token t (row q0 + t); without masks a chain: every drafted token up to its own.
__device__ __forceinline__ uint64_t tree_bits(const int64_t* mask, int q0, int t) {
  return mask ? uint64_t(mask[q0 + t]) : (uint64_t(2) << t) - 1;
}
// Whether a row with mask `bits` sees the key `rel` places past the cached ones.
__device__ __forceinline__ bool tree_sees(uint64_t bits, int rel) {
  return rel < 0 || (rel < kMaxTree && ((bits >> (rel & 63)) & 1));
}

// ------------------------------------------------------------------ the line of chunks

// How the line is cut: chunks of kChunk keys; kStart units that an item counts for besides its chunks, so that a share
// in which one starts, which begins a segment more, has less to do; shares of a multiple of kRound units.  (Attention,
// kStart 4 against none: 8 sequences of 4096, 64 rows of 128 40.2 and 43.0 us; 26 others 13 % less to 2 % more.  Account,
// 8 against none: one sequence of 16000, 256 rows of 128 25 and 35 us; 9 others 12 % less to 14 % more.)
template <int kChunk_, int kStart_, int kRound_>
struct TreeCut {
  static constexpr int kChunk = kChunk_, kStart = kStart_, kRound = kRound_;
};
// 64 sequences, one a lane: counts, and how many units their items have in all.
template <typename Cut>
struct TreeBatch {
  int b0, q0, T, len, keys;
  uint32_t w, upto;  // chunks of the lane's sequence; of the batch's up to and with it
  __device__ __forceinline__ void fetch(const TreeShape& sh, const int* lens, const int* cu_q, int first) {
    b0 = first;
    const int b = first + int(threadIdx.x & 63);
    TreeSeq q{0, 0, 0, 0};
    if (b < sh.B) q = tree_seq(sh, lens, cu_q, b);
    q0 = q.q0;
    T = q.T;
    len = q.len;
    keys = q.keys;
    w = uint32_t(sh.Hkv) * items(sh, q.T) * units(q.keys);
    upto = wave_prefix(w);
  }
  __device__ static __forceinline__ uint32_t items(const TreeShape& sh, int T) {  // of a KV head
    return uint32_t(T * sh.G + sh.item_rows() - 1) >> sh.item_shift;
  }
  __device__ static __forceinline__ uint32_t units(int keys) {
    return keys > 0 ? uint32_t(keys + Cut::kChunk - 1) / Cut::kChunk + Cut::kStart : 0;
  }
  __device__ __forceinline__ uint32_t all() const { return lane_of(upto, 63); }
};
// Chunks of one share: at least 128 keys, so that joins stay few.
template <typename Cut>
__device__ __forceinline__ uint32_t tree_share(uint32_t total, int wgs) {
  const uint32_t share = max(uint32_t(128 / Cut::kChunk), (total + uint32_t(wgs) - 1) / uint32_t(wgs));
  return (share + Cut::kRound - 1) / Cut::kRound * Cut::kRound;
}
template <typename Cut>
__device__ __forceinline__ uint32_t tree_total(const TreeShape& sh, const int* lens, const int* cu_q,
                                               TreeBatch<Cut>& first) {
  first.fetch(sh, lens, cu_q, 0);
  uint32_t total = first.all();
  for (int b0 = 64; b0 < sh.B; b0 += 64) {
    TreeBatch<Cut> t;
    t.fetch(sh, lens, cu_q, b0);
    total += t.all();
  }
  return total;
}
// A segment: rows r0 .. of KV head g of sequence b, keys [k0, k1), its partial result's place.
struct TreeSegment {
  int b, g, r0, q0, T, len, keys, k0, k1, slot;
};
// The mask of drafted token t of the segment's sequence, without the bits of tokens that the sequence has not.
__device__ __forceinline__ uint64_t tree_bits(const int64_t* mask, const TreeSegment& q, int t) {
  const int n = q.keys - q.len;
  return tree_bits(mask, q.q0, t) & (n >= 64 ? ~uint64_t(0) : (uint64_t(1) << n) - 1);
}
// Which of the four keys from `rel` places past the cached ones on a row with such a mask sees: a bit each.
__device__ __forceinline__ uint32_t tree_sees4(uint64_t bits, int rel) {
  const uint64_t drafted = rel < 64 ? bits >> (rel & 63) : 0, both = ~(~bits << (-rel & 63));
  return uint32_t(rel >= 0 ? drafted : rel > -4 ? both : ~uint64_t(0)) & 15u;
}
// Calls f with the segments of this workgroup's share, a multiple of kRound chunks, in turn; all values are uniform.
// Neighbouring shares, whose items have keys in common, go to one XCD, and all XCDs (every 8th workgroup of the grid, a
// multiple of 8) get as many of the shares there are: with shares rounded up there can be far fewer than workgroups.
template <typename Cut, typename F>
__device__ __forceinline__ void tree_walk(const TreeShape& sh, const int* lens, const int* cu_q, F&& f) {
  TreeBatch<Cut> t;
  const uint32_t total = tree_total<Cut>(sh, lens, cu_q, t), share = tree_share<Cut>(total, gridDim.x);
  const uint32_t shares = (total + share - 1) / share, of_xcd = (shares + 7) / 8;
  const int wg = int((blockIdx.x & 7) * of_xcd + (blockIdx.x >> 3));
  if ((blockIdx.x >> 3) >= of_xcd || uint32_t(wg) >= shares) return;
  uint32_t at = uint32_t(wg) * share;
  const uint32_t end = min(total, at + share);
  uint32_t off = 0;  // of the batch, then of the sequence
  while (off + t.all() <= at) {
    off += t.all();
    t.fetch(sh, lens, cu_q, t.b0 + 64);
  }
  int j = __builtin_ctzll(__ballot(off + t.upto > at));
  off += lane_of(t.upto, j) - lane_of(t.w, j);
  while (true) {
    TreeSegment s;
    s.b = t.b0 + j;
    s.q0 = int(lane_of(uint32_t(t.q0), j));
    s.T = int(lane_of(uint32_t(t.T), j));
    s.len = int(lane_of(uint32_t(t.len), j));
    s.keys = int(lane_of(uint32_t(t.keys), j));
    const uint32_t n = TreeBatch<Cut>::units(s.keys), items = TreeBatch<Cut>::items(sh, s.T);
    const uint32_t item = (at - off) / n, c0 = at - off - item * n, c1 = min(n, c0 + (end - at));
    s.g = __builtin_amdgcn_readfirstlane(int(item / items));
    const int part = __builtin_amdgcn_readfirstlane(int(item % items));
    s.r0 = part << sh.item_shift;
    s.k0 = __builtin_amdgcn_readfirstlane(max(0, int(c0) - Cut::kStart) * Cut::kChunk);
    s.k1 = __builtin_amdgcn_readfirstlane(min(s.keys, max(0, int(c1) - Cut::kStart) * Cut::kChunk));
    s.slot = wg + (s.b * sh.Hkv + s.g) * sh.items + part;  // grows from segment to segment
    if (Cut::kStart == 0 || s.k0 < s.k1) f(s);
    at += c1 - c0;
    if (at >= end) return;
    if (at - off >= lane_of(t.w, j)) {
      off += lane_of(t.w, j);
      do {
        if (++j == 64) {
          t.fetch(sh, lens, cu_q, t.b0 + 64);
          j = 0;
        }
      } while (lane_of(t.w, j) == 0);
    }
  }
}

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) {
  *p = __builtin_bit_cast(uint16_t, __bf16(v));  // round to nearest even
}

// What differs between the types.  16 bytes of a row, a fragment, are 8 bf16 or 4 fp32 values; a 16-key block's scores
// of 16 rows take one v_mfma_f32_16x16x32_bf16 for every 64 bytes of a row, or four v_mfma_f32_16x16x4_f32 (its k:
// value j of the four lanes' fragments, the same in both operands).  Chunks of keys are equally large in bytes.
template <typename T>
struct TreeMath;
template <>
struct TreeMath<uint16_t> {
  typedef bf16x8_t Frag;
  static constexpr int kC = 32;  // keys of a chunk
  __device__ static __forceinline__ f32x4_t scores(const Frag& k, const Frag& q, const f32x4_t& s) {
    return mfma_bf16(k, q, s);
  }
};
template <>
struct TreeMath<float> {
  typedef f32x4_t Frag;
  static constexpr int kC = 16;
  __device__ static __forceinline__ f32x4_t scores(const Frag& k, const Frag& q, f32x4_t s) {
#pragma unroll
    for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j], q[j], s, 0, 0, 0);
    return s;
  }
};

template <typename T>
using AttnCut = TreeCut<TreeMath<T>::kC, 4, 1>;

// Items of 16 rows a wave, chunks of 32 keys (fp32: 16).
//
// S^T = K Q^T: a lane holds one row (column lane % 16 of the products) and, of each of the chunk's 16-key blocks, keys
// 4 fq .. 4 fq + 3 (fq = lane / 16).  These weights are at once the lane's part of the second product's operand,
// O^T = V^T P^T, if V's part holds the same keys for one of its columns: two transposing reads for 32 keys of bf16; for
// fp32, where a product takes one key of each fq, 16-byte reads along a row of V, the lane's columns then being
// neighbours.  So scores never leave the registers.  The reference of a row's exponentials follows its maximum only
// when a score passes it by 2^16 (sums and weights stay far from overflow): most chunks neither exchange maxima
// between lanes nor rescale O.
//
// The chunks' K and V parts go straight from memory into a ring of five parts.  Up to 16 rows: one wave that uses the
// ring alone, without barriers, and counts its own transfers, two and a half chunks ahead; memory bounds it.  More
// rows: kW waves of 16 rows each share the ring, so that the keys are fetched once for all of them, and there are more
// waves on a compute unit to hide one another's waits.  16-byte pieces are swizzled so that the 16 rows of a K read
// and the 8 of a transposing V read lie in distinct banks.
//
// Measured: one row of 32 heads on 8 KV heads of 128, one sequence of 32767: 26.2 us, 5.1 TB/s; 32 sequences of 500 to
// 4000: 52 us, 4.4 TB/s.  31 drafted tokens, 4 heads of 64 on a KV head, 8 sequences of 900 to 8100: 25.8 us, of which
// 5 us pass before the first chunk and after the last; its exponentials alone are 4 us of the chip's.  fp32, the first
// of these: 46 us, 5.8 TB/s; 31 drafted tokens at 8 sequences of 4500: 95 us, bf16 27.
template <typename T, int DH, int kW, bool kScores>
__global__ __launch_bounds__(64 * kW, 2) void tree_attn_kernel(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
    const int* __restrict__ lens, const int* __restrict__ cu_q, const int64_t* __restrict__ mask, TreeShape sh,
    float c2, float* __restrict__ scores, int pitch, float* __restrict__ part_m, float* __restrict__ part_l,
    float* __restrict__ part_o) {
  using Math = TreeMath<T>;
  using Frag = typename Math::Frag;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kC = Math::kC, kB = kC / 16, kRow = DH * int(sizeof(T)), kPart = kC * kRow, kSlots = 5;
  constexpr int kL = kPart / 1024, kLw = kL / kW;  // transfers for a part; of a wave
  constexpr int kPieces = kRow / 16, kNF = kPieces / 4, kND = DH / 16;
  constexpr int kWindow = kPieces >= 16 ? 1 : 16 / kPieces;  // rows in 256 bytes
  constexpr int kVW = kND < 4 ? kND : 4;                     // fp32: neighbouring columns of a lane
  typedef float cols_t __attribute__((ext_vector_type(kVW)));
  static_assert(kL % kW == 0, "waves share a part's transfers equally");
  // The ring, and 16 rows of Q for each of several waves: tree_lds(DH, kW, sizeof(T)) bytes.  (Dynamic: of a size it
  // knows, the compiler takes one wave a SIMD for granted at a head size of 128, and copies sums between two register
  // files.)
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, fr = lane & 15, fq = lane >> 4, G = sh.G;
  const int wave = kW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t off_k[kLw], off_v[kLw];
#pragma unroll
  for (int i = 0; i < kLw; ++i) {
    const int piece = 64 * (kW * i + wave) + lane, row = piece / kPieces, c = piece % kPieces;
    off_k[i] = uint32_t(row * kRow + (c ^ (row / kWindow & (kPieces - 1))) * 16);
    off_v[i] = uint32_t(row * kRow + (kBf16 ? c ^ (2 * (row / kWindow & (kPieces / 2 - 1))) : c) * 16);
  }
  auto read_k = [&](const char* part, int row, int c) {  // fragment 4 c + fq of a row of a K part
    return *reinterpret_cast<const Frag*>(part + row * kRow + ((4 * c + fq) ^ (row / kWindow & (kPieces - 1))) * 16);
  };
  // column of O in o[d][z]
  auto column = [&](int d, int z) {
    return kBf16 ? 16 * d + 4 * fq + z : 16 * kVW * (d / kVW) + kVW * (4 * fq + z) + d % kVW;
  };
  auto unit_of = [](int row) { return row / kWindow & (kPieces / 2 - 1); };  // swizzle of a V part, in 32 bytes
  tree_walk<AttnCut<T>>(sh, lens, cu_q, [&](const TreeSegment& q) {
    const int bg = q.b * sh.Hkv + q.g, r0 = q.r0 + 16 * wave, R = q.T * G, r = r0 + fr;
    const char* Kb = reinterpret_cast<const char*>(K) + size_t(bg) * sh.cap * kRow;
    const char* Vb = reinterpret_cast<const char*>(V) + size_t(bg) * sh.cap * kRow;
    int pf_key = q.k0, pf_slot = 0;
    auto issue = [&](const char* base, const uint32_t (&off)[kLw]) {  // past the range: an empty resource, no access
      const int left = min(kC, q.keys - pf_key);
      const u32x4_t rsrc = rsrc_words(base + size_t(pf_key) * kRow, pf_key < q.k1 ? uint32_t(left) * kRow : 0u);
#pragma unroll
      for (int i = 0; i < kLw; ++i) dma16(rsrc, off[i], 0, lds + pf_slot * kPart + 1024 * (kW * i + wave));
      pf_slot = pf_slot + 1 == kSlots ? 0 : pf_slot + 1;
    };
    const uint64_t bits = r < R ? tree_bits(mask, q, sh.token(r)) : 0;
    if (kW > 1) lds_barrier();  // every wave's reads of the last segment are done
    // the wave's rows of Q come first, laid out as a K part, through the ring's last slot or places of their own: a
    // load into registers would wait for every transfer issued around it
    char* const own = lds + (kW == 1 ? (kSlots - 1) * kPart : kSlots * kPart + wave * (16 * kRow));
    const u32x4_t rq = rsrc_words(reinterpret_cast<const char*>(Q) + size_t(q.q0) * sh.Hq * kRow,
                                  uint32_t(q.T) * uint32_t(sh.Hq) * uint32_t(kRow));
#pragma unroll
    for (int i = 0; i < kRow / 64; ++i) {
      const int at = (64 * i + lane) / kPieces, row = r0 + at;
      const uint32_t piece = uint32_t((64 * i + lane) % kPieces ^ (at / kWindow & (kPieces - 1))) * 16u;
      const uint32_t tok = uint32_t(sh.token(row)), head = uint32_t(q.g * G + row) - tok * uint32_t(G);
      dma16(rq, row < R ? (tok * uint32_t(sh.Hq) + head) * kRow + piece : kPastEnd, 0, own + 1024 * i);
    }
    issue(Kb, off_k);
    issue(Vb, off_v);
    pf_key += kC;
    issue(Kb, off_k);
    issue(Vb, off_v);
    pf_key += kC;
    arrived<4 * kLw>();
    Frag qf[kNF];
#pragma unroll
    for (int c = 0; c < kNF; ++c) qf[c] = read_k(own, fr, c);
    lds_read_done();
    if (kW == 1) issue(Kb, off_k);
    float m = -INFINITY, l = 0.f;
    f32x4_t o[kND];
#pragma unroll
    for (int d = 0; d < kND; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int slot = 0;
    // A part may be read when it has landed, its slot be filled again when it is read.  One wave: four parts stay in
    // flight, the fifth follows the read.  Several: a barrier says that every wave's transfers of the part have landed
    // and that every wave has read the part before it, whose slot the next transfers take.
    auto part_landed = [&]() {
      arrived<(kW == 1 ? 4 : 3) * kLw>();
      if (kW > 1) lds_barrier();
    };
    for (int k = q.k0; k < q.k1; k += kC) {
      const bool edge = k + kC > q.len;  // holds drafted tokens, or ends the sequence
      // ---- scores
      part_landed();
      if (kW > 1) issue(Kb, off_k);
      Frag kf[kB][kNF];
#pragma unroll
      for (int a = 0; a < kB; ++a)
#pragma unroll
        for (int c = 0; c < kNF; ++c) kf[a][c] = read_k(lds + slot * kPart, 16 * a + fr, c);
      lds_read_done();
      if (kW == 1) {
        issue(Vb, off_v);
        pf_key += kC;
      }
      slot = slot + 1 == kSlots ? 0 : slot + 1;
      f32x4_t s[kB];
#pragma unroll
      for (int a = 0; a < kB; ++a) {
        s[a] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kNF; ++c) s[a] = Math::scores(kf[a][c], qf[c], s[a]);
      }
      if (edge) {
#pragma unroll
        for (int a = 0; a < kB; ++a) {
          const uint32_t sees = tree_sees4(bits, k + 16 * a + 4 * fq - q.len);
#pragma unroll
          for (int z = 0; z < 4; ++z) s[a][z] = (sees >> z) & 1 ? s[a][z] : -INFINITY;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4 * kB; ++e) mx = fmaxf(mx, s[e / 4][e % 4]);
      mx *= c2;
      if (kScores && r < R) {
        float* w = scores + (size_t(bg) * sh.most_rows() + fr) * pitch + k + 4 * fq;
#pragma unroll
        for (int a = 0; a < kB; ++a) *reinterpret_cast<f32x4_t*>(w + 16 * a) = s[a] * c2;
      }
      if (__any(mx > m + 16.f)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        mx = fmaxf(mx, m);
        const float f = fast_exp2(m - (mx == -INFINITY ? 0.f : mx));
        m = mx;
        l *= f;
#pragma unroll
        for (int d = 0; d < kND; ++d) o[d] *= f;
      }
      const float ref = m == -INFINITY ? 0.f : m;  // nothing seen yet: all weights are 0
      // For bf16 the matrix cores take the weights as two numbers, the second what the rounding of the first leaves:
      // O is rounded once, where it is written (with the first alone its error is 1.4 times that, at the same speed
      // where memory bounds it).
      float p[4 * kB];
      u32x4_t pf, pf_lo;
#pragma unroll
      for (int e = 0; e < 4 * kB; ++e) {
        p[e] = fast_exp2(fmaf(s[e / 4][e % 4], c2, -ref));
        l += p[e];
      }
      if constexpr (kBf16)
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // two at a time
          pf[e] = pack_bf16(p[2 * e], p[2 * e + 1]);
          pf_lo[e] = pack_bf16(p[2 * e] - __uint_as_float(pf[e] << 16),
                               p[2 * e + 1] - __uint_as_float(pf[e] & 0xffff0000u));
        }
      // ---- output
      part_landed();
      if (kW > 1) {
        issue(Vb, off_v);
        pf_key += kC;
      }
      const char* vs = lds + slot * kPart;
      bf16x8_t vf[kBf16 ? kND : 1];
      cols_t vc[kBf16 ? 1 : 4][kBf16 ? 1 : kND / kVW];  // fp32: of keys 4 fq + i
      if constexpr (kBf16) {
#pragma unroll
        for (int d = 0; d < kND; ++d) {
          const int row = 4 * fq + (fr >> 2);  // and 16 further on: the swizzle is the same
          const char* w = vs + row * kRow + (d ^ unit_of(row)) * 32 + (fr & 3) * 8;
          vf[d] = join_tr(read_tr(w), read_tr(w + 16 * kRow));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int u = 0; u < kND / kVW; ++u)
            vc[i][u] = *reinterpret_cast<const cols_t*>(vs + (4 * fq + i) * kRow + (16 * u + fr) * (4 * kVW));
      }
      lds_read_done();
      if (edge) {
        // A drafted token that a row does not see has weight 0 there, which a non-finite value must not meet: such
        // values leave the product and are added, one by one, to the rows that see them.
        bool bad = false;
        if constexpr (kBf16) {
          u16x2_t top{0, 0};  // the largest exponent
#pragma unroll
          for (int d = 0; d < kND; ++d) {
            const u32x4_t v = __builtin_bit_cast(u32x4_t, vf[d]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, v[e] & 0x7f807f80u));
          }
          bad = top[0] == 0x7f80 || top[1] == 0x7f80;
        } else {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < kND; ++d)
              top = max(top, __float_as_uint(vc[i][d / kVW][d % kVW]) & 0x7f800000u);
          bad = top == 0x7f800000u;
        }
        if (__any(bad)) {
          if constexpr (kBf16) {
#pragma unroll
            for (int d = 0; d < kND; ++d) {
              s16x8_t v = __builtin_bit_cast(s16x8_t, vf[d]);
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = (v[e] & 0x7f80) == 0x7f80 ? short(0) : v[e];
              vf[d] = __builtin_bit_cast(bf16x8_t, v);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int d = 0; d < kND; ++d) {
                const float v = vc[i][d / kVW][d % kVW];
                vc[i][d / kVW][d % kVW] = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? 0.f : v;
              }
          }
          for (int j = 0; j < kC && k + j < q.keys; ++j) {
            const int from = fr + 16 * (j % 16 / 4), e = j / 16 * 4 + j % 4;
            float mine = 0.f;
#pragma unroll
            for (int z = 0; z < 4 * kB; ++z) mine = z == e ? p[z] : mine;
            const float w = __shfl(mine, from, 64);
            if (!tree_sees(bits, k + j - q.len)) continue;
#pragma unroll
            for (int d = 0; d < kND; ++d)
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                const int at = column(d, z);
                if constexpr (kBf16) {
                  const uint16_t v = *reinterpret_cast<const uint16_t*>(
                      vs + j * kRow + ((at / 16) ^ unit_of(j)) * 32 + (at % 16) * 2);
                  if ((v & 0x7f80) == 0x7f80) o[d][z] += w * bf16_to_f32(v);
                } else {
                  const float v = *reinterpret_cast<const float*>(vs + j * kRow + at * 4);
                  if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[d][z] += w * v;
                }
              }
          }
          lds_read_done();
        }
      }
      if (kW == 1) issue(Kb, off_k);
      slot = slot + 1 == kSlots ? 0 : slot + 1;
      if constexpr (kBf16) {
#pragma unroll
        for (int d = 0; d < kND; ++d) o[d] = mfma_bf16(vf[d], __builtin_bit_cast(bf16x8_t, pf), o[d]);
#pragma unroll
        for (int d = 0; d < kND; ++d) o[d] = mfma_bf16(vf[d], __builtin_bit_cast(bf16x8_t, pf_lo), o[d]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int d = 0; d < kND; ++d)
            o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vc[i][d / kVW][d % kVW], p[i], o[d], 0, 0, 0);
      }
    }
    arrived<0>();  // no transfer into LDS outlives the segment
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (r >= R) return;
    const size_t row = size_t(q.slot) * (16 * kW) + 16 * wave + fr;
    if (fq == 0) {
      part_m[row] = m;
      part_l[row] = l;
    }
    if constexpr (kBf16) {
#pragma unroll
      for (int d = 0; d < kND; ++d) *reinterpret_cast<f32x4_t*>(part_o + row * DH + column(d, 0)) = o[d];
    } else {
#pragma unroll
      for (int u = 0; u < kND / kVW; ++u)
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          cols_t v;
#pragma unroll
          for (int e = 0; e < kVW; ++e) v[e] = o[kVW * u + e][z];
          *reinterpret_cast<cols_t*>(part_o + row * DH + column(kVW * u, z)) = v;
        }
    }
  });
}

// Where the partial results of an item lie: those of its n_seg segments, item_rows rows apart, the first's at row0.
struct TreeParts {
  int n_seg;
  size_t row0;
};
// of part `part` of KV head g of the sequence in lane j of t, whose chunks start `off` chunks into the line
template <typename Cut>
__device__ __forceinline__ TreeParts tree_parts(const TreeShape& sh, const TreeBatch<Cut>& t, int j, uint32_t off,
                                                uint32_t share, int g, int part) {
  const uint32_t n = TreeBatch<Cut>::units(int(lane_of(uint32_t(t.keys), j)));
  const uint32_t items = TreeBatch<Cut>::items(sh, int(lane_of(uint32_t(t.T), j)));
  off += lane_of(t.upto, j) - lane_of(t.w, j) + (uint32_t(g) * items + uint32_t(part)) * n;
  const uint32_t wg0 = (off + Cut::kStart) / share;  // the first with a chunk of it
  return {n > 0 ? int((off + n - 1) / share - wg0) + 1 : 0,
          (size_t(wg0) + size_t((t.b0 + j) * sh.Hkv + g) * sh.items + part) << sh.item_shift};
}
// Running (maximum, sum) of a row over 64 segments of its item, first, first + step, ... < n_seg, one a lane; returns
// the weight of the lane's segment against the new maximum.  The row's states start at part_m, part_l + row0.
__device__ __forceinline__ float tree_fold(const float* part_m, const float* part_l, size_t row0, int item_shift,
                                           int n_seg, int first, int step, float& M, float& l, float& down) {
  const int p = first + step * int(threadIdx.x & 63);
  const size_t at = row0 + (size_t(min(p, n_seg - 1)) << item_shift);
  const float ms = part_m[at], ls = part_l[at];
  const float lp = p < n_seg ? ls : 0.f, mp = lp == 0.f ? -INFINITY : ms;  // 0: the segment holds nothing the row sees
  const float top = fmaxf(M, wave_max(mp)), ref = top == -INFINITY ? 0.f : top;
  down = fast_exp2(M - ref);
  const float f = lp == 0.f ? 0.f : fast_exp2(mp - ref);
  M = top;
  l = l * down + wave_sum(f * lp);
  return f;
}

// Joins the partial results of the segments of row (token tok, head h).  kWaves waves share a row and take every
// kWaves-th segment; a lane fetches the state of one segment, 64 at a time, and DH / 64 (at least one) columns of
// each.  Rows past the last sequence's are left as they are.  Latency bounds it, a chain of four loads: 6 us for a few
// rows, 8.0 us for 31 tokens of 32 heads in 8 sequences (34 MB of partial results).
template <typename T, int DH, int kWaves>
__device__ __forceinline__ void tree_join(const float* __restrict__ part_m, const float* __restrict__ part_l,
                                          const float* __restrict__ part_o, const int* __restrict__ lens,
                                          const int* __restrict__ cu_q, const TreeShape& sh, int wgs, int tok, int h,
                                          T* __restrict__ O, float* __restrict__ lse) {
  constexpr int kE = DH >= 64 ? DH / 64 : 1;
  typedef float vec_t __attribute__((ext_vector_type(kE)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = kWaves == 1 ? 0 : wave;
  if (h >= sh.Hq || tok >= cu_q[sh.B]) return;
  using Cut = AttnCut<T>;
  TreeBatch<Cut> t;
  const uint32_t total = tree_total<Cut>(sh, lens, cu_q, t), share = tree_share<Cut>(total, wgs);
  uint32_t off = 0;
  uint64_t here;
  while (!(here = __ballot(tok >= t.q0 && tok < t.q0 + t.T)) && t.b0 + 64 < sh.B) {
    off += t.all();
    t.fetch(sh, lens, cu_q, t.b0 + 64);
  }
  if (!here) return;  // counts out of range (invalid input)
  const int j = __builtin_ctzll(here), g = sh.token(h);
  const int r = (tok - int(lane_of(uint32_t(t.q0), j))) * sh.G + h - g * sh.G;
  const TreeParts parts = tree_parts(sh, t, j, off, share, g, r >> sh.item_shift);
  const size_t row0 = parts.row0 + (r & (sh.item_rows() - 1));
  const bool mine = kE * lane < DH;
  float M = -INFINITY, l = 0.f;
  vec_t o = 0.f;
  for (int p0 = first; p0 < parts.n_seg; p0 += 64 * kWaves) {
    const int n = min(64, (parts.n_seg - p0 + kWaves - 1) / kWaves);
    auto columns = [&](vec_t(&v)[4], int x) {  // of four segments
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[u] = 0.f;
        if (x + u < n && mine)
          v[u] = *reinterpret_cast<const vec_t*>(
              part_o + (row0 + (size_t(p0 + kWaves * (x + u)) << sh.item_shift)) * DH + kE * lane);
      }
    };
    vec_t v[4], next[4];
    columns(v, 0);  // on their way before the states have come
    float down;
    const float f = tree_fold(part_m, part_l, row0, sh.item_shift, parts.n_seg, p0, kWaves, M, l, down);
    o *= down;
    for (int x = 0; x < n; x += 4) {
      columns(next, x + 4);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        o += __uint_as_float(lane_of(__float_as_uint(f), min(x + u, 63))) * v[u];
        v[u] = next[u];
      }
    }
  }
  if constexpr (kWaves > 1) {
    __shared__ float sh_m[kWaves], sh_l[kWaves], sh_o[kWaves][64 * kE];
    if (lane == 0) {
      sh_m[wave] = M;
      sh_l[wave] = l;
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) sh_o[wave][kE * lane + e] = o[e];
    __syncthreads();
    if (wave != 0) return;
    M = -INFINITY;
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sh_m[w]);
    const float ref = M == -INFINITY ? 0.f : M;
    l = 0.f;
    o = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(sh_m[w] - ref);
      l = fmaf(f, sh_l[w], l);
#pragma unroll
      for (int e = 0; e < kE; ++e) o[e] = fmaf(f, sh_o[w][kE * lane + e], o[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (mine)
#pragma unroll
    for (int e = 0; e < kE; ++e) store1(O + (size_t(tok) * sh.Hq + h) * DH + kE * lane + e, o[e] * inv);
  if (lane == 0) lse[size_t(h) * sh.n_q + tok] = l == 0.f ? -INFINITY : kLn2 * (M + fast_log2(l));
}
constexpr int tree_join_threads(int waves) { return waves == 1 ? 256 : 64 * waves; }
// One workgroup a row, or four rows of a token (one wave a row).
template <typename T, int DH, int kWaves>
__global__ __launch_bounds__(tree_join_threads(kWaves)) void tree_join_kernel(
    const float* __restrict__ part_m, const float* __restrict__ part_l, const float* __restrict__ part_o,
    const int* __restrict__ lens, const int* __restrict__ cu_q, TreeShape sh, int wgs, T* __restrict__ O,
    float* __restrict__ lse) {
  const int h = kWaves == 1 ? int(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : int(blockIdx.y);
  tree_join<T, DH, kWaves>(part_m, part_l, part_o, lens, cu_q, sh, wgs, blockIdx.x, h, O, lse);
}

// The join, and beside it acc[b][g][key] += sum over the rows of exp(s - lse) from the scores (base 2) that the
// attention kernel has stored.  Workgroups n_join and on take 4 keys a thread of a (sequence, KV head), whose few rows'
// normalisers they form for themselves: so neither waits for the other's launch (6.7 us for one token at 32767, 7.3 us
// for 32 sequences of 500 to 4000; in two launches 11.5 and 13 us).
template <typename T, int DH, int kWaves>
__global__ __launch_bounds__(tree_join_threads(kWaves)) void tree_finish_kernel(
    const float* __restrict__ part_m, const float* __restrict__ part_l, const float* __restrict__ part_o,
    const int* __restrict__ lens, const int* __restrict__ cu_q, TreeShape sh, int wgs, T* __restrict__ O,
    float* __restrict__ lse, int n_join, const float* __restrict__ scores, int pitch, float* __restrict__ acc) {
  constexpr int kThreads = tree_join_threads(kWaves);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (int(blockIdx.x) < n_join) {
    const uint32_t per = kWaves == 1 ? uint32_t(sh.Hq + 3) / 4 : uint32_t(sh.Hq);  // workgroups of a token
    const uint32_t tok = blockIdx.x / per, y = blockIdx.x - tok * per;
    tree_join<T, DH, kWaves>(part_m, part_l, part_o, lens, cu_q, sh, wgs, int(tok),
                                            kWaves == 1 ? int(4 * y) + wave : int(y), O, lse);
    return;
  }
  __shared__ float lse2[16];
  const uint32_t id = blockIdx.x - n_join, groups = uint32_t(sh.B * sh.Hkv);
  const uint32_t bg = id % groups, k0 = id / groups * (4 * kThreads);
  const int b = int(bg / uint32_t(sh.Hkv)), g = int(bg) - b * sh.Hkv;
  using Cut = AttnCut<T>;
  TreeBatch<Cut> t;
  const uint32_t total = tree_total<Cut>(sh, lens, cu_q, t), share = tree_share<Cut>(total, wgs);
  uint32_t off = 0;
  while (t.b0 + 64 <= b) {
    off += t.all();
    t.fetch(sh, lens, cu_q, t.b0 + 64);
  }
  const int j = b - t.b0, keys = int(lane_of(uint32_t(t.keys), j)), R = int(lane_of(uint32_t(t.T), j)) * sh.G;
  if (int(k0) >= keys || R == 0) return;
  const TreeParts parts = tree_parts(sh, t, j, off, share, g, 0);
  const int k = int(k0) + 4 * int(threadIdx.x);
  const float* s = scores + size_t(bg) * sh.most_rows() * pitch + k;
  f32x4_t first{0.f, 0.f, 0.f, 0.f};  // the first row's, on their way
  if (k < keys) first = *reinterpret_cast<const f32x4_t*>(s);
  for (int r = wave; r < R; r += kThreads / 64) {
    float M = -INFINITY, l = 0.f, down;
    for (int p0 = 0; p0 < parts.n_seg; p0 += 64)
      tree_fold(part_m, part_l, parts.row0 + r, sh.item_shift, parts.n_seg, p0, 1, M, l, down);
    if ((threadIdx.x & 63) == 0) lse2[r] = l == 0.f ? INFINITY : M + fast_log2(l);  // (infinite: adds nothing)
  }
  __syncthreads();
  if (k >= keys) return;
  f32x4_t sum{0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < R; ++r) {
    const f32x4_t x = r == 0 ? first : *reinterpret_cast<const f32x4_t*>(s + size_t(r) * pitch);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += fast_exp2(x[e] - lse2[r]);
  }
  float* a = acc + size_t(bg) * sh.cap + k;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (k + e < keys) a[e] += sum[e];
}

// acc[b][g][key] += sum over the rows of w exp(s - lse) with the scores formed again.  An item's rows wait in LDS,
// 128 at a time, with their weights, normalisers and masks; a workgroup's share of 32-key tiles goes to its four
// waves in turn, a tile's K in registers (the next tile's under way) while the rows pass, 16 at a time.  A product's
// columns are rows: their sums join at the end of a tile, each exchange halving the values a lane still holds.  Every
// score costs an exponential and two FMAs (16 rows and 32 keys: 300 cycles of a SIMD); vector instructions are in flight
// 40 to 46 % of the cycles of long calls, and waits for K and LDS are the rest.  Short calls are bound by their ends, some
// 6 us until the first tile is done: 31 drafted tokens, 4 heads of 64 on a KV head, 8 sequences of 900 to 8100: 14.5 us
// (28 %); 23 tokens, heads of 128, 16 of 700 to 6000, a part of the rows accepted: 19.4 us, 4.6 TB/s.  fp32, the first at
// 8 of 4500: 64 us.
constexpr int kWRows = 128;  // rows in LDS
constexpr int kWKeys = 32;   // keys of a tile
// Workgroups of a compute unit: what its registers hold.
constexpr int tree_weight_wgs(int row_bytes) { return row_bytes >= 512 ? 2 : row_bytes >= 256 ? 3 : 4; }
template <typename T, int DH>
__global__ __launch_bounds__(256, tree_weight_wgs(DH * int(sizeof(T)))) void tree_weight_kernel(
    const T* __restrict__ Q, const T* __restrict__ K, const float* __restrict__ lse, const int* __restrict__ lens,
    const int* __restrict__ cu_q, const int64_t* __restrict__ mask, const float* __restrict__ row_weight, TreeShape sh,
    float c2, float* __restrict__ acc) {
  using Math = TreeMath<T>;
  using Frag = typename Math::Frag;
  constexpr int kRow = DH * int(sizeof(T)), kPieces = kRow / 16, kNF = kPieces / 4;
  constexpr int kWindow = kPieces >= 16 ? 1 : 16 / kPieces;
  struct RowInfo {  // of weight 0: not used
    float w, l2;
    uint64_t bits;
    int r;  // row of Q
  };
  __shared__ __attribute__((aligned(16))) char qs[kWRows * kRow];
  __shared__ __attribute__((aligned(16))) RowInfo info[kWRows];
  __shared__ int live[2];
  RowInfo mine{0.f, 0.f, 0, 0};
  int place = 0;
  const int tid = threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4, G = sh.G;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  tree_walk<TreeCut<kWKeys, 8, 4>>(sh, lens, cu_q, [&](const TreeSegment& q) {
    const int R = q.T * G;
    const size_t at = size_t(q.b * sh.Hkv + q.g) * sh.cap;
    auto load_k = [&](Frag(&kf)[2][kNF], int k) {
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const size_t key = at + size_t(min(k + 16 * a + fr, q.keys - 1));
#pragma unroll
        for (int c = 0; c < kNF; ++c)
          kf[a][c] = reinterpret_cast<const Frag*>(K + key * DH)[4 * c + fq];
      }
    };
    for (int r0 = 0; r0 < R; r0 += kWRows) {
      Frag kf[2][kNF], kn[2][kNF];
      const int first = q.k0 + kWKeys * wave;
      if (first < q.k1) load_k(kf, first);
      int n_rows = min(kWRows, R - r0);
      __syncthreads();  // the last rows are read
      // the rows that count, next to each other (of a tree often few: the accepted ones); the rest of the last 16 are
      // the last of them again, with weight 0 and an infinite normaliser
      if (tid < kWRows) {
        RowInfo x{0.f, 0.f, 0, 0};
        if (tid < n_rows) {
          const int r = r0 + tid, t = sh.token(r), tok = q.q0 + t;
          const float w = row_weight ? row_weight[tok] : 1.f, l = lse[size_t(q.g * G + r - t * G) * sh.n_q + tok];
          const uint64_t bits = tree_bits(mask, q, t);
          if (w != 0.f && l != -INFINITY) x = RowInfo{w, l * kLog2e, bits, tok * sh.Hq + q.g * G + r - t * G};
        }
        const uint64_t counts = __ballot(x.w != 0.f);
        if (lane == 0) live[wave] = int(__popcll(counts));
        info[tid] = RowInfo{0.f, INFINITY, 0, 0};
        mine = x;
        place = int(__popcll(counts & ((uint64_t(1) << lane) - 1)));
      }
      __syncthreads();
      if (tid < kWRows && mine.w != 0.f) info[place + (wave == 1 ? live[0] : 0)] = mine;
      n_rows = live[0] + live[1];
      __syncthreads();
      for (int i = tid; i < (n_rows + 15) / 16 * 16 * kPieces; i += 256) {
        const int row = i / kPieces, c = i % kPieces, r = info[min(row, n_rows - 1)].r;
        *reinterpret_cast<uint4*>(qs + row * kRow + (c ^ (row / kWindow & (kPieces - 1))) * 16) =
            reinterpret_cast<const uint4*>(Q)[size_t(r) * kPieces + c];
      }
      __syncthreads();
      for (int k = first; k < q.k1; k += 4 * kWKeys) {
        const bool edge = k + kWKeys > q.len;
        const int key = k + 16 * ((fr >> 2) & 1) + 4 * fq + (fr & 3);  // whose sum ends up in this lane (fr < 8)
        const bool writes = fr < 8 && key < q.keys && n_rows > 0;
        float was = 0.f;
        if (writes) was = acc[at + key];
        if (k + 4 * kWKeys < q.k1) load_k(kn, k + 4 * kWKeys);
        float sum[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        auto add_rows = [&](auto at_edge) {
          for (int r = 0; r < n_rows; r += 16) {
            const float w = info[r + fr].w, l2 = info[r + fr].l2;
            const uint64_t bits = decltype(at_edge)::value ? info[r + fr].bits : 0;
            Frag qf[kNF];
#pragma unroll
            for (int c = 0; c < kNF; ++c)
              qf[c] = *reinterpret_cast<const Frag*>(qs + (r + fr) * kRow +
                                                         ((4 * c + fq) ^ ((r + fr) / kWindow & (kPieces - 1))) * 16);
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const uint32_t sees = decltype(at_edge)::value ? tree_sees4(bits, k + 16 * a + 4 * fq - q.len) : 15u;
              f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int c = 0; c < kNF; ++c) s = Math::scores(kf[a][c], qf[c], s);
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                // (cached keys are seen by every row; one behind the last adds 0 exp2(score - infinity), NaN only where
                // the last row's is)
                const float p = fast_exp2(fmaf(s[z], c2, -l2));
                if constexpr (decltype(at_edge)::value)
                  sum[4 * a + z] = (sees >> z) & 1 ? fmaf(w, p, sum[4 * a + z]) : sum[4 * a + z];
                else
                  sum[4 * a + z] = fmaf(w, p, sum[4 * a + z]);
              }
            }
          }
        };
        if (edge)
          add_rows(std::true_type{});
        else
          add_rows(std::false_type{});
#pragma unroll
        for (int half = 4; half >= 1; half >>= 1) {
          const bool upper = (fr & half) != 0;
#pragma unroll
          for (int e = 0; e < half; ++e) {
            const float keep = upper ? sum[e + half] : sum[e], give = upper ? sum[e] : sum[e + half];
            sum[e] = keep + __shfl_xor(give, half, 64);
          }
        }
        sum[0] += __shfl_xor(sum[0], 8, 64);
        if (writes) acc[at + key] = was + sum[0];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int c = 0; c < kNF; ++c) kf[a][c] = kn[a][c];
      }
    }
  });
}

// ------------------------------------------------------------------ plan and workspace

// How a call is cut: items of 2^item_shift rows, 16 a wave, at most `items` of them a
// (sequence, KV head), their chunks shared by `wgs` workgroups.
struct TreePlan {
  int waves;  // of a workgroup
  int item_shift, items, wgs;
  bool stored;  // the scores are kept for the account, if there is one and the workspace holds them
};
// Waves that share a ring: as many as have a transfer of each part (two at a head size of 32).
constexpr int tree_waves(int dh) { return dh == 32 ? 2 : 4; }
// LDS of tree_attn_kernel: the ring, and the rows of Q of several waves.
inline int tree_lds(int dh, int waves, int es) { return 320 * dh + (waves > 1 ? waves * 16 * dh * es : 0); }
inline TreePlan plan_tree(int B, int max_q, int max_kv, int Hq, int Hkv, int dh, int dtype) {
  const int64_t rows = int64_t(max_q) * (Hq / Hkv);
  TreePlan p;
  // One wave's rows up to 16: with 8 sequences of 4096, heads of 128, 12 rows take 41.7 us so and 50.5 us with three
  // waves idle.  More rows: 20 rows 36.2 us with four waves of 16 rows, 38.2 us with a wave of 32; 64 rows 41.6 and
  // 59.9; 92 rows at 16 sequences of 3000 63.3 and 113.6.
  p.waves = rows <= 16 ? 1 : tree_waves(dh);
  p.item_shift = p.waves == 1 ? 4 : p.waves == 2 ? 5 : 6;
  p.items = int((rows + (1 << p.item_shift) - 1) >> p.item_shift);
  // one grid fills the chip: what 160 KB of LDS hold of the rings, or registers of the waves, on 256 units
  const int64_t fill = p.waves == 1 ? 1024 * (128 / dh) : 512 * std::min(128 / dh, 4);
  const int64_t shares = (int64_t(B) * Hkv * p.items * ((int64_t(max_kv) + 31) / 32) + 3) / 4;  // at most
  p.wgs = int((std::min(fill, shares) + 7) / 8 * 8);
  // Scores: 8 bytes a row and key, written and read, against 2 dh for forming them again.  8 sequences of 4096 or 8192,
  // attention with account, kept against formed again: dh 128, 4 rows 42 and 49 us, 16 rows 50.5 and 50.8; dh 64, 4
  // rows 27.3 and 32.8, 8 rows 47.9 and 50.1, 16 rows 53.8 and 51.6; dh 32, 4 rows 29.4 and 33.0, 8 rows 34.6 and
  // 34.5.
  p.stored = p.waves == 1 && rows * 16 <= dh * (dtype == ESTP_F32 ? 4 : 2);
  return p;
}

struct TreeBuffers {
  float *m, *l, *o, *lse, *scores;
  int pitch;
  size_t bytes;
};
inline TreeBuffers carve_tree(const TreePlan& p, int B, int max_q, int64_t n_q, int Hq, int Hkv, int max_kv, int dh,
                              void* ws) {
  // a segment more than the last for every workgroup and for every item
  const size_t rows = (size_t(p.wgs) + size_t(B) * Hkv * p.items) << p.item_shift;
  Carver c(ws);
  TreeBuffers t;
  t.m = c.take<float>(rows);
  t.l = c.take<float>(rows);
  t.o = c.take<float>(rows * dh);
  t.lse = c.take<float>(size_t(n_q) * Hq);
  t.pitch = (max_kv + 31) / 32 * 32;
  t.scores = c.take<float>(p.stored ? size_t(B) * max_q * Hq * t.pitch : 0);
  t.bytes = c.bytes();
  return t;
}

int check_tree_args(const char* fn, const void* Q, const void* K, const int32_t* lens, const int32_t* cu_q, int B,
                    int max_q, int64_t n_q, int Hq, int Hkv, int64_t cap, int max_kv, int dh, float scale, int dtype) {
  ESTP_REQUIRE(Q && K && lens && cu_q, ESTP_ERR_INVALID_ARG, "%s: Q, K, lens and cu_q must be non-null", fn);
  ESTP_REQUIRE(B >= 1 && n_q >= 1 && n_q <= INT32_MAX && Hq >= 1 && Hkv >= 1, ESTP_ERR_INVALID_ARG,
               "%s: B, n_q, Hq and Hkv must be >= 1", fn);
  ESTP_REQUIRE(Hq % Hkv == 0, ESTP_ERR_INVALID_ARG, "%s: Hq = %d is not a multiple of Hkv = %d", fn, Hq, Hkv);
  ESTP_REQUIRE(max_q >= 1 && max_q <= n_q, ESTP_ERR_INVALID_ARG, "%s: max_q = %d must be in [1, n_q = %lld]", fn, max_q,
               (long long)n_q);
  ESTP_REQUIRE(cap >= 1 && cap <= INT32_MAX - 256 && max_kv >= 1 && max_kv <= cap, ESTP_ERR_INVALID_ARG,
               "%s: max_kv = %d must be in [1, cap = %lld]", fn, max_kv, (long long)cap);
  ESTP_REQUIRE(n_q <= int64_t(B) * max_q, ESTP_ERR_INVALID_ARG, "%s: n_q = %lld, more than B max_q = %lld", fn,
               (long long)n_q, (long long)B * max_q);
  ESTP_REQUIRE(std::isfinite(scale) && scale > 0.f, ESTP_ERR_INVALID_ARG, "%s: scale must be finite and > 0", fn);
  ESTP_REQUIRE(dtype == ESTP_BF16 || dtype == ESTP_F32, ESTP_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  ESTP_REQUIRE(aligned(Q, 16) && aligned(K, 16), ESTP_ERR_INVALID_ARG, "%s: Q and K must be 16-byte aligned", fn);
  ESTP_REQUIRE(aligned(lens, 4) && aligned(cu_q, 4), ESTP_ERR_INVALID_ARG, "%s: lens and cu_q must be 4-byte aligned",
               fn);
  ESTP_REQUIRE(dh == 32 || dh == 64 || dh == 128, ESTP_ERR_UNSUPPORTED, "%s: head_dim %d not in {32, 64, 128}", fn, dh);
  ESTP_REQUIRE(max_q <= kMaxTree, ESTP_ERR_UNSUPPORTED, "%s: max_q = %d, at most %d drafted tokens", fn, max_q,
               kMaxTree);
  ESTP_REQUIRE(int64_t(max_q) * (Hq / Hkv) <= 65535 && Hq / Hkv <= 32768 && Hq <= 65535, ESTP_ERR_UNSUPPORTED,
               "%s: %d query heads, %d sharing a KV head", fn, Hq, Hq / Hkv);
  ESTP_REQUIRE(int64_t(B) * Hkv <= 65535 && n_q * Hq <= INT32_MAX / 64, ESTP_ERR_UNSUPPORTED,
               "%s: B Hkv = %lld (at most 65535) or n_q Hq = %lld too large", fn, (long long)B * Hkv,
               (long long)n_q * Hq);
  const size_t tiles = (size_t(max_kv) + 63) / 64;
  ESTP_REQUIRE(fits_launch(tiles * size_t(B) * Hkv, 256), ESTP_ERR_UNSUPPORTED, "%s: B Hkv max_kv too large", fn);
  return ESTP_OK;
}

// ESTP_DEBUG_CHECKS=1: lens and cu_q against what the header asks of them, before any kernel reads them
int debug_check_tree(const char* fn, const int32_t* lens, const int32_t* cu_q, int B, int max_q, int64_t n_q,
                     int max_kv, hipStream_t s) {
  if (!debug_checks_enabled()) return ESTP_OK;
  std::vector<int> l, cu;
  int st = debug_copy(fn, "lens", lens, size_t(B), s, &l);
  if (st == ESTP_OK) st = debug_copy(fn, "cu_q", cu_q, size_t(B) + 1, s, &cu);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(cu[0] == 0, ESTP_ERR_INVALID_ARG, "%s: debug check: cu_q[0] = %d, must be 0", fn, cu[0]);
  for (int b = 0; b < B; ++b) {
    const int64_t T = int64_t(cu[b + 1]) - cu[b];
    ESTP_REQUIRE(T >= 0 && T <= max_q, ESTP_ERR_INVALID_ARG,
                 "%s: debug check: sequence %d has %lld drafted tokens, must be in [0, max_q = %d]", fn, b,
                 (long long)T, max_q);
    ESTP_REQUIRE(l[b] >= 0 && l[b] + T <= max_kv, ESTP_ERR_INVALID_ARG,
                 "%s: debug check: sequence %d has %d cached and %lld drafted tokens, max_kv = %d", fn, b, l[b],
                 (long long)T, max_kv);
  }
  ESTP_REQUIRE(cu[B] <= n_q, ESTP_ERR_INVALID_ARG, "%s: debug check: cu_q[B] = %d, n_q = %lld", fn, cu[B],
               (long long)n_q);
  return ESTP_OK;
}

// acc: with stored scores, else null
template <typename T, int DH>
int launch_tree(const T* Q, const T* K, const T* V, const int* lens, const int* cu_q, const int64_t* mask,
                const TreeShape& sh, const TreePlan& p, float scale, T* O, float* lse, float* acc,
                const TreeBuffers& t, hipStream_t s) {
  const dim3 grid{unsigned(p.wgs)};
  auto kernel = p.waves > 1 ? tree_attn_kernel<T, DH, tree_waves(DH), false>
                : acc       ? tree_attn_kernel<T, DH, 1, true>
                            : tree_attn_kernel<T, DH, 1, false>;
  kernel<<<grid, dim3(64 * p.waves), tree_lds(DH, p.waves, int(sizeof(T))), s>>>(
      Q, K, V, lens, cu_q, mask, sh, scale * kLog2e, t.scores, t.pitch, t.m, t.l, t.o);
  ESTP_CHECK_LAUNCH("tree_attn_kernel");
  // Segments of an item, about, and by them the waves of a row.  18 segments (8 sequences of 4096, 64 rows of 64): one
  // wave 27.1 us with the attention, four 30.1; 34 segments (the same, 16 rows): 24.9 and 23.5; 66 (2 of 16000, 4
  // rows of 128): four 33.3, sixteen 32.8; 130 (one of 32767): one 47.4, four 35.8, sixteen 33.4.
  const int64_t segs = std::min<int64_t>(int64_t(p.wgs) / (int64_t(sh.B) * sh.Hkv * p.items), sh.max_kv / 128) + 2;
  auto join = [&](auto waves) -> int {
    constexpr int kWaves = decltype(waves)::value, kThreads = tree_join_threads(kWaves);
    const int per = kWaves == 1 ? (sh.Hq + 3) / 4 : sh.Hq;  // workgroups of a token
    if (acc) {
      const unsigned n_join = unsigned(sh.n_q) * unsigned(per);
      const unsigned n_keys = unsigned((sh.max_kv + 4 * kThreads - 1) / (4 * kThreads)) * unsigned(sh.B * sh.Hkv);
      tree_finish_kernel<T, DH, kWaves><<<dim3(n_join + n_keys), dim3(kThreads), 0, s>>>(
          t.m, t.l, t.o, lens, cu_q, sh, p.wgs, O, lse, int(n_join), t.scores, t.pitch, acc);
      ESTP_CHECK_LAUNCH("tree_finish_kernel");
      return ESTP_OK;
    }
    tree_join_kernel<T, DH, kWaves><<<dim3(unsigned(sh.n_q), unsigned(per)), dim3(kThreads), 0, s>>>(
        t.m, t.l, t.o, lens, cu_q, sh, p.wgs, O, lse);
    ESTP_CHECK_LAUNCH("tree_join_kernel");
    return ESTP_OK;
  };
  if (segs <= 24) return join(std::integral_constant<int, 1>{});
  if (segs <= 64) return join(std::integral_constant<int, 4>{});
  return join(std::integral_constant<int, 16>{});
}
template <typename T, int DH>
int launch_weight(const T* Q, const T* K, const float* lse, const int* lens, const int* cu_q, const int64_t* mask,
                  const float* row_weight, TreeShape sh, float scale, float* acc, hipStream_t s) {
  sh.item_shift = 16;  // all rows of a (sequence, KV head) in one item: one workgroup adds to a slot
  const size_t shares = (size_t(sh.max_kv) + 127) / 128 * size_t(sh.B) * sh.Hkv;  // of 128 keys or more: at most
  const dim3 grid(unsigned(std::min<size_t>(256 * tree_weight_wgs(DH * int(sizeof(T))), (shares + 7) / 8 * 8)));
  tree_weight_kernel<T, DH><<<grid, dim3(256), 0, s>>>(Q, K, lse, lens, cu_q, mask, row_weight, sh, scale * kLog2e,
                                                       acc);
  ESTP_CHECK_LAUNCH("tree_weight_kernel");
  return ESTP_OK;
}

// f(element, head size) for the call's type and head size
template <typename F>
int tree_dispatch(int dtype, int dh, F&& f) {
  if (dtype == ESTP_F32) {
    if (dh == 32) return f(float{}, std::integral_constant<int, 32>{});
    if (dh == 64) return f(float{}, std::integral_constant<int, 64>{});
    return f(float{}, std::integral_constant<int, 128>{});
  }
  if (dh == 32) return f(uint16_t{}, std::integral_constant<int, 32>{});
  if (dh == 64) return f(uint16_t{}, std::integral_constant<int, 64>{});
  return f(uint16_t{}, std::integral_constant<int, 128>{});
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_tree_attention_workspace_size(int32_t B, int32_t max_q, int64_t n_q, int32_t Hq, int32_t Hkv,
                                                     int32_t max_kv, int32_t dh, int dtype) {
  if (B < 1 || max_q < 1 || n_q < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || max_kv < 1 || dh < 1 ||
      max_kv > INT32_MAX - 256)
    return 0;
  return carve_tree(plan_tree(B, max_q, max_kv, Hq, Hkv, dh, dtype), B, max_q, n_q, Hq, Hkv, max_kv, dh, nullptr)
      .bytes;
}

extern "C" int estp_tree_attention(const void* Q, const void* K, const void* V, const int32_t* lens,
                                   const int32_t* cu_q, const int64_t* tree_mask, int32_t B, int32_t max_q,
                                   int64_t n_q, int32_t Hq, int32_t Hkv, int64_t cap, int32_t max_kv, int32_t dh,
                                   float scale, int dtype, void* O, float* lse, float* acc, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_tree_attention";
  const int st = check_tree_args(fn, Q, K, lens, cu_q, B, max_q, n_q, Hq, Hkv, cap, max_kv, dh, scale, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(V && O, ESTP_ERR_INVALID_ARG, "%s: V and O must be non-null", fn);
  ESTP_REQUIRE(aligned(V, 16) && aligned(O, 16) && aligned(tree_mask, 8) && aligned(lse, 4) && aligned(acc, 4),
               ESTP_ERR_INVALID_ARG, "%s: V and O must be 16-byte, tree_mask 8-byte, lse and acc 4-byte aligned", fn);
  // A workspace without room for the scores serves too, as that of a larger max_q, whose scores are formed again: they
  // are formed again here, too.
  TreePlan p = plan_tree(B, max_q, max_kv, Hq, Hkv, dh, dtype);
  p.stored = p.stored && acc &&
             workspace_bytes >= estp_tree_attention_workspace_size(B, max_q, n_q, Hq, Hkv, max_kv, dh, dtype);
  const size_t need = carve_tree(p, B, max_q, n_q, Hq, Hkv, max_kv, dh, nullptr).bytes;
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  ESTP_REQUIRE(fits_launch(2 * size_t(n_q) * Hq, 1024) &&
                   int64_t(B) * Hkv * p.items * ((int64_t(max_kv) + 15) / 16 + 4) <= INT32_MAX,
               ESTP_ERR_UNSUPPORTED, "%s: B Hkv max_kv max_q Hq too large", fn);
  const TreeShape sh = tree_shape(B, max_q, n_q, Hq, Hkv, cap, max_kv, p.item_shift, p.items);
  const TreeBuffers t = carve_tree(p, B, max_q, n_q, Hq, Hkv, max_kv, dh, workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int checked = debug_check_tree(fn, lens, cu_q, B, max_q, n_q, max_kv, s);
  if (checked != ESTP_OK) return checked;
  float* row_lse = lse ? lse : t.lse;
  return tree_dispatch(dtype, dh, [&](auto element, auto size) -> int {
    using T = decltype(element);
    constexpr int DH = decltype(size)::value;
    const int rc = launch_tree<T, DH>(static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V),
                                      lens, cu_q, tree_mask, sh, p, scale, static_cast<T*>(O), row_lse,
                                      p.stored ? acc : nullptr, t, s);
    if (rc != ESTP_OK || !acc || p.stored) return rc;
    return launch_weight<T, DH>(static_cast<const T*>(Q), static_cast<const T*>(K), row_lse, lens, cu_q, tree_mask,
                                nullptr, sh, scale, acc, s);
  });
}

extern "C" int estp_tree_importance(const void* Q, const void* K, const float* lse, const int32_t* lens,
                                    const int32_t* cu_q, const int64_t* tree_mask, const float* row_weight, int32_t B,
                                    int32_t max_q, int64_t n_q, int32_t Hq, int32_t Hkv, int64_t cap, int32_t max_kv,
                                    int32_t dh, float scale, int dtype, float* acc, void* stream) {
  clear_error();
  const char* fn = "estp_tree_importance";
  const int st = check_tree_args(fn, Q, K, lens, cu_q, B, max_q, n_q, Hq, Hkv, cap, max_kv, dh, scale, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(lse && acc, ESTP_ERR_INVALID_ARG, "%s: lse and acc must be non-null", fn);
  ESTP_REQUIRE(aligned(tree_mask, 8) && aligned(lse, 4) && aligned(acc, 4) && aligned(row_weight, 4),
               ESTP_ERR_INVALID_ARG, "%s: tree_mask must be 8-byte, lse, row_weight and acc 4-byte aligned", fn);
  const TreeShape sh = tree_shape(B, max_q, n_q, Hq, Hkv, cap, max_kv, 4, 1);
  const int checked = debug_check_tree(fn, lens, cu_q, B, max_q, n_q, max_kv, static_cast<hipStream_t>(stream));
  if (checked != ESTP_OK) return checked;
  return tree_dispatch(dtype, dh, [&](auto element, auto size) -> int {
    using T = decltype(element);
    return launch_weight<T, decltype(size)::value>(static_cast<const T*>(Q), static_cast<const T*>(K), lse, lens, cu_q,
                                                   tree_mask, row_weight, sh, scale, acc,
                                                   static_cast<hipStream_t>(stream));
  });
}
