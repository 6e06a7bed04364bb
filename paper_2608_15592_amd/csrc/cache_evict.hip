// Eviction from a cache by accumulated attention weight.
//
// Of the lens[b] slots of a (sequence, KV head) the `keep` best stay: first
// those guarded by their position (the first `sink` and the last `recent`
// positions), then by the weight in acc, the lowest slot among equals.  The
// kept slots past `keep` (survivors) move into the evicted ones before it
// (holes), both in ascending order: no row moves that need not, sources
// (>= keep) and destinations (< keep) never overlap, so all rows of K and V
// move at once in place.  The order of the slots carries no meaning, their
// positions are in pos.
//
// evict_select_kernel, one workgroup per (sequence, KV head), a thread per every 1024th slot: the weights' keys stay in
// registers (caches of up to 16384 slots; longer ones are cut, see below).  Four histogram passes of 8 bits in LDS find
// the key of the last one kept; places in slot order (of ties, holes and survivors) come from ballots, a count per 64
// slots, one prefix over all counts.  Latency bounds it: so every wave searches the histogram and forms the prefix for
// itself, which leaves one barrier a pass and a prefix.  The survivors' rows move in the same kernel where they are
// few, else in evict_move_kernel.  Everything is exact: whole numbers and copies.
//
// 6 groups of 1029 slots cut to 1024: 8.7 us.  256 groups of 700 to 4096 slots cut to 1024, heads of 128: selection
// 11.5 us, then 22 us for the rows, 100 MB read and written at 4.5 TB/s.  64 groups of 16384 slots: selection 35 us on a
// compute unit a group, where vector instructions are in flight some two fifths of the cycles and waves wait 54 % of
// theirs, for barriers and LDS.
#include <algorithm>
#include <vector>

#include "estp_common.h"
#include "lds_ops.h"

namespace estp {
namespace detail {

typedef uint32_t piece_t __attribute__((ext_vector_type(4)));  // 16 bytes of a row
constexpr int kEThreads = 1024;
constexpr int kEWaves = kEThreads / 64;
constexpr int kMovesHere = 256;  // rows that evict_select_kernel moves itself, at most

// Weights as whole numbers in the same order: NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float v) {
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u & 0x7fffffffu) == 0) return 0x80000000u;
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// One row of the slots' 1024: the thread's slot of round i is 1024 i + tid.
struct EvictArgs {
  const float* acc;
  const int *pos, *lens, *seen;
  int Hkv, cap, keep, recent, sink;
  float* acc_out;
  int *pos_out, *idx;
  int2* moves;
  int* n_moves;
  piece_t *K, *V;  // rows moved here, or null: by evict_move_kernel
  int row16;
  int* lens_out;  // written here when the rows are
};

// Pieces first, first + step, ... of the listed rows, four at a time: their places, then their loads, are in flight
// together.  row16 is a power of two.
__device__ __forceinline__ void move_rows(piece_t* __restrict__ K, piece_t* __restrict__ V, size_t base, int row16,
                                          const int2* moves, int n, int64_t first, int64_t step) {
  constexpr int kAhead = 4;
  const int shift = __builtin_ctz(unsigned(row16));
  const int64_t total = int64_t(n) << shift;
  for (int64_t i = first; i < total; i += kAhead * step) {
    int from[kAhead], to[kAhead];
    piece_t k[kAhead], v[kAhead];
    int c[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t at = min(i + u * step, total - 1);
      const int2 e = moves[at >> shift];
      from[u] = e.x;
      to[u] = e.y;
      c[u] = int(at) & (row16 - 1);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const size_t p = ((base + from[u]) << shift) + c[u];
      k[u] = K[p];
      v[u] = V[p];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i + u * step < total) {
        const size_t p = ((base + to[u]) << shift) + c[u];
        K[p] = k[u];
        V[p] = v[u];
      }
  }
}

// kE rounds of 1024 slots in registers.
template <int kE>
__global__ __launch_bounds__(kEThreads) void evict_select_kernel(EvictArgs g) {
  constexpr int kHists = 2;               // copies of the histogram: equal weights meet on fewer threads
  constexpr int kPer = (kE * kEWaves + 63) / 64;  // counts of a lane
  constexpr bool kRaw = kE <= 4;  // weights and positions stay in registers, not the keys alone
  __shared__ __attribute__((aligned(16))) uint32_t hist[4][kHists][256];  // of the four digits
  __shared__ uint32_t n_guarded_sh, counts[2][64 * kPer];
  __shared__ int hole_sh[kE * (kEThreads / 2)];  // at most half of the slots
  __shared__ int2 moves_sh[kMovesHere];
  const int bg = blockIdx.x, b = bg / g.Hkv, tid = threadIdx.x, lane = tid & 63, keep = g.keep;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t base = size_t(bg) * g.cap;
  const float* acc = g.acc + base;
  const int* pos = g.pos + base;
  float* acc_out = g.acc_out + base;
  int* pos_out = g.pos_out + base;
  int* idx = g.idx + size_t(bg) * keep;
  int2* moves = g.moves + size_t(bg) * keep;
  const bool copy = acc_out != acc || pos_out != pos;
  // the whole capacity's weights and positions, on their way while the length is
  float a[kRaw ? kE : 1];
  int ps[kRaw ? kE : 1];
  if constexpr (kRaw) {
#pragma unroll
    for (int r = 0; r < kE; ++r) {
      const int i = min(r * kEThreads + tid, g.cap - 1);
      a[r] = acc[i];
      ps[r] = pos[i];
    }
  }
  const int n = max(0, min(g.lens[b], g.cap));
  const int64_t first_recent = int64_t(g.seen[b]) - g.recent;
  for (int i = tid; i < 4 * kHists * 256; i += kEThreads) (&hist[0][0][0])[i] = 0;
  for (int i = tid; i < 2 * 64 * kPer; i += kEThreads) (&counts[0][0])[i] = 0;
  if (tid == 0) n_guarded_sh = 0;
  if (g.K && tid == 0 && bg % g.Hkv == 0) g.lens_out[b] = min(n, keep);
  if (n <= keep) {  // everything stays
    for (int i = tid; i < keep; i += kEThreads) idx[i] = i < n ? i : -1;
    if (copy)
      for (int i = tid; i < n; i += kEThreads) {
        acc_out[i] = acc[i];
        pos_out[i] = pos[i];
      }
    if (tid == 0) g.n_moves[bg] = 0;
    return;
  }
  auto is_guarded = [&](int p) { return p < g.sink || p >= first_recent; };
  auto weight = [&](int r) {
    if constexpr (kRaw)
      return a[r];
    else
      return acc[r * kEThreads + tid];
  };
  auto position = [&](int r) {
    if constexpr (kRaw)
      return ps[r];
    else
      return pos[r * kEThreads + tid];
  };
  auto each_round = [&](auto&& f) {
#pragma unroll
    for (int r = 0; r < kE; ++r)
      if (r * kEThreads < n) f(r);
  };
  auto rounds_in_memory = [&](auto&& f) {  // what needs no keys
    if constexpr (kRaw) {
      each_round(f);
    } else {
#pragma unroll 2
      for (int r = 0; r < min(kE, (n + kEThreads - 1) / kEThreads); ++r) f(r);
    }
  };
  // choice[r]: one more than the key of round r's slot, 0 where there is none or it is not in the choice
  uint32_t choice[kE];
  uint64_t guard = 0;  // a bit a round
#pragma unroll
  for (int r = 0; r < kE; ++r) {
    const bool in = r * kEThreads + tid < n;
    choice[r] = 0;
    if (in) choice[r] = 1 + weight_key(weight(r));
    guard |= uint64_t(in && is_guarded(position(r))) << r;
  }
  auto guarded = [&](int r) { return ((guard >> r) & 1) != 0; };
  __syncthreads();
  uint32_t in_wave = 0;
  each_round([&](int r) { in_wave += uint32_t(__popcll(__ballot(guarded(r)))); });
  if (lane == 0 && in_wave) atomicAdd(&n_guarded_sh, in_wave);
  __syncthreads();
  // guarded slots: all stay if they fit, else the best of them do and nothing else
  const int n_guarded = int(n_guarded_sh);
  const bool among = n_guarded >= keep;  // whether the choice is among the guarded slots
  uint32_t need = uint32_t(among ? keep : keep - n_guarded);
#pragma unroll
  for (int r = 0; r < kE; ++r) choice[r] = guarded(r) == among ? choice[r] : 0;
  // the number of the need-th best in the choice, 8 bits at a time; `need` becomes how many of its equals stay.  (At
  // least `need` are in the choice: what is not, 0, is never reached.)
  uint32_t prefix = 0;
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    each_round([&](int r) {
      const uint32_t k = choice[r];
      if (pass == 0 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
        atomicAdd(&hist[pass][wave % kHists][255 - ((k >> shift) & 255)], 1u);
    });
    __syncthreads();
    // descending digits: lane j has the counts of 255 - 4 j down to 252 - 4 j; where the running count reaches `need`
    u32x4_t c = *reinterpret_cast<const u32x4_t*>(&hist[pass][0][4 * lane]);
#pragma unroll
    for (int h = 1; h < kHists; ++h) c += *reinterpret_cast<const u32x4_t*>(&hist[pass][h][4 * lane]);
    const uint32_t sum = (c[0] + c[1]) + (c[2] + c[3]), upto = wave_prefix(sum);
    const uint64_t reached = __ballot(upto >= need);
    const int j = reached ? __builtin_ctzll(reached) : 63;
    uint32_t above = lane_of(upto, j) - lane_of(sum, j), digit = uint32_t(255 - 4 * j);
#pragma unroll
    for (int z = 0; z < 3; ++z) {
      const uint32_t cz = lane_of(c[z], j);
      if (digit == uint32_t(255 - 4 * j - z) && above + cz < need) {
        above += cz;
        --digit;
      }
    }
    prefix |= digit << shift;
    need -= above;
  }

  // Places in slot order: first the ties are counted, to see which of them stay, then holes (low half) and survivors
  // (high half).  A count for every 64 slots, one prefix over all counts, the lanes' own.
  auto below = [&](bool x) { return uint32_t(__popcll(__ballot(x) & ((uint64_t(1) << lane) - 1))); };
  // Exclusive prefix of a count array (16 a round), which every wave forms for itself: lane j holds counts kPer j ..,
  // of which the wave needs one.
  struct Prefix {
    uint32_t mine, total;
    int shift_lane;
    __device__ __forceinline__ uint32_t of(int round) const {
      return lane_of(mine, round * (kEWaves / kPer) + shift_lane);
    }
  };
  auto prefix_of = [&](const uint32_t* counted) {
    uint32_t c[kPer], sum = 0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      c[q] = counted[kPer * lane + q];
      sum += c[q];
    }
    const uint32_t upto = wave_prefix(sum);
    uint32_t run = upto - sum;
    Prefix p{0, lane_of(upto, 63), wave / kPer};
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      p.mine = wave % kPer == q ? run : p.mine;
      run += c[q];
    }
    return p;
  };
  uint64_t tie = 0, stays = 0;  // a bit a round
  each_round([&](int r) {
    const uint32_t k = choice[r];
    const bool t = k == prefix;
    tie |= uint64_t(t) << r;
    stays |= uint64_t(k > prefix || (!among && guarded(r))) << r;
    const uint64_t m = __ballot(t);
    if (lane == 0) counts[0][r * kEWaves + wave] = uint32_t(__popcll(m));
  });
  __syncthreads();
  {
    const Prefix p = prefix_of(counts[0]);
    rounds_in_memory([&](int r) {
      const bool t = (tie >> r) & 1;
      const uint32_t rank = p.of(r) + below(t);
      if (t && rank < need) stays |= uint64_t(1) << r;
    });
  }
  rounds_in_memory([&](int r) {  // (at most 8192 of either)
    const int i = r * kEThreads + tid;
    const bool st = (stays >> r) & 1;
    const uint64_t h = __ballot(i < n && i < keep && !st), l = __ballot(st && i >= keep);
    if (lane == 0) counts[1][r * kEWaves + wave] = uint32_t(__popcll(h)) | uint32_t(__popcll(l)) << 16;
  });
  __syncthreads();
  const Prefix p = prefix_of(counts[1]);
  rounds_in_memory([&](int r) {  // holes are listed, kept slots below `keep` copied
    const int i = r * kEThreads + tid;
    const bool st = (stays >> r) & 1, hole = i < n && i < keep && !st;
    const uint32_t h = (p.of(r) & 0xffff) + below(hole);
    if (hole) hole_sh[h] = i;
    if (st && i < keep) {
      idx[i] = i;
      if (copy) {
        acc_out[i] = weight(r);
        pos_out[i] = position(r);
      }
    }
  });
  __syncthreads();
  rounds_in_memory([&](int r) {
    const int i = r * kEThreads + tid;
    const bool late = ((stays >> r) & 1) && i >= keep;
    const uint32_t l = (p.of(r) >> 16) + below(late);
    if (i < n && i >= keep) {
      if (late) {
        const int to = hole_sh[l];
        idx[to] = i;
        acc_out[to] = weight(r);
        pos_out[to] = position(r);
        if (g.K)
          moves_sh[l] = int2{i, to};
        else
          moves[l] = int2{i, to};
      }
      acc_out[i] = 0.f;  // a freed slot
      pos_out[i] = -1;
    }
  });
  if (g.K) __syncthreads();
  const int holes = int(p.total & 0xffff);  // as many as survivors
  if (tid == 0) g.n_moves[bg] = holes;
  if (g.K) move_rows(g.K, g.V, base, g.row16, moves_sh, holes, tid, kEThreads);
}

// The listed rows of K and V.  Also writes lens_out, which may be lens: by now evict_select_kernel has read it.
__global__ __launch_bounds__(256) void evict_move_kernel(piece_t* __restrict__ K, piece_t* __restrict__ V, int cap,
                                                         int row16, const int2* __restrict__ moves, int keep,
                                                         const int* __restrict__ n_moves, const int* lens, int Hkv,
                                                         int* lens_out) {
  const int bg = blockIdx.y, n = n_moves[bg];
  if (blockIdx.x == 0 && threadIdx.x == 0 && bg % Hkv == 0) lens_out[bg / Hkv] = min(max(lens[bg / Hkv], 0), keep);
  move_rows(K, V, size_t(bg) * cap, row16, moves + size_t(bg) * keep, n, int64_t(blockIdx.x) * 256 + threadIdx.x,
            int64_t(gridDim.x) * 256);
}

// ------------------------------------------------------------------ long caches
//
// A group of more slots than kMostHeld is cut into segments, a workgroup each, none across slot `keep`.  The weights'
// digits are 11, 11 and 10 bits: evict_hist_kernel counts a segment's digits (the first for guarded slots and others
// apart), the next launch adds up all segments' counts, finds the digit and counts the next one.  The counts also say
// how many slots of each segment stay, so evict_place_kernel knows where a segment's holes (slots below `keep`, first
// launch) and survivors (second launch, which moves their rows where they fill the chip) stand in the order of all.
// Five launches, each a read of the weights at most and 5 to 20 us: 64 groups of 60000 slots cut to 2048, head size 64,
// take 91 us (one workgroup a group, with its keys in registers, took 151), of 131072 cut to 4096 138 us (reading them
// on each pass 598).  The launches and what each adds up before it starts bound it: caches of up to 16384 slots are
// faster with a group on one workgroup (16384 cut to 2048: 46 us, so 60).

constexpr int kMostHeld = 16 * kEThreads;
constexpr int kBins = 2048;       // of a digit
constexpr int kSegments = 16;     // of a group at most, and one more for the cut at `keep`
constexpr int64_t kAllSegments = 512;  // of all groups, about; every group has one and one more
struct EvictCut {
  int seg, low, n;  // slots of a segment; segments of [0, keep); of the capacity
};
inline EvictCut evict_cut(int64_t groups, int64_t cap, int keep) {
  const int64_t most = std::min<int64_t>(kSegments, std::max<int64_t>(1, kAllSegments / groups - 1));
  const int64_t seg = std::max<int64_t>(4096, (cap + most - 1) / most + kEThreads - 1) / kEThreads * kEThreads;
  const int64_t low = (keep + seg - 1) / seg;
  return {int(seg), int(low), int(low + (cap - keep + seg - 1) / seg)};
}
// At least as many as evict_cut makes of so many groups or fewer, whatever the capacity and `keep`: a workspace of a
// larger call serves a smaller one, whose groups may be cut into more.
inline size_t evict_segments_room(size_t groups) {
  return std::min<size_t>((kSegments + 1) * groups, std::max<size_t>(kAllSegments, 2 * groups));
}
struct EvictLong {
  EvictArgs g;
  EvictCut cut;
  uint32_t* hist[2];   // [group][segment][2 kBins], [kBins]: of the even and the odd digits
  uint32_t* counted;   // [group][segment][4]: guarded slots, and how many of the choice pass the first, second digit
  uint32_t* state;     // [group][2][4]: after each of two digits what is found of the key, how many of those stay, among
  int* n_of;           // [group]: slots in use, at first
  int* lens_out;
};
struct EvictSegment {
  int bg, s, n, lo, hi;  // slots [lo, hi), none: hi <= lo
};
__device__ __forceinline__ int segment_start(const EvictLong& e, int s) {
  return s < e.cut.low ? s * e.cut.seg : min(e.g.cap, e.g.keep + (s - e.cut.low) * e.cut.seg);
}
__device__ __forceinline__ EvictSegment evict_segment(const EvictLong& e, int bg, int s, int n) {
  const int lo = segment_start(e, s);
  const int64_t to = int64_t(lo) + e.cut.seg, end = s < e.cut.low ? min(int64_t(e.g.keep), to) : to;
  return {bg, s, n, lo, int(min(int64_t(n), end))};
}
// Segments that hold slots of a group with n > keep in use: the first so many.
__device__ __forceinline__ int live_segments(const EvictLong& e, int n) {
  int x = 0;
  while (x < e.cut.n && segment_start(e, x) < n) ++x;
  return x;
}
// The bin (digits in descending order) at which the running count of the bins reaches `need`, and the count of those
// before it; c holds bins per tid .. per tid + per - 1, per 1 or 2.  Every thread gets both.
__device__ __forceinline__ void find_bin(int per, uint32_t need, const uint32_t (&c)[2], uint32_t* sh, uint32_t* bin,
                                         uint32_t* before) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t sum = c[0] + c[1], upto = wave_prefix(sum);
  __syncthreads();  // sh may hold what the caller has read
  if (lane == 63) sh[wave] = upto;
  if (tid == 0) {
    sh[16] = 0;
    sh[17] = 0;
  }
  __syncthreads();
  uint32_t run = upto - sum;
  for (int w = 0; w < kEWaves; ++w) run += w < wave ? sh[w] : 0;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (run < need && run + c[q] >= need) {
      sh[16] = uint32_t(tid * per + q);
      sh[17] = run;
    }
    run += c[q];
  }
  __syncthreads();
  *bin = sh[16];
  *before = sh[17];
}
struct EvictState {
  uint32_t key, need;  // digits found (the others 0); how many of the slots that fit them stay
  bool among;          // the choice is among the guarded slots
};
__device__ __forceinline__ uint32_t digit_shift(int digit) { return digit == 0 ? 21u : digit == 1 ? 10u : 0u; }
// What digit `digit` adds to the state: from the sums of all segments' counts of it.
__device__ __forceinline__ EvictState next_digit(const EvictLong& e, int bg, int n, int digit, uint32_t* sh) {
  EvictState st{0, 0, false};
  const uint32_t* h = e.hist[digit & 1];
  const size_t pitch = digit & 1 ? kBins : 2 * kBins, first = size_t(bg) * e.cut.n;
  const int live = live_segments(e, n), lane = threadIdx.x & 63;
  if (digit == 0) {
    const uint32_t g = lane < live ? e.counted[(first + lane) * 4] : 0;
    const uint32_t guarded = lane_of(wave_prefix(g), 63);
    st.among = guarded >= uint32_t(e.g.keep);
    st.need = st.among ? uint32_t(e.g.keep) : uint32_t(e.g.keep) - guarded;
  } else {
    const uint32_t* from = e.state + (size_t(bg) * 2 + digit - 1) * 4;
    st = EvictState{from[0], from[1], from[2] != 0};
  }
  // all segments' counts, on their way together
  const int per = digit == 2 ? 1 : 2;
  const uint32_t* mine = h + first * pitch + (digit == 0 && st.among ? kBins : 0) + threadIdx.x * per;
  uint32_t c[2] = {0, 0}, bin, before;
  uint2 x[kSegments + 1];
#pragma unroll
  for (int s = 0; s <= kSegments; ++s) {
    const uint32_t* from = mine + s * pitch;
    x[s] = uint2{0, 0};
    if (s >= live) continue;
    if (digit == 2)
      x[s].x = from[0];
    else
      x[s] = *reinterpret_cast<const uint2*>(from);
  }
#pragma unroll
  for (int s = 0; s <= kSegments; ++s) {
    c[0] += x[s].x;
    c[1] += x[s].y;
  }
  find_bin(per, st.need, c, sh, &bin, &before);
  st.need -= before;
  st.key |= uint32_t((digit == 2 ? kBins / 2 : kBins) - 1 - int(bin)) << digit_shift(digit);
  return st;
}
__device__ __forceinline__ bool evict_guarded(const EvictArgs& g, int pos, int64_t first_recent) {
  return pos < g.sink || pos >= first_recent;
}

template <int kDigit>
__global__ __launch_bounds__(kEThreads) void evict_hist_kernel(EvictLong e) {
  __shared__ uint32_t hist[2 * kBins], sh[32];
  const int bg = blockIdx.x / e.cut.n, s = blockIdx.x - bg * e.cut.n, b = bg / e.g.Hkv, tid = threadIdx.x;
  const int n = max(0, min(e.g.lens[b], e.g.cap));
  if (kDigit == 0 && s == 0 && tid == 0) e.n_of[bg] = n;
  if (n <= e.g.keep) return;
  const EvictSegment q = evict_segment(e, bg, s, n);
  if (q.hi <= q.lo) return;
  constexpr int kSides = kDigit == 0 ? 2 : 1, kMine = kDigit == 2 ? kBins / 2 : kBins;
  const size_t at = size_t(bg) * e.cut.n + s;
  EvictState st{0, 0, false};
  if (kDigit > 0) {
    st = next_digit(e, bg, n, kDigit - 1, sh);
    if (s == 0 && tid == 0) {
      uint32_t* to = e.state + (size_t(bg) * 2 + kDigit - 1) * 4;
      to[0] = st.key;
      to[1] = st.need;
      to[2] = st.among;
    }
    // this segment's slots that pass the digit
    const int mine = kBins - 1 - int((st.key >> digit_shift(kDigit - 1)) & (kBins - 1));
    const uint32_t* h = e.hist[(kDigit - 1) & 1] + at * (kDigit == 1 ? 2 * kBins : kBins) +
                        (kDigit == 1 && st.among ? kBins : 0);
    uint32_t over = 0;
    for (int i = tid; i < mine; i += kEThreads) over += h[i];
    const uint32_t wave_over = wave_prefix(over);
    __syncthreads();
    if (tid == 0) sh[20] = 0;
    __syncthreads();
    if ((tid & 63) == 63) atomicAdd(&sh[20], wave_over);
    __syncthreads();
    if (tid == 0) e.counted[at * 4 + kDigit] = sh[20];
  }
  for (int i = tid; i < kSides * kBins; i += kEThreads) hist[i] = 0;
  if (tid == 0) sh[21] = 0;
  __syncthreads();
  const float* acc = e.g.acc + size_t(bg) * e.g.cap;
  const int* pos = e.g.pos + size_t(bg) * e.g.cap;
  const int64_t first_recent = int64_t(e.g.seen[b]) - e.g.recent;
  uint32_t guarded = 0;
#pragma unroll 4
  for (int i = q.lo + tid; i < q.hi; i += kEThreads) {
    const uint32_t k = 1 + weight_key(acc[i]);
    const bool in_guard = evict_guarded(e.g, pos[i], first_recent);
    guarded += in_guard;
    if (kDigit == 0)
      atomicAdd(&hist[(in_guard ? kBins : 0) + kBins - 1 - (k >> 21)], 1u);
    else if (in_guard == st.among && (k >> digit_shift(kDigit - 1)) == (st.key >> digit_shift(kDigit - 1)))
      atomicAdd(&hist[kMine - 1 - ((k >> digit_shift(kDigit)) & (kMine - 1))], 1u);
  }
  if (kDigit == 0 && guarded) atomicAdd(&sh[21], guarded);
  __syncthreads();
  uint32_t* out = e.hist[kDigit & 1] + at * (kDigit & 1 ? kBins : 2 * kBins);
  for (int i = tid; i < kSides * kMine; i += kEThreads) out[i] = hist[i];
  if (kDigit == 0 && tid == 0) e.counted[at * 4] = sh[21];
}

// kHigh: survivors of the segments past `keep`, each into its hole; else the holes of the segments before it, and what
// stays there.
template <bool kHigh>
__global__ __launch_bounds__(kEThreads) void evict_place_kernel(EvictLong e, int segments) {
  constexpr int kAhead = 64 / kEWaves;  // rounds of 1024 slots that are worked off together
  __shared__ uint32_t sh[32], ties[kSegments + 2], stay[kSegments + 2], counts[2][64];
  const int bg = blockIdx.x / segments, s = blockIdx.x - bg * segments + (kHigh ? e.cut.low : 0), tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6, keep = e.g.keep, b = bg / e.g.Hkv, n = e.n_of[bg];
  if (kHigh && bg % e.g.Hkv == 0 && s == e.cut.low && tid == 0) e.lens_out[b] = min(n, keep);
  const size_t base = size_t(bg) * e.g.cap;
  const float* acc = e.g.acc + base;
  const int* pos = e.g.pos + base;
  float* acc_out = e.g.acc_out + base;
  int* pos_out = e.g.pos_out + base;
  int* idx = e.g.idx + size_t(bg) * keep;
  const bool copy = acc_out != acc || pos_out != pos;
  if (n <= keep) {  // everything stays
    if (kHigh && s == e.cut.low && tid == 0) e.g.n_moves[bg] = 0;
    if (kHigh) return;
    const int end = int(min(int64_t(keep), int64_t(s + 1) * e.cut.seg));
    for (int i = s * e.cut.seg + tid; i < end; i += kEThreads) {
      idx[i] = i < n ? i : -1;
      if (copy && i < n) {
        acc_out[i] = acc[i];
        pos_out[i] = pos[i];
      }
    }
    return;
  }
  const EvictSegment q = evict_segment(e, bg, s, n);
  if (q.hi <= q.lo) return;
  const size_t first = size_t(bg) * e.cut.n;
  const EvictState st = next_digit(e, bg, n, 2, sh);
  // of every segment: slots of the threshold's weight, and slots that stay whatever happens to those
  const int mine = kBins / 2 - 1 - int(st.key & (kBins / 2 - 1));
  const int live = live_segments(e, n);
  for (int x = wave; x < live; x += kEWaves) {
    const uint32_t* h = e.hist[0] + (first + x) * (2 * kBins);
    uint32_t over = 0;
#pragma unroll
    for (int i = 0; i < kBins / 2; i += 64) {
      const uint32_t c = h[i + lane];
      over += i + lane < mine ? c : 0;
    }
    const uint32_t all = lane_of(wave_prefix(over), 63);
    if (lane == 0) {
      const uint32_t* c = e.counted + (first + x) * 4;
      ties[x] = h[mine];
      stay[x] = all + c[1] + c[2] + (st.among ? 0u : c[0]);
    }
  }
  __syncthreads();
  // before this segment: ties, and holes or survivors
  uint32_t ties_before = 0, placed = 0;
  for (int x = 0; x < s; ++x) {
    const uint32_t t = ties[x], kept = ties_before < st.need ? min(t, st.need - ties_before) : 0u;
    if (x < e.cut.low && !kHigh)
      placed += uint32_t(min(int64_t(keep), int64_t(x + 1) * e.cut.seg)) - uint32_t(x * e.cut.seg) - stay[x] - kept;
    else if (x >= e.cut.low && kHigh)
      placed += stay[x] + kept;
    ties_before += t;
  }
  const int64_t first_recent = int64_t(e.g.seen[b]) - e.g.recent;
  int2* list = e.g.moves + size_t(bg) * keep;
  // The places of a thread's slots among those of 4 rounds that m marks (a ballot a round): every wave counts its own,
  // lane j then has the count of round j / 16, wave j % 16.
  auto places = [&](const uint64_t (&m)[kAhead], int which, uint32_t (&at)[kAhead]) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (lane == 0) counts[which][u * kEWaves + wave] = uint32_t(__popcll(m[u]));
    __syncthreads();
    const uint32_t c = counts[which][lane], upto = wave_prefix(c);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      at[u] = lane_of(upto - c, u * kEWaves + wave) + uint32_t(__popcll(m[u] & ((uint64_t(1) << lane) - 1)));
    return lane_of(upto, 63);
  };
  const uint32_t first_placed = placed;
  for (int64_t r = q.lo; r < q.hi; r += kAhead * kEThreads) {
    float a[kAhead];
    int p[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t i = min(r + u * kEThreads + tid, int64_t(q.hi) - 1);
      a[u] = acc[i];
      p[u] = pos[i];
    }
    bool stays[kAhead], tie[kAhead], in[kAhead];
    uint64_t m[kAhead];
    uint32_t at[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      in[u] = r + u * kEThreads + tid < q.hi;
      const uint32_t k = 1 + weight_key(a[u]);
      const bool in_guard = in[u] && evict_guarded(e.g, p[u], first_recent), chosen = in[u] && in_guard == st.among;
      tie[u] = chosen && k == st.key;
      stays[u] = (chosen && k > st.key) || (!st.among && in_guard);
      m[u] = __ballot(tie[u]);
    }
    const uint32_t n_ties = places(m, 0, at);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      stays[u] |= tie[u] && ties_before + at[u] < st.need;
      m[u] = __ballot(in[u] && stays[u] == kHigh);
    }
    const uint32_t n_placed = places(m, 1, at);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (!in[u]) continue;
      const int i = int(r) + u * kEThreads + tid;
      int2* const entry = list + min(placed + at[u], uint32_t(keep - 1));
      if (kHigh) {
        if (stays[u]) {
          const int to = entry->y;
          entry->x = i;
          idx[to] = i;
          acc_out[to] = a[u];
          pos_out[to] = p[u];
        }
        acc_out[i] = 0.f;  // a freed slot
        pos_out[i] = -1;
      } else if (!stays[u]) {
        entry->y = i;
      } else {
        idx[i] = i;
        if (copy) {
          acc_out[i] = a[u];
          pos_out[i] = p[u];
        }
      }
    }
    ties_before += n_ties;
    placed += n_placed;
    __syncthreads();  // the counts are read, the list is written
  }
  if (kHigh && q.hi == n && tid == 0) e.g.n_moves[bg] = int(placed);
  if (kHigh && e.g.K)
    move_rows(e.g.K, e.g.V, base, e.g.row16, list + first_placed, int(placed - first_placed), tid, kEThreads);
}

struct EvictBuffers {
  int2* moves;
  int* n_moves;
  EvictLong e;  // of long caches
  size_t bytes;
};
inline EvictBuffers carve_evict(size_t groups, int64_t cap, int keep, void* ws) {
  Carver c(ws);
  EvictBuffers b{};
  b.moves = c.take<int2>(groups * size_t(keep));
  b.n_moves = c.take<int>(groups);
  if (cap > kMostHeld) {
    b.e.cut = evict_cut(int64_t(groups), cap, keep);
    const size_t segments = evict_segments_room(groups);
    b.e.hist[0] = c.take<uint32_t>(segments * 2 * kBins);
    b.e.hist[1] = c.take<uint32_t>(segments * kBins);
    b.e.counted = c.take<uint32_t>(segments * 4);
    b.e.state = c.take<uint32_t>(groups * 2 * 4);
    b.e.n_of = c.take<int>(groups);
  }
  b.bytes = c.bytes();
  return b;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_cache_evict_workspace_size(int32_t B, int32_t Hkv, int64_t cap, int32_t keep) {
  if (B < 1 || Hkv < 1 || keep < 1 || cap < keep || cap > INT32_MAX - 65536) return 0;
  return carve_evict(size_t(B) * size_t(Hkv), cap, keep, nullptr).bytes;
}

extern "C" int estp_cache_evict(void* K, void* V, const float* acc, const int32_t* pos, const int32_t* lens,
                                const int32_t* seen, int32_t B, int32_t Hkv, int64_t cap, int32_t dh, int dtype,
                                int32_t keep, int32_t recent, int32_t sink, float* acc_out, int32_t* pos_out,
                                int32_t* lens_out, int32_t* idx, void* workspace, size_t workspace_bytes,
                                void* stream) {
  clear_error();
  const char* fn = "estp_cache_evict";
  ESTP_REQUIRE(K && V && acc && pos && lens && seen && acc_out && pos_out && lens_out && idx, ESTP_ERR_INVALID_ARG,
               "%s: no pointer but the workspace and the stream may be null", fn);
  ESTP_REQUIRE(K != V, ESTP_ERR_INVALID_ARG, "%s: K and V are the same memory", fn);
  ESTP_REQUIRE(B >= 1 && Hkv >= 1 && cap >= 1 && cap <= INT32_MAX - 65536, ESTP_ERR_INVALID_ARG,
               "%s: B, Hkv and cap must be >= 1, cap below 2^31 - 65536", fn);
  ESTP_REQUIRE(dtype == ESTP_BF16 || dtype == ESTP_F32, ESTP_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  ESTP_REQUIRE(keep >= 1 && keep <= cap, ESTP_ERR_INVALID_ARG, "%s: keep = %d must be in [1, cap = %lld]", fn, keep,
               (long long)cap);
  ESTP_REQUIRE(recent >= 0 && sink >= 0 && int64_t(recent) + sink <= keep, ESTP_ERR_INVALID_ARG,
               "%s: recent = %d and sink = %d must be >= 0 and fit into keep = %d", fn, recent, sink, keep);
  ESTP_REQUIRE(dh == 32 || dh == 64 || dh == 128, ESTP_ERR_UNSUPPORTED, "%s: head_dim %d not in {32, 64, 128}", fn, dh);
  ESTP_REQUIRE(int64_t(B) * Hkv <= 65535, ESTP_ERR_UNSUPPORTED, "%s: B Hkv = %lld, at most 65535", fn,
               (long long)B * Hkv);
  ESTP_REQUIRE(aligned(K, 16) && aligned(V, 16), ESTP_ERR_INVALID_ARG, "%s: K and V must be 16-byte aligned", fn);
  ESTP_REQUIRE(aligned(acc, 4) && aligned(pos, 4) && aligned(lens, 4) && aligned(seen, 4) && aligned(acc_out, 4) &&
                   aligned(pos_out, 4) && aligned(lens_out, 4) && aligned(idx, 4),
               ESTP_ERR_INVALID_ARG, "%s: acc, pos, lens, seen and the outputs must be 4-byte aligned", fn);
  const size_t need = estp_cache_evict_workspace_size(B, Hkv, cap, keep);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  const int groups = B * Hkv;
  EvictBuffers e = carve_evict(size_t(groups), cap, keep, workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (debug_checks_enabled()) {
    std::vector<int> l;
    const int st = debug_copy(fn, "lens", lens, size_t(B), s, &l);
    if (st != ESTP_OK) return st;
    for (int b = 0; b < B; ++b)
      ESTP_REQUIRE(l[b] >= 0 && l[b] <= cap, ESTP_ERR_INVALID_ARG,
                   "%s: debug check: sequence %d has %d slots in use, cap = %lld", fn, b, l[b], (long long)cap);
  }
  const int row16 = dh * (dtype == ESTP_F32 ? 4 : 2) / 16;
  const int64_t most = std::min<int64_t>(keep, cap - keep) * row16;  // 16-byte pieces that can move, of K or V
  // Rows move in the selecting kernel where there can be few: a kernel of their own costs its launch, but spreads the
  // rows over the chip (B Hkv = 64, 1152 slots cut to 1024, head size 128: here 10.9 us, apart 13.5; 1280 slots, fp32:
  // 14.2 against 16.0; B Hkv = 256: 25.6 against 29.7).  Not in place of lens, which workgroups of the same sequence
  // still read.
  const bool here = std::min<int64_t>(keep, cap - keep) <= kMovesHere && lens_out != lens;
  EvictArgs g{acc, pos, lens, seen, Hkv, int(cap), keep, recent, sink, acc_out, pos_out, idx, e.moves, e.n_moves,
              here ? static_cast<piece_t*>(K) : nullptr, static_cast<piece_t*>(V), row16, lens_out};
  if (cap > kMostHeld) {
    EvictLong& l = e.e;
    l.g = g;
    // The rows move with their places where the survivors' workgroups fill the chip, else in a launch of their own that
    // does.  60000 slots cut to 30000, head size 128: 2 groups 71.8 us with, 54.0 apart; 16 groups 122.8 and 94.8; 32
    // groups, of 256 such workgroups, 173.1 and 174.3.
    const int high = std::max(1, l.cut.n - l.cut.low);
    const bool with_places = int64_t(groups) * high >= 256;
    l.g.K = with_places ? static_cast<piece_t*>(K) : nullptr;
    l.lens_out = lens_out;
    const dim3 all(unsigned(groups * l.cut.n)), block(kEThreads);
    evict_hist_kernel<0><<<all, block, 0, s>>>(l);
    evict_hist_kernel<1><<<all, block, 0, s>>>(l);
    evict_hist_kernel<2><<<all, block, 0, s>>>(l);
    ESTP_CHECK_LAUNCH("evict_hist_kernel");
    evict_place_kernel<false><<<dim3(unsigned(groups * l.cut.low)), block, 0, s>>>(l, l.cut.low);
    evict_place_kernel<true><<<dim3(unsigned(groups * high)), block, 0, s>>>(l, high);
    ESTP_CHECK_LAUNCH("evict_place_kernel");
    if (with_places) return ESTP_OK;
  } else {
    // Rounds in registers: all are gone through.  64 groups: 4096 slots 12.5 us in 4 rounds, 15.8 in 16.
    auto select = cap <= 4 * kEThreads ? evict_select_kernel<4> : evict_select_kernel<16>;
    select<<<dim3(unsigned(groups)), dim3(kEThreads), 0, s>>>(g);
    ESTP_CHECK_LAUNCH("evict_select_kernel");
    if (here) return ESTP_OK;
  }
  const int64_t wgs = std::max<int64_t>(1, std::min<int64_t>((most + 255) / 256, std::max(1, 4096 / groups)));
  evict_move_kernel<<<dim3(unsigned(wgs), unsigned(groups)), dim3(256), 0, s>>>(
      static_cast<piece_t*>(K), static_cast<piece_t*>(V), int(cap), row16, e.moves, keep, e.n_moves, lens, Hkv,
      lens_out);
  ESTP_CHECK_LAUNCH("evict_move_kernel");
  return ESTP_OK;
}
