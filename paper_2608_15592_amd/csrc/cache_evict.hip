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
// evict_select_kernel, one workgroup per (sequence, KV head), a thread per every 1024th slot: the weights' keys
// stay in registers (caches of up to 65536 slots; longer ones are read again on each pass).  Four histogram passes of
// 8 bits in LDS find the key of the last one kept; places in slot order (of ties, holes and survivors) come from
// ballots, a count per 64 slots, one prefix over all counts.  Latency bounds it: so every wave searches the histogram
// and forms the prefix for itself, which leaves one barrier a pass and a prefix.  The survivors' rows move in the same
// kernel where they are few, else in evict_move_kernel.  Everything is exact: whole numbers and copies.
//
// 6 groups of 1029 slots cut to 1024: 8.7 us.  256 groups of 700 to 4096 slots cut to 1024,
// heads of 128: selection 11.2 us, then 22 us for the rows, 100 MB read and written at 4.5 TB/s.  Past 4096 slots a
// group's vector instructions bound it: selection in 64 groups of 16384 slots 35 us, of 65536 153 us, of 100000, from
// memory, 421 us.  One group stays on one compute unit, so few groups leave the others idle.
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

// kE rounds of 1024 slots in registers; kE = 0: any number, read from memory on every pass.
template <int kE>
__global__ __launch_bounds__(kEThreads) void evict_select_kernel(EvictArgs g) {
  constexpr int kHists = 2;               // copies of the histogram: equal weights meet on fewer threads
  constexpr int kSpan = kE > 0 ? kE : 32;  // rounds whose counts one prefix covers
  constexpr int kPer = (kSpan * kEWaves + 63) / 64;  // counts of a lane
  constexpr bool kHeld = kE > 0;           // keys stay in registers, holes in LDS
  constexpr bool kRaw = kE > 0 && kE <= 4;  // weights and positions too
  __shared__ __attribute__((aligned(16))) uint32_t hist[4][kHists][256];  // of the four digits
  __shared__ uint32_t n_guarded_sh, counts[2][64 * kPer];
  __shared__ int hole_sh[kHeld ? kE * (kEThreads / 2) : 1];  // at most half of the slots
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
  const int rounds = kE > 0 ? kE : (n + kEThreads - 1) / kEThreads;
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
  auto rounds_from = [&](int r0, int r1, auto&& f) {
    if constexpr (kE > 0) {
#pragma unroll
      for (int r = 0; r < kE; ++r)
        if (r * kEThreads < n) f(r);
    } else {
#pragma unroll 4
      for (int r = r0; r < r1; ++r) f(r);
    }
  };
  auto rounds_in_memory = [&](int r0, int r1, auto&& f) {  // what needs no keys
    if constexpr (kRaw) {
      rounds_from(r0, r1, f);
    } else {
#pragma unroll 2
      for (int r = r0; r < min(r1, (n + kEThreads - 1) / kEThreads); ++r) f(r);
    }
  };
  // choice[r]: one more than the key of round r's slot, 0 where there is none or it is not in the choice
  uint32_t choice[kHeld ? kE : 1];
  uint64_t guard = 0;  // a bit a round
  if constexpr (kHeld) {
#pragma unroll
    for (int r = 0; r < kE; ++r) {
      const bool in = r * kEThreads + tid < n;
      choice[r] = 0;
      if (in) choice[r] = 1 + weight_key(weight(r));
      guard |= uint64_t(in && is_guarded(position(r))) << r;
    }
  }
  auto guarded = [&](int r) {
    if constexpr (kHeld)
      return ((guard >> r) & 1) != 0;
    else
      return r * kEThreads + tid < n && is_guarded(position(r));
  };
  __syncthreads();
  uint32_t in_wave = 0;
  rounds_from(0, rounds, [&](int r) { in_wave += uint32_t(__popcll(__ballot(guarded(r)))); });
  if (lane == 0 && in_wave) atomicAdd(&n_guarded_sh, in_wave);
  __syncthreads();
  // guarded slots: all stay if they fit, else the best of them do and nothing else
  const int n_guarded = int(n_guarded_sh);
  const bool among = n_guarded >= keep;  // whether the choice is among the guarded slots
  uint32_t need = uint32_t(among ? keep : keep - n_guarded);
  if constexpr (kHeld) {
#pragma unroll
    for (int r = 0; r < kE; ++r) choice[r] = guarded(r) == among ? choice[r] : 0;
  }
  auto chosen_by = [&](int r) {
    if constexpr (kHeld) {
      return choice[r];
    } else {
      const bool in = r * kEThreads + tid < n;
      return in && guarded(r) == among ? 1 + weight_key(weight(r)) : 0u;
    }
  };
  // the number of the need-th best in the choice, 8 bits at a time; `need` becomes how many of its equals stay.  (At
  // least `need` are in the choice: what is not, 0, is never reached.)
  uint32_t prefix = 0;
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    rounds_from(0, rounds, [&](int r) {
      uint32_t k;
      if constexpr (kHeld) {
        k = choice[r];
      } else {  // (the position is read where the digits before this one fit)
        if (r * kEThreads + tid >= n) return;
        k = 1 + weight_key(weight(r));
      }
      if (pass == 0 || (k >> (shift + 8)) == (prefix >> (shift + 8))) {
        if constexpr (!kHeld)
          if (guarded(r) != among) return;
        atomicAdd(&hist[pass][wave % kHists][255 - ((k >> shift) & 255)], 1u);
      }
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

  // Places in slot order, over spans of rounds: first the ties are counted, to see which of them stay, then holes (low
  // half) and survivors (high half).  A count for every 64 slots, one prefix over all counts, the lanes' own.
  uint32_t ties_before = 0, holes_before = 0, late_before = 0;
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
  for (int r0 = 0; r0 < rounds; r0 += kSpan) {
    const int r1 = min(rounds, r0 + kSpan);
    uint64_t tie = 0, stays = 0;  // a bit a round
    rounds_from(r0, r1, [&](int r) {
      const uint32_t k = chosen_by(r);
      const bool t = k == prefix;
      tie |= uint64_t(t) << (r - r0);
      stays |= uint64_t(k > prefix || (!among && guarded(r))) << (r - r0);
      const uint64_t m = __ballot(t);
      if (lane == 0) counts[0][(r - r0) * kEWaves + wave] = uint32_t(__popcll(m));
    });
    __syncthreads();
    {
      const Prefix p = prefix_of(counts[0]);
      rounds_in_memory(r0, r1, [&](int r) {
        const bool t = (tie >> (r - r0)) & 1;
        const uint32_t rank = ties_before + p.of(r - r0) + below(t);
        if (t && rank < need) stays |= uint64_t(1) << (r - r0);
      });
      ties_before += p.total;
    }
    // holes in the low half, survivors in the high one: at most 32768 each a span
    rounds_in_memory(r0, r1, [&](int r) {
      const int i = r * kEThreads + tid;
      const bool st = (stays >> (r - r0)) & 1;
      const uint64_t h = __ballot(i < n && i < keep && !st), l = __ballot(st && i >= keep);
      if (lane == 0) counts[1][(r - r0) * kEWaves + wave] = uint32_t(__popcll(h)) | uint32_t(__popcll(l)) << 16;
    });
    __syncthreads();
    const Prefix p = prefix_of(counts[1]);
    rounds_in_memory(r0, r1, [&](int r) {  // holes are listed, kept slots below `keep` copied
      const int i = r * kEThreads + tid;
      const bool st = (stays >> (r - r0)) & 1, hole = i < n && i < keep && !st;
      const uint32_t h = holes_before + (p.of(r - r0) & 0xffff) + below(hole);
      if (hole) {
        if constexpr (kHeld)
          hole_sh[h] = i;
        else
          moves[h].y = i;
      }
      if (st && i < keep) {
        idx[i] = i;
        if (copy) {
          acc_out[i] = weight(r);
          pos_out[i] = position(r);
        }
      }
    });
    __syncthreads();  // every hole that this span's survivors fill is listed: all holes lie before all survivors
    rounds_in_memory(r0, r1, [&](int r) {
      const int i = r * kEThreads + tid;
      const bool late = ((stays >> (r - r0)) & 1) && i >= keep;
      const uint32_t l = late_before + (p.of(r - r0) >> 16) + below(late);
      if (i < n && i >= keep) {
        if (late) {
          int to;
          if constexpr (kHeld)
            to = hole_sh[l];
          else
            to = moves[l].y;
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
    holes_before += p.total & 0xffff;
    late_before += p.total >> 16;
    if (kE == 0) {  // the next span may be shorter: no counts of this one's stay
      __syncthreads();
      for (int i = tid; i < 2 * 64 * kPer; i += kEThreads) (&counts[0][0])[i] = 0;
      __syncthreads();
    }
  }
  if (g.K) __syncthreads();
  const int holes = int(holes_before);  // as many as survivors
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

struct EvictBuffers {
  int2* moves;
  int* n_moves;
  size_t bytes;
};
inline EvictBuffers carve_evict(size_t groups, int keep, void* ws) {
  Carver c(ws);
  EvictBuffers e;
  e.moves = c.take<int2>(groups * size_t(keep));
  e.n_moves = c.take<int>(groups);
  e.bytes = c.bytes();
  return e;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_cache_evict_workspace_size(int32_t B, int32_t Hkv, int32_t keep) {
  if (B < 1 || Hkv < 1 || keep < 1) return 0;
  return carve_evict(size_t(B) * size_t(Hkv), keep, nullptr).bytes;
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
  const size_t need = estp_cache_evict_workspace_size(B, Hkv, keep);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  const int groups = B * Hkv;
  const EvictBuffers e = carve_evict(size_t(groups), keep, workspace);
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
  // Rounds in registers: the fewest that hold the capacity, as all are gone through.  64 groups, us: 4096 slots 12.5 in
  // 4 rounds, 15.8 in 16; 10000 slots 35.4 in 16, 38.4 in 32; 32768 slots 87 in 32, 114 in 64; 65536 slots 210 in 64,
  // 291 from memory.
  auto select = cap <= 4 * kEThreads    ? evict_select_kernel<4>
                : cap <= 16 * kEThreads ? evict_select_kernel<16>
                : cap <= 32 * kEThreads ? evict_select_kernel<32>
                : cap <= 64 * kEThreads ? evict_select_kernel<64>
                                        : evict_select_kernel<0>;
  select<<<dim3(unsigned(groups)), dim3(kEThreads), 0, s>>>(g);
  ESTP_CHECK_LAUNCH("evict_select_kernel");
  if (here) return ESTP_OK;
  const int64_t wgs = std::max<int64_t>(1, std::min<int64_t>((most + 255) / 256, std::max(1, 4096 / groups)));
  evict_move_kernel<<<dim3(unsigned(wgs), unsigned(groups)), dim3(256), 0, s>>>(
      static_cast<piece_t*>(K), static_cast<piece_t*>(V), int(cap), row16, e.moves, keep, e.n_moves, lens, Hkv,
      lens_out);
  ESTP_CHECK_LAUNCH("evict_move_kernel");
  return ESTP_OK;
}
