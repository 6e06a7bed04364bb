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
// evict_select_kernel, one workgroup per (sequence, KV head), a thread per every 1024th slot: the weights'
// order-preserving 32-bit keys stay in registers (caches of up to 65536 slots; longer ones are read again on each
// pass).  Four histogram passes of 8 bits in LDS find the key of the last one kept.  Places in slot order (of ties,
// holes and survivors) come from ballots: a count per 64 slots, one prefix over all counts.  The survivors' rows move
// in the same kernel where its workgroups fill the chip or there is little to move, else in evict_move_kernel.
// Everything is exact: whole numbers and copies.
#include <algorithm>

#include "estp_common.h"

namespace estp {
namespace detail {

typedef uint32_t piece_t __attribute__((ext_vector_type(4)));  // 16 bytes of a row
constexpr int kEThreads = 1024;
constexpr int kEWaves = kEThreads / 64;

// Weights as whole numbers in the same order: NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float v) {
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u & 0x7fffffffu) == 0) return 0x80000000u;
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// Exclusive prefix of a thread's pair of counts over the workgroup (every thread calls), in the halves of 64 bits.
__device__ __forceinline__ uint64_t block_prefix(uint64_t v, uint64_t* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) sh[wave] = x;
  __syncthreads();
  uint64_t before = x - v;
#pragma unroll
  for (int w = 0; w < kEWaves; ++w) before += w < wave ? sh[w] : 0;
  return before;
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
                                          const int2* __restrict__ moves, int n, int64_t first, int64_t step) {
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
  constexpr int kHists = 4;  // copies of the histogram: equal weights meet on fewer threads
  constexpr int kSpan = kE > 0 ? kE : 64;  // rounds whose counts one prefix covers
  __shared__ int hist[kHists][256];
  __shared__ uint32_t found[2];
  __shared__ int n_guarded_sh;
  __shared__ uint64_t wave_sum_sh[kEWaves], counts[kSpan * kEWaves], carry;
  const int bg = blockIdx.x, b = bg / g.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t base = size_t(bg) * g.cap;
  const int n = max(0, min(g.lens[b], g.cap)), keep = g.keep;
  const float* acc = g.acc + base;
  const int* pos = g.pos + base;
  float* acc_out = g.acc_out + base;
  int* pos_out = g.pos_out + base;
  int* idx = g.idx + size_t(bg) * keep;
  int2* moves = g.moves + size_t(bg) * keep;
  const bool copy = acc_out != acc || pos_out != pos;
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
  const int64_t first_recent = int64_t(g.seen[b]) - g.recent;
  auto is_guarded = [&](int i) { return pos[i] < g.sink || pos[i] >= first_recent; };
  const int rounds = kE > 0 ? kE : (n + kEThreads - 1) / kEThreads;

  uint32_t key[kE > 0 ? kE : 1];
  uint64_t guard = 0;
  if (tid == 0) n_guarded_sh = 0;
  for (int i = tid; i < kHists * 256; i += kEThreads) (&hist[0][0])[i] = 0;
  __syncthreads();
  int mine = 0;
  if constexpr (kE > 0) {
#pragma unroll
    for (int r = 0; r < kE; ++r) {
      const int i = r * kEThreads + tid;
      key[r] = i < n ? weight_key(acc[i]) : 0;
      const bool gd = i < n && is_guarded(i);
      guard |= uint64_t(gd) << r;
      mine += gd;
    }
  } else {
    for (int i = tid; i < n; i += kEThreads) mine += is_guarded(i);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
  if (lane == 0 && mine) atomicAdd(&n_guarded_sh, mine);
  __syncthreads();
  // guarded slots: all stay if they fit, else the best of them do and nothing else
  const int n_guarded = n_guarded_sh;
  const bool among = n_guarded >= keep;  // whether the choice is among the guarded slots
  uint32_t need = uint32_t(among ? keep : keep - n_guarded);
  // Round r's slot of this thread: its key, and whether it is in the choice.
  auto at = [&](int r, uint32_t* k, bool* in, bool* gd) {
    const int i = r * kEThreads + tid;
    *in = i < n;
    if constexpr (kE > 0) {
      *k = key[r];
      *gd = (guard >> r) & 1;
    } else {
      *k = *in ? weight_key(acc[i]) : 0;
      *gd = *in && is_guarded(i);
    }
  };
  auto each_round = [&](auto&& f) {
    if constexpr (kE > 0) {
#pragma unroll
      for (int r = 0; r < kE; ++r) f(r);
    } else {
      for (int r = 0; r < rounds; ++r) f(r);
    }
  };
  // the key of the need-th best candidate, 8 bits at a time; `need` becomes how many of its equals stay
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    each_round([&](int r) {
      uint32_t k;
      bool in, gd;
      at(r, &k, &in, &gd);
      if (in && gd == among && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
        atomicAdd(&hist[wave % kHists][(k >> shift) & 255], 1);
    });
    __syncthreads();
    if (wave == 0) {  // lane j: bins 255 - 4 j down to 252 - 4 j; the first lane whose running count reaches `need`
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        c[q] = 0;
#pragma unroll
        for (int h = 0; h < kHists; ++h) {
          c[q] += uint32_t(hist[h][255 - 4 * lane - q]);
          hist[h][255 - 4 * lane - q] = 0;
        }
        sum += c[q];
      }
      uint32_t x = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
      }
      const uint64_t reached = __ballot(x >= need);
      if (reached && lane == __builtin_ctzll(reached)) {
        uint32_t above = x - sum;
        int q = 0;
        while (q < 3 && above + c[q] < need) above += c[q++];
        found[0] = uint32_t(255 - 4 * lane - q);
        found[1] = need - above;
      }
    }
    __syncthreads();
    prefix |= found[0] << shift;
    need = found[1];
  }

  // Places in slot order: pass 0 counts ties and sees which of them stay, pass 1 counts holes (low half) and
  // survivors (high half) and lists them.  Per span of rounds: a count for every 64 slots, one prefix, the lanes' own.
  uint64_t stays = 0;  // kE > 0: a bit a round
  int ties_before = 0;
  uint64_t moved_before = 0;
  auto span = [&](int r0, auto&& flags) {  // flags(r, &low, &high): exclusive counts before the thread's slot
    const int nr = min(kSpan, rounds - r0);
    for (int r = r0; r < r0 + nr; ++r) {
      bool lo, hi;
      flags(r, &lo, &hi);
      const uint64_t bl = __ballot(lo), bh = __ballot(hi);
      if (lane == 0) counts[(r - r0) * kEWaves + wave] = uint64_t(__popcll(bl)) | uint64_t(__popcll(bh)) << 32;
    }
    __syncthreads();
    const uint64_t c = tid < nr * kEWaves ? counts[tid] : 0;
    const uint64_t before = block_prefix(c, wave_sum_sh);
    if (tid < nr * kEWaves) counts[tid] = before;
    if (tid == nr * kEWaves - 1) carry = before + c;
    __syncthreads();
  };
  auto below = [&](bool x) { return uint32_t(__popcll(__ballot(x) & ((uint64_t(1) << lane) - 1))); };
  auto stays_at = [&](int r, uint32_t tie_rank, bool* in_out) {
    uint32_t k;
    bool in, gd;
    at(r, &k, &in, &gd);
    *in_out = in;
    return in && ((gd && !among) || (gd == among && (k > prefix || (k == prefix && tie_rank < need))));
  };
  auto is_tie = [&](int r) {
    uint32_t k;
    bool in, gd;
    at(r, &k, &in, &gd);
    return in && gd == among && k == prefix;
  };
  for (int r0 = 0; r0 < rounds; r0 += kSpan) {
    const int r1 = min(rounds, r0 + kSpan);
    span(r0, [&](int r, bool* lo, bool* hi) {
      *lo = is_tie(r);
      *hi = false;
    });
    uint64_t bits = 0;  // of this span: stays
    for (int r = r0; r < r1; ++r) {
      const uint32_t rank = uint32_t(ties_before) + uint32_t(counts[(r - r0) * kEWaves + wave]) + below(is_tie(r));
      bool in;
      bits |= uint64_t(stays_at(r, rank, &in)) << (r - r0);
    }
    ties_before += int(uint32_t(carry));
    stays = bits;
    __syncthreads();  // counts and carry are read
    span(r0, [&](int r, bool* lo, bool* hi) {
      const int i = r * kEThreads + tid;
      const bool st = (stays >> (r - r0)) & 1;
      *lo = i < n && i < keep && !st;
      *hi = st && i >= keep;
    });
    for (int r = r0; r < r1; ++r) {
      const int i = r * kEThreads + tid;
      const bool st = (stays >> (r - r0)) & 1, hole = i < n && i < keep && !st, late = st && i >= keep;
      const uint64_t c = moved_before + counts[(r - r0) * kEWaves + wave];
      const uint32_t h = uint32_t(c) + below(hole), l = uint32_t(c >> 32) + below(late);
      if (hole) moves[h].y = i;
      if (late) moves[l].x = i;
      if (st && i < keep) {
        idx[i] = i;
        if (copy) {
          acc_out[i] = acc[i];
          pos_out[i] = pos[i];
        }
      }
    }
    moved_before += carry;
    __syncthreads();  // counts and carry are read, and the moves of this span written
  }
  const int holes = int(uint32_t(moved_before));  // as many as survivors
  for (int m = tid; m < holes; m += kEThreads) {
    const int2 e = moves[m];
    idx[e.y] = e.x;
    acc_out[e.y] = acc[e.x];
    pos_out[e.y] = pos[e.x];
  }
  __syncthreads();  // freed slots are cleared after the moves have read them
  for (int i = keep + tid; i < n; i += kEThreads) {
    acc_out[i] = 0.f;
    pos_out[i] = -1;
  }
  if (tid == 0) g.n_moves[bg] = holes;
  if (g.K) move_rows(g.K, g.V, base, g.row16, moves, holes, tid, kEThreads);
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
  const int row16 = dh * (dtype == ESTP_F32 ? 4 : 2) / 16;
  const int64_t most = std::min<int64_t>(keep, cap - keep) * row16;  // 16-byte pieces that can move, of K or V
  // Rows move in the selecting kernel where there are few: a kernel of their own costs its launch, but spreads the
  // rows of the longest sequences over the chip.  Not in place of lens, which workgroups of the same sequence still
  // read.
  const bool here = most <= 1024 && lens_out != lens;
  EvictArgs g{acc, pos, lens, seen, Hkv, int(cap), keep, recent, sink, acc_out, pos_out, idx, e.moves, e.n_moves,
              here ? static_cast<piece_t*>(K) : nullptr, static_cast<piece_t*>(V), row16, lens_out};
  auto select = cap <= kEThreads        ? evict_select_kernel<1>
                : cap <= 4 * kEThreads  ? evict_select_kernel<4>
                : cap <= 16 * kEThreads ? evict_select_kernel<16>
                : cap <= 64 * kEThreads ? evict_select_kernel<64>
                                        : evict_select_kernel<0>;
  select<<<dim3(unsigned(groups)), dim3(kEThreads), 0, s>>>(g);
  ESTP_CHECK_LAUNCH("evict_select_kernel");
  if (here) return ESTP_OK;
  const int64_t wgs = std::max<int64_t>(1, std::min<int64_t>((most + 255) / 256, std::max(1, 4096 / groups)));
  evict_move_kernel<<<dim3(unsigned(wgs), unsigned(groups)), dim3(256), 0, s>>>(
      static_cast<piece_t*>(K), static_cast<piece_t*>(V), int(cap), row16, e.moves, keep, e.n_moves, lens, Hkv, lens_out);
  ESTP_CHECK_LAUNCH("evict_move_kernel");
  return ESTP_OK;
}
