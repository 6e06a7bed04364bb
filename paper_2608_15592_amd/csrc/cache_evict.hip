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
// evict_select_kernel, one workgroup per (sequence, KV head): the weights'
// order-preserving 32-bit keys are cut to the threshold of the last one kept
// by four histogram passes of 8 bits (LDS), then one pass in slot order counts
// ties, holes and survivors and lists the moves.  evict_move_kernel copies the
// listed rows.  Everything is exact: whole numbers and copies.
#include <algorithm>

#include "estp_common.h"

namespace estp {
namespace detail {

constexpr int kEThreads = 1024;
constexpr int kEWaves = kEThreads / 64;

// Weights as whole numbers in the same order: NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float v) {
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u & 0x7fffffffu) == 0) return 0x80000000u;
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// Exclusive prefix of `v` over the workgroup (every thread calls), and its total.
struct Scan {
  int before, total;
};
__device__ __forceinline__ Scan block_scan(int v, int* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();  // the previous scan's totals are read
  if (lane == 63) sh[wave] = x;
  __syncthreads();
  Scan r{x - v, 0};
#pragma unroll
  for (int w = 0; w < kEWaves; ++w) {
    r.before += w < wave ? sh[w] : 0;
    r.total += sh[w];
  }
  return r;
}

__global__ __launch_bounds__(kEThreads) void evict_select_kernel(
    const float* __restrict__ acc, const int* __restrict__ pos, const int* __restrict__ lens,
    const int* __restrict__ seen, int Hkv, int cap, int keep, int recent, int sink, float* acc_out, int* pos_out,
    int* __restrict__ idx, int2* __restrict__ moves, int* __restrict__ n_moves) {
  __shared__ int hist[256], sh[kEWaves], found[2];
  const int bg = blockIdx.x, b = bg / Hkv, tid = threadIdx.x;
  const size_t base = size_t(bg) * cap;
  const int n = max(0, min(lens[b], cap));
  acc += base;
  pos += base;
  acc_out += base;
  pos_out += base;
  idx += size_t(bg) * keep;
  moves += size_t(bg) * keep;
  if (n <= keep) {  // everything stays
    for (int i = tid; i < keep; i += kEThreads) idx[i] = i < n ? i : -1;
    for (int i = tid; i < n; i += kEThreads) {
      acc_out[i] = acc[i];
      pos_out[i] = pos[i];
    }
    if (tid == 0) n_moves[bg] = 0;
    return;
  }
  const int64_t first_recent = int64_t(seen[b]) - recent;
  auto guarded = [&](int i) { return pos[i] < sink || pos[i] >= first_recent; };
  // guarded slots: all stay if they fit, else the best of them do and nothing else
  int mine = 0;
  for (int i = tid; i < n; i += kEThreads) mine += guarded(i);
  const int n_guarded = block_scan(mine, sh).total;
  const bool among = n_guarded >= keep;  // whether the choice is among the guarded slots
  int need = among ? keep : keep - n_guarded;
  // the key of the need-th best candidate, 8 bits at a time; `need` becomes how many of its equals stay
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kEThreads) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kEThreads) {
      const uint32_t k = weight_key(acc[i]);
      if (guarded(i) == among && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))))
        atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int above = 0, d = 255;
      while (d > 0 && above + hist[d] < need) above += hist[d--];
      found[0] = d;
      found[1] = need - above;
    }
    __syncthreads();
    prefix |= uint32_t(found[0]) << shift;
    need = found[1];
  }
  // in slot order: which slots stay, and the moves
  int ties = 0, holes = 0, late = 0;
  for (int at = 0; at < n; at += kEThreads) {
    const int i = at + tid;
    const bool in = i < n;
    const bool gd = in && guarded(i);
    const uint32_t k = in ? weight_key(acc[i]) : 0;
    const bool tie = in && gd == among && k == prefix;
    const Scan st = block_scan(tie, sh);
    const bool stays = in && ((gd && !among) || (gd == among && k > prefix) || (tie && ties + st.before < need));
    ties += st.total;
    const Scan sl = block_scan(stays && i >= keep, sh);
    const Scan so = block_scan(in && !stays && i < keep, sh);
    if (in && i < keep) {
      if (stays)
        idx[i] = i;
      else
        moves[holes + so.before].y = i;
    } else if (stays) {
      moves[late + sl.before].x = i;
    }
    holes += so.total;
    late += sl.total;
  }
  __syncthreads();  // the list is complete (holes == late), and acc and pos are read no more but where they stay
  for (int m = tid; m < holes; m += kEThreads) {
    const int2 e = moves[m];
    idx[e.y] = e.x;
    acc_out[e.y] = acc[e.x];
    pos_out[e.y] = pos[e.x];
  }
  if (acc_out != acc || pos_out != pos) {
    __syncthreads();  // idx is complete
    for (int i = tid; i < keep; i += kEThreads) {
      if (idx[i] != i) continue;
      acc_out[i] = acc[i];
      pos_out[i] = pos[i];
    }
  }
  __syncthreads();  // freed slots are cleared after the moves have read them
  for (int i = keep + tid; i < n; i += kEThreads) {
    acc_out[i] = 0.f;
    pos_out[i] = -1;
  }
  if (tid == 0) n_moves[bg] = holes;
}

// Rows of 16-byte pieces: destination moves[m].y, source moves[m].x, of K and of V.  Also writes lens_out, which may
// be lens: by now evict_select_kernel has read it.
__global__ __launch_bounds__(256) void evict_move_kernel(uint4* __restrict__ K, uint4* __restrict__ V, int cap,
                                                         int row16, const int2* __restrict__ moves, int keep,
                                                         const int* __restrict__ n_moves, const int* lens, int Hkv,
                                                         int* lens_out) {
  const int bg = blockIdx.y, n = n_moves[bg];
  if (blockIdx.x == 0 && threadIdx.x == 0 && bg % Hkv == 0) lens_out[bg / Hkv] = min(max(lens[bg / Hkv], 0), keep);
  const size_t base = size_t(bg) * cap;
  moves += size_t(bg) * keep;
  const int64_t total = int64_t(n) * row16;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
    const int2 e = moves[i / row16];
    const int c = int(i % row16);
    K[(base + e.y) * row16 + c] = K[(base + e.x) * row16 + c];
    V[(base + e.y) * row16 + c] = V[(base + e.x) * row16 + c];
  }
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
  evict_select_kernel<<<dim3(unsigned(groups)), dim3(kEThreads), 0, s>>>(acc, pos, lens, seen, Hkv, int(cap), keep,
                                                                         recent, sink, acc_out, pos_out, idx, e.moves,
                                                                         e.n_moves);
  ESTP_CHECK_LAUNCH("evict_select_kernel");
  const int row16 = dh * (dtype == ESTP_F32 ? 4 : 2) / 16;
  const int64_t most = std::min<int64_t>(keep, cap - keep) * row16;
  const int64_t wgs = std::max<int64_t>(1, std::min<int64_t>((most + 255) / 256, std::max(1, 4096 / groups)));
  evict_move_kernel<<<dim3(unsigned(wgs), unsigned(groups)), dim3(256), 0, s>>>(
      static_cast<uint4*>(K), static_cast<uint4*>(V), int(cap), row16, e.moves, keep, e.n_moves, lens, Hkv, lens_out);
  ESTP_CHECK_LAUNCH("evict_move_kernel");
  return ESTP_OK;
}
