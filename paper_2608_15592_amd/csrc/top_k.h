// The k largest of many logits, ties to the lowest index, by a workgroup of 256 threads (logprobs.hip).
//
// Every thread's largest key is known first.  The k largest keys of all lie in the k threads whose own largest are the
// largest (if one lay in another, k threads would hold a larger one), so the k-th largest of the 256 maxima bounds them
// from below, and at most k times a thread's keys reach the bound; a few more than k, as a rule.
//
// A logit is ordered by one whole number, its key: the logit's bits made ascending, NaN below all, then the lowest index
// first.  No two keys are equal, so the order in which lists are filled changes nothing.
#pragma once

#include "estp_common.h"

namespace estp {
namespace detail {

constexpr int kMaxTop = 128;

// Ascending as the logits are, never 0.
__device__ __forceinline__ uint32_t ascending(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);  // (-0 is 0)
  return z != z ? 1u : u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t key_of(uint32_t up, int id) { return uint64_t(up) << 32 | uint32_t(~id); }
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t up = uint32_t(key >> 32);
  return up == 1u ? __uint_as_float(0x7fc00000u) : __uint_as_float(up & 0x80000000u ? up ^ 0x80000000u : ~up);
}
__device__ __forceinline__ int id_of(uint64_t key) { return int(~uint32_t(key)); }

// Key 0 is none.  kCap: keys of the list.
template <int kCap>
struct TopK {
  uint64_t list[kCap], maxima[256], bound;
  int count;

  // Keys of a wave's 256 that hold.
  template <typename Holds>
  __device__ static __forceinline__ int number(Holds&& holds) {
    int n = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) n += __popcll(__ballot(holds(u)));
    return n;
  }
  __device__ static __forceinline__ int enough(int k) { return min(k + 32, kMaxTop); }
  __device__ static __forceinline__ uint32_t top_of(const uint32_t (&hi)[4], int k, int* reach) {
    uint32_t top = 0;
    *reach = 256;
    for (uint32_t bit = 0x80000000u; bit && *reach > enough(k); bit >>= 1) {
      const uint32_t c = top | bit;
      const int n = number([&](int u) { return hi[u] >= c; });
      if (n >= k) {
        top = c;
        *reach = n;
      }
    }
    return top;
  }

  // A key that k of the threads' keys reach, and kMaxTop at most, or 1 where fewer than k threads have one.  One wave, four
  // keys a lane, forms it bit by bit, until few enough reach it, and what lies below the logit's bits only where equal
  // logits need it.
  __device__ __forceinline__ uint64_t bound_of(uint64_t mine, int k) {
    const int tid = threadIdx.x;
    maxima[tid] = mine;
    __syncthreads();
    if (tid < 64) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint64_t v = maxima[64 * u + tid];
        hi[u] = uint32_t(v >> 32);
        lo[u] = uint32_t(v);
      }
      uint32_t low = 0;
      int reach;
      const uint32_t top = top_of(hi, k, &reach);
      const int left = k - number([&](int u) { return hi[u] > top; });
      if (top && reach > enough(k))
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
          const uint32_t c = low | bit;
          if (number([&](int u) { return hi[u] == top && lo[u] >= c; }) >= left) low = c;
        }
      if (tid == 0) bound = top ? uint64_t(top) << 32 | low : 1;
    }
    __syncthreads();
    return bound;
  }
  // The same of the logits' bits alone: a logit that k of the threads' largest reach, and kMaxTop at most; a NaN where
  // equal, infinite or too few ones allow none.
  __device__ __forceinline__ float bound_of(uint32_t mine, int k) {
    const int tid = threadIdx.x;
    uint32_t* of = reinterpret_cast<uint32_t*>(maxima);
    of[tid] = mine;
    __syncthreads();
    if (tid < 64) {
      uint32_t hi[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) hi[u] = of[64 * u + tid];
      int reach;
      const uint32_t top = top_of(hi, k, &reach);
      constexpr uint32_t kLowest = 0x00800000u;  // of the largest negative number
      if (tid == 0) bound = reach > enough(k) || top < kLowest ? 1u : top;
    }
    __syncthreads();
    return logit_of(bound << 32);
  }

  // put(rank, key) by some thread for the k largest of the n keys listed, n <= kCap, the largest first.  All
  // threads call it, after a barrier; the list may be used again after one.
  template <typename Put>
  __device__ __forceinline__ void rank(int n, int k, Put&& put) {
    const int tid = threadIdx.x;
    while (n > 256) {  // (at most k of every n / 256 stay)
      constexpr int kE = (kCap + 255) / 256;
      uint64_t own[kE], mine = 0;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        own[e] = 256 * e + tid < n ? list[256 * e + tid] : 0;
        mine = own[e] > mine ? own[e] : mine;
      }
      const uint64_t from = bound_of(mine, k);
      if (tid == 0) count = 0;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < kE; ++e)
        if (own[e] >= from) list[atomicAdd(&count, 1)] = own[e];
      __syncthreads();
      n = count;
      __syncthreads();
    }
    if (tid < n) {
      const uint64_t own = list[tid];
      int r = 0;
#pragma unroll 4
      for (int t = 0; t < n; ++t) r += list[t] > own;
      if (r < k) put(r, own);
    }
  }
};

}  // namespace detail
}  // namespace estp
