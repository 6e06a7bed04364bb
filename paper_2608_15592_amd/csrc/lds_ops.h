// gfx950 matrix-core step, transposing LDS reads and transfers into LDS, shared by the LM-head gradient and the
// attention over a cache.
#pragma once

#include "estp_common.h"

namespace estp {
namespace detail {

__device__ __forceinline__ f32x4_t mfma_bf16(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Two numbers rounded to bf16, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2_t{__bf16(lo), __bf16(hi)});
}
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

// Lane s of a 16-lane group reads 4 elements at `p`; lane i gets element i % 4 of lanes i / 4, 4 + i / 4, 8 + i / 4
// and 12 + i / 4.
__device__ __forceinline__ s16x4_t read_tr(const char* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(p));
#else
  return s16x4_t{};
#endif
}

// lds_dma16_buf as one instruction that the compiler counts no wait for: before every transposing read it would wait
// for all transfers in flight (vmcnt 0), which the kernels here order by themselves.  There is no register result
// to wait for.  The resource is make_rsrc's, as the four words it is.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4_t rsrc_words(const void* base, uint32_t bytes) {
  const uint64_t a = uint64_t(base);
  return u32x4_t{uint32_t(a), uint32_t(a >> 32) & 0xffffu, bytes, 0x00020000u};
}
template <bool kStream = false>
__device__ __forceinline__ void dma16(u32x4_t r, uint32_t voffset, uint32_t soffset, char* dst_wave_base) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t m0 = uint32_t(uintptr_t((__attribute__((address_space(3))) char*)(dst_wave_base)));
  if constexpr (kStream)  // non-temporal: a line used once
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, %3 offen nt lds"
        :
        : "s"(m0), "v"(voffset), "s"(r), "s"(soffset)
        : "memory", "m0");
  else
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, %3 offen lds"
        :
        : "s"(m0), "v"(voffset), "s"(r), "s"(soffset)
        : "memory", "m0");
#endif
}

__device__ __forceinline__ bf16x8_t join_tr(s16x4_t lo, s16x4_t hi) {
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Inclusive prefix sum over the wave, without LDS: shifts within rows of 16 lanes, then the rows' last lanes.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
  x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x111, 0xf, 0xf, false));  // row_shr 1, 2, 4, 8
  x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x112, 0xf, 0xf, false));
  x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x114, 0xf, 0xf, false));
  x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x118, 0xf, 0xf, false));
  x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x142, 0xa, 0xf, false));  // row_bcast 15 into rows 1 and 3
  x += uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x143, 0xc, 0xf, false));  // row_bcast 31 into rows 2 and 3
#endif
  return x;
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) {
  return uint32_t(__builtin_amdgcn_readlane(int(v), lane));
}

// At most N of this wave's vector-memory operations still in flight; LDS reads after it stay after it.
template <int N>
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_sched_barrier(0);
  wait_vm<N>();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_sched_barrier(0);
}
// This wave's LDS reads are done: what they read may be overwritten.
__device__ __forceinline__ void lds_read_done() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_sched_barrier(0);
}

}  // namespace detail
}  // namespace estp
