// What the tile kernels share: blocks of 128 bytes of a row in LDS, brought there by
// direct loads, and the asm statements around their matrix instructions.
#pragma once

#include <atomic>
#include <type_traits>

#include "ws_fp8_common.hpp"

namespace wsg {

constexpr uint32_t kOutside = 0x80000000u;  // an offset past every buffer: reads zeros

template <int N, typename F>
__device__ __forceinline__ void static_for(const F& f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

#define WSG_LDS __attribute__((address_space(3)))

// Byte position, in a row of 128, of 16-byte chunk c of tile row r.  The operand
// read (lane l: row l % 16, chunk l / 16 or four more) is free of bank conflicts
// so; with (r ^ r / 8 % 2) % 8, which suits reads of 32 rows, it took twice as long
// (SQ_LDS_BANK_CONFLICT).  The choice depends on r % 16 only, which is fixed for
// a lane.
__device__ __forceinline__ int chunk_at(int r, int c) { return (c ^ (r & 7)) * 16; }

// A buffer descriptor as four scalars, for asm.
__device__ __forceinline__ i32x4_t raw_buffer(const uint8_t* base, uint32_t bytes) {
  const uint64_t at = (uint64_t)base;
  return i32x4_t{(int)__builtin_amdgcn_readfirstlane((uint32_t)at), (int)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)),
                 (int)__builtin_amdgcn_readfirstlane(bytes), 0x00027000};
}

// 64 lanes' 16 bytes from buffer offsets `at` + k straight to 1 KiB of LDS at
// `to` (zeros where `at` is outside).  As asm, so that the compiler does not wait
// for it before LDS reads of other addresses; whoever reads what it brings waits
// for vmcnt himself.  Nothing else in these kernels uses m0.
__device__ __forceinline__ void load_to_lds(i32x4_t r, uint32_t at, uint32_t k, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile(
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(at),
      "s"(r), "s"(__builtin_amdgcn_readfirstlane(k)), "s"(__builtin_amdgcn_readfirstlane(to)));
#endif
}

// Waits for this wave's LDS accesses and all but its last YOUNGER loads, then for
// the workgroup.
template <int YOUNGER = 0>
__device__ __forceinline__ void drain_and_meet() {
  static_assert(YOUNGER >= 0 && YOUNGER <= 63, "vmcnt");
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(YOUNGER) : "memory");
#endif
}

// Keeps what reads acc behind the asm statements before, the wait for the last
// products among them.
template <bool AGPR>
__device__ __forceinline__ void settle(f32x4_t& acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (AGPR) asm volatile("" : "+a"(acc));
  else asm volatile("" : "+v"(acc));
#endif
}

// -- host -------------------------------------------------------------------------

// Compute units of the current device, asked for once (256 where it does not say).
inline int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace wsg
