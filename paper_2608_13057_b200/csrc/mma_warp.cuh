// MMA issue by a whole warp.  tcgen05.mma takes its operands from uniform registers: issued from a branch that one
// lane took, every descriptor word is first moved there (about 65 clocks per instruction measured); with the whole warp in
// the loop, waits decided by votes and the elected lane a predicate of the instruction, the loop's values are uniform to
// begin with.
#pragma once

#include "ffn_common.cuh"

namespace tempo {

__device__ __forceinline__ uint32_t elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r;
}
__device__ __forceinline__ int warp_uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// Bounded wait of a whole warp, the same answer in every lane (see mbar_wait).
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                               unsigned long long limit_ns) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  unsigned long long t0 = 0;
  for (uint32_t it = 0;; ++it) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((it & 63u) == 63u) {
      bool gone = *abort_flag != 0;
      const unsigned long long now = global_timer_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > limit_ns) gone = true;
      if (__any_sync(0xffffffffu, gone)) { *abort_flag = 1; return false; }
    }
  }
}

// Shared-memory descriptor of a K-major operand in the 128-byte swizzle (rows of 128 bytes, groups of 8 rows 1024 bytes
// apart): only its low word differs from tile to tile.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo_sw128(uint32_t addr) { return ((addr >> 4) & 0x3fffu) | (1u << 16); }

__device__ __forceinline__ void warp_mma_fp8(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                             uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, l;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 l, %8, 0;\n\t"
      "mov.b64 da, {%1, %7};\n\tmov.b64 db, {%2, %7};\n\t"
      "@l tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], da, db, %3, [%5], [%6], p;\n\t}"
      ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb), "r"(kDescHi), "r"(leader) : "memory");
}
__device__ __forceinline__ void warp_mma_bf16(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc,
                                              uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, l;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 l, %6, 0;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "@l tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
      ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"(leader) : "memory");
}
__device__ __forceinline__ void warp_cp_sf(uint32_t leader, uint32_t tmem_addr, uint32_t smem_addr) {
  const uint64_t desc = smem_desc_sf(smem_addr);
  asm volatile("{\n\t.reg .pred l;\n\tsetp.ne.b32 l, %2, 0;\n\t@l tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
               ::"r"(tmem_addr), "l"(desc), "r"(leader) : "memory");
}
__device__ __forceinline__ void warp_commit(uint32_t leader, uint32_t bar) {
  asm volatile("{\n\t.reg .pred l;\n\tsetp.ne.b32 l, %1, 0;\n\t"
               "@l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
               ::"r"(bar), "r"(leader) : "memory");
}

}  // namespace tempo
