// The 4-bit paged cache: where a token's codes and scales lie, and how codes become fp16 values (see tempo.h).
#pragma once

#include <cuda_fp16.h>

#include "tempo_kernels.cuh"

namespace tempo {

constexpr int kUnit = 16;          // tokens of a unit, the smallest piece of the cache that is contiguous for a head
constexpr int kGroup = 32;         // elements that share a scale and a zero point
constexpr uint32_t kMarked = 0xff; // scale byte of a marked token: read as fp16 it is NaN

template <int D>
struct CacheUnit {
  static constexpr int kCodes = kUnit * D / 2, kParams = kUnit * D / 16, kBytes = kCodes + kParams;
  static constexpr int kKeyRow = D / 2, kKeyParams = D / 16;      // of a token
  static constexpr int kPairRow = D, kPairParams = D / 8;         // of two tokens' values
};

// First byte of the unit that holds token `at` of a page.  kv: 0 keys, 1 values.
template <int D>
__host__ __device__ __forceinline__ size_t unit_offset(int64_t page, int head, int kv, int at, int Hkv, int page_size) {
  return ((static_cast<size_t>(page) * Hkv + head) * 2 + kv) * (static_cast<size_t>(page_size / kUnit) * CacheUnit<D>::kBytes) +
         static_cast<size_t>(at / kUnit) * CacheUnit<D>::kBytes;
}

__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t as_u32(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }

// Two groups' (s, 16 z) byte pairs in the halves of p: s and -s (64 + z) as fp16, both exact (4 and 11 significant bits).
__device__ __forceinline__ void group_params(uint32_t p, uint32_t& s, uint32_t& b) {
  s = (p & 0x00ff00ffu) << 7;
  b = as_u32(__hmul2(as_half2(s), as_half2(((p >> 8) & 0x00f000f0u) | 0xd400d400u)));
}

// The byte pairs of two tokens' values, `left` of which (and more behind them) exist: what lies in the others may be anything.  Nor
// need a token that exists have been written: a scale is at most 768, which is the most that the append stores, since an infinite one or a
// NaN would reach the rows that do not see the token as 0 * NaN.
__device__ __forceinline__ uint32_t edge_params(uint32_t p, int left) {
  p = (p & 0xff00ff00u) | __vminu2(p & 0x00ff00ffu, 0x00c400c4u);
  return left >= 2 ? p : left == 1 ? p & 0xffffu : 0u;
}

// (v & mask) | bits in one instruction: with both as immediates it would be two, and logic is what bounds the decoding.
__device__ __forceinline__ uint32_t and_or(uint32_t v, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(v), "r"(mask), "r"(bits));
  return r;
}

// The constants of decode8, in registers for a whole loop (the compiler cannot see that they are constants).
struct Decode {
  uint32_t low, high, m1024, m64, down;
  __device__ __forceinline__ Decode() {
    asm volatile("mov.b32 %0, 0x000f000f;\n\tmov.b32 %1, 0x00f000f0;\n\tmov.b32 %2, 0x64006400;\n\tmov.b32 %3, 0x54005400;\n\tmov.b32 %4, 0xe380e380;"
                 : "=r"(low), "=r"(high), "=r"(m1024), "=r"(m64), "=r"(down));   // down: -960 twice
  }
};

// A word of eight codes -> four pairs, pair n of the codes n and n + 4 (bits 4n and 4n + 16).  A code in bits 4 to 7 under the
// exponent of 64 is the fp16 number 64 + c, one in bits 0 to 3 under the exponent of 1024 is 1024 + c and one exact sum from
// 64 + c; one fused step takes that to s (64 + c) - s (64 + z) = s (c - z), which has 8 significant bits: nothing is rounded.
// 11 instructions for 8 elements, 5 of them on the pipe of logic and shifts, which has half the rate of the other one.
__device__ __forceinline__ void decode8(const Decode& k, uint32_t w, uint32_t s, uint32_t b, uint32_t (&v)[4]) {
  const uint32_t t = w >> 8;
  v[1] = as_u32(__hfma2(as_half2(and_or(w, k.high, k.m64)), as_half2(s), as_half2(b)));
  v[3] = as_u32(__hfma2(as_half2(and_or(t, k.high, k.m64)), as_half2(s), as_half2(b)));
  v[0] = as_u32(__hfma2(__hadd2(as_half2(and_or(w, k.low, k.m1024)), as_half2(k.down)), as_half2(s), as_half2(b)));
  v[2] = as_u32(__hfma2(__hadd2(as_half2(and_or(t, k.low, k.m1024)), as_half2(k.down)), as_half2(s), as_half2(b)));
}

}  // namespace tempo
