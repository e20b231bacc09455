// Shared by the kernels of attention over the paged 4-bit cache: the unpacking of codes, and the launch for many columns.
#pragma once
#include "q8_attend.h"
#pragma clang fp contract(fast)

namespace q8 {

namespace {

// Half bytes u as binary16: the low ones of w's bytes 0 and 2 as 1024 + u, the high ones as 1024 + 16 u, one instruction
// for two (mask and pattern in registers: one instruction takes them, not two literals).
struct Unpack {
  unsigned low_mask = 0x000f000fu, high_mask = 0x00f000f0u, one = 0x64006400u;
  __device__ __forceinline__ Unpack() { asm volatile("" : "+s"(low_mask), "+s"(high_mask), "+v"(one)); }
  __device__ __forceinline__ h2 low(unsigned w) const { return __builtin_bit_cast(h2, (w & low_mask) | one); }
  __device__ __forceinline__ h2 high(unsigned w) const { return __builtin_bit_cast(h2, (w & high_mask) | one); }
};
}  // namespace

// The launch for many columns (q8_kv4_wide.hip); p.tiles: of kWideCols columns.
int kv4_attend_wide(int G, const AttendParams& p, const void* q, void* out, int type, hipStream_t stream);

}  // namespace q8
