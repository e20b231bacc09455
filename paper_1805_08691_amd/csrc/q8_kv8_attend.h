// Shared by the kernels of attention over the paged 8-bit cache: the unpacking of codes, factors' logarithms, and the launch
// for many columns.
#pragma once
#include "q8_attend.h"
#include "q8_kv8.h"
#pragma clang fp contract(fast)

namespace q8 {

namespace {

// Bytes u as binary16 1024 + u (u is the low byte of its bit pattern), less 1152: the codes, exactly, two to an instruction.
struct Codes {
  unsigned pattern = 0x64646464u;
  __device__ __forceinline__ Codes() { asm volatile("" : "+s"(pattern)); }
  __device__ __forceinline__ h2 two(unsigned w, unsigned order) const {
    constexpr _Float16 kMore = 1152.0f16;
    return __builtin_bit_cast(h2, __builtin_amdgcn_perm(pattern, w, order)) - h2{kMore, kMore};
  }
  __device__ __forceinline__ h8 eight(unsigned a, unsigned b) const {
    const h2 x[4] = {two(a, 0x04010400u), two(a, 0x04030402u), two(b, 0x04010400u), two(b, 0x04030402u)};
    return h8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
  }
};

// The first of the eight channels that lane j has in product g of a key: 16 neighbours in two products, 8 in the last of an
// odd number (q8_kv8.h).
template <int G>
__device__ __forceinline__ constexpr int key_channel(int g, int j) {
  return g < G / 2 * 2 ? g / 2 * 64 + 16 * j + 8 * (g & 1) : 32 * g + 8 * j;
}

// The logarithm of a values' factor, and a number below all of them for 0.
__device__ __forceinline__ float log2_of(float f) { return fmaxf(__builtin_log2f(f), -200.0f); }

}  // namespace

// The launch for many columns (q8_kv8_wide.hip); p.tiles: of kWideCols columns.
int kv8_attend_wide(int G, const AttendParams& p, const void* q, void* out, int type, hipStream_t stream);

}  // namespace q8
