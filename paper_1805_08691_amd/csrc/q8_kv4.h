// The layout of the paged 4-bit cache, shared by the kernels that fill it and the attention that reads it.
//
// uint8 [pages][heads][page / 16][18 D]: sixteen consecutive tokens of a head are 576 G bytes, G = D / 32:
//   0      key codes      [token][j < 4][g < G][4 bytes]   byte b: channels 32 g + 8 j + 2 b (low half) and the next
//   256 G  value codes    [g < G][r < 16][token]           channels 32 g + r (low half) and 32 g + 16 + r
//   512 G  key factors    [token][g < G]                   binary16
//   544 G  value factors  [g < G][place of the token]      binary16; in each four tokens the order is 0, 2, 1, 3
// A half byte holds its code plus 8.  Lane (r, j) of a wavefront that multiplies 16 tokens' keys reads 4 G bytes of
// token r, the 8 channels that it stands for in each of the G groups; the one that multiplies values reads the 16
// tokens of its channel pair, and their factors in the order in which a pair of half bytes unpacks.
#pragma once
#include "q8_value.h"

namespace q8 {

constexpr int kMaxHead = 256;

inline bool kv4_page_ok(int page) { return page >= 16 && page <= (1 << 20) && (page & (page - 1)) == 0; }
inline bool kv4_shape_ok(int D, int page) { return D >= 32 && D <= kMaxHead && D % 32 == 0 && kv4_page_ok(page); }

// Where the value factor of token t of a sixteen lies.
__device__ __forceinline__ int kv4_place(int t) { return (t & ~3) | (t & 1) << 1 | (t & 2) >> 1; }

// The factor of a group whose largest finite magnitude is m: m * fl(1/7) in binary16, at most 8188 (8 * 8188 is
// binary16's largest value: whatever the cache holds is a binary16 number's size); 1 where that is 0.
__device__ __forceinline__ _Float16 kv4_factor(float m) {
  const _Float16 q = (_Float16)fminf(__fmul_rn(m, 1.0f / 7.0f), 8188.0f);
  return q == (_Float16)0.0f ? (_Float16)1.0f : q;
}

template <typename V>
inline bool kv4_rows_aligned(const void* k, const void* v, size_t k_stride, size_t k_head, size_t v_stride,
                             size_t v_head) {
  return q8_aligned(k, 16) && q8_aligned(v, 16) && ((k_stride | k_head | v_stride | v_head) * sizeof(V)) % 16 == 0;
}

}  // namespace q8
