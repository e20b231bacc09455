// The layout of the paged 8-bit cache, shared by the kernels that fill it and the attention that reads it.
//
// uint8 [pages][heads][page / 16][32 D + 64]: sixteen consecutive tokens of a head, whose keys share a factor and whose
// values share one (fp32, 0 where all were zero).  A byte holds its code plus 128.
//   0          key codes    [token / 4][chunk < D / 64][j < 4][token % 4][16 bytes]   channels 64 chunk + 16 j + byte;
//                           behind the chunks of an odd D / 32 [j < 4][token % 4][8 bytes], channels D - 32 + 8 j + byte
//   16 D       value codes  [channel][token]
//   32 D       the keys' factor, the values' factor, 8 bytes free
//   32 D + 16  in head 0: 3 bytes for each token, the number in the last call that wrote to it (below)
// Lane (r, j) of a wavefront that multiplies the keys of four sixteens reads, for four tokens of each, 16 bytes of token
// r % 4 of sixteen r / 4: 16 lanes have 64 neighbouring bytes of each.  The one that multiplies values reads the 16 tokens
// of a channel: 16 lanes have 256 neighbouring bytes.
#pragma once
#include "q8_kv4.h"

namespace q8 {

constexpr int kv8_sixteen(int D) { return 32 * D + 64; }

// Where the code of channel c (a multiple of 8; the next 7 lie behind it) of token t's key lies.
__device__ __forceinline__ int kv8_key(int D, int t, int c) {
  const int row = (t >> 2) * 4 * D, chunk = c >> 6;
  if (chunk < D >> 6) return row + chunk * 256 + ((c >> 4 & 3) * 4 + (t & 3)) * 16 + (c & 15);
  return row + chunk * 256 + ((c >> 3 & 3) * 4 + (t & 3)) * 8;
}

}  // namespace q8
