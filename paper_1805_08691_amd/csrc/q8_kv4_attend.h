// Shared by the kernels of attention over the paged 4-bit cache: what a launch and a tile are, the unpacking of codes.
#pragma once
#include "q8_conv_common.h"
#include "q8_kv4.h"
#include <type_traits>
#pragma clang fp contract(fast)

namespace q8 {

struct AttendParams {
  const uint8_t* __restrict__ cache;
  const int* __restrict__ table;
  const int* __restrict__ lengths;
  const int* __restrict__ starts;      // null: request b is row b
  float* __restrict__ parts;           // workspace of the split, null: none is split
  int* __restrict__ counters;          // of the parts of a cut tile and head that are done; zero between calls
  size_t q_stride, q_head, o_stride, o_head, table_stride;
  long n_pages;
  int T, B, H, ratio, width, shift;    // shift: page = 16 << shift tokens
  int tiles, window;
  float scale_log2;                    // scale * log2(e)
};

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 64;              // keys of a wavefront's step
constexpr int kWaves = 4;
constexpr int kCols = 16;              // columns of an MFMA tile

// What a workgroup works on: COLS columns of request b, whose row 0 is q row `row`.
struct Tile {
  int b, row, first, cols, len, n;     // first column, columns of the request, keys, new tokens
  int seen, lo, steps;                 // first key that a row sees, that key's step's first one, and steps of kStep keys
};

// Request i's tiles begin at floor(starts[i] ratio / COLS) + i: none overlap, and those behind its last are empty.
__device__ __forceinline__ int request_start(const AttendParams& p, int i) { return min(max(p.starts[i], 0), p.T); }
template <int COLS>
__device__ __forceinline__ int first_tile(const AttendParams& p, int start, int i) {
  return (int)((long)start * p.ratio / COLS) + i;
}

// Tile w, of request b whose tiles begin at `base`, whose rows are row .. next - 1 and whose keys are `length`.
template <int COLS>
__device__ __forceinline__ bool set_tile(const AttendParams& p, int w, int b, int base, int row, int next, int length, Tile* t) {
  t->b = b;
  t->row = row;
  t->n = next - row;
  t->first = (w - base) * COLS;
  t->cols = t->n * p.ratio;
  if (t->first < 0 || t->first >= t->cols) return false;
  const long longest = (long)p.width << (p.shift + 4);
  t->len = (int)min((long)max(length, 0), longest);
  const int tok0 = t->first / p.ratio, tok1 = (min(t->first + COLS, t->cols) - 1) / p.ratio;
  const int pos0 = t->len - t->n + tok0, pos1 = t->len - t->n + tok1;
  t->seen = p.window > 0 ? max(0, pos0 - p.window + 1) : 0;
  t->lo = t->seen & ~(kStep - 1);
  t->steps = pos1 < t->lo ? 0 : (pos1 - t->lo) / kStep + 1;
  return true;
}

// Tile w, which a whole wavefront looks for: 64 requests at a time, one trip to memory for most launches.
template <int COLS>
__device__ __forceinline__ bool find_tile(const AttendParams& p, int w, Tile* t) {
  if (!p.starts) {
    const int per = (p.ratio + COLS - 1) / COLS, b = w / per;
    return b < p.B && set_tile<COLS>(p, w, b, b * per, b, b + 1, p.lengths[b], t);
  }
  int lo = 0, hi = p.B - 1;
  while (hi - lo >= 64) {
    const int mid = (lo + hi + 1) >> 1;
    if (first_tile<COLS>(p, request_start(p, mid), mid) <= w) lo = mid; else hi = mid - 1;
  }
  const int lane = threadIdx.x & 63, i = min(lo + lane, hi);
  const int row = request_start(p, i), next = request_start(p, i + 1), length = p.lengths[i], base = first_tile<COLS>(p, row, i);
  const unsigned long begun = __ballot(lo + lane <= hi && base <= w);
  if (begun == 0) return false;
  const int k = 63 - __builtin_clzl(begun);
  return set_tile<COLS>(p, w, lo + k, __builtin_amdgcn_readlane(base, k), __builtin_amdgcn_readlane(row, k),
                        __builtin_amdgcn_readlane(next, k), __builtin_amdgcn_readlane(length, k), t);
}

// Bits t0 .. 15 of those below t1, each end within 0 .. 16: which of a sixteen's tokens count.
__device__ __forceinline__ unsigned token_bits(int t0, int t1) {
  return ((1u << min(max(t1, 0), 16)) - 1u) & ~((1u << min(max(t0, 0), 16)) - 1u);
}

// Half bytes u as binary16: the low ones of w's bytes 0 and 2 as 1024 + u, the high ones as 1024 + 16 u, one instruction
// for two (mask and pattern in registers: one instruction takes them, not two literals).
struct Unpack {
  unsigned low_mask = 0x000f000fu, high_mask = 0x00f000f0u, one = 0x64006400u;
  __device__ __forceinline__ Unpack() { asm volatile("" : "+s"(low_mask), "+s"(high_mask), "+v"(one)); }
  __device__ __forceinline__ h2 low(unsigned w) const { return __builtin_bit_cast(h2, (w & low_mask) | one); }
  __device__ __forceinline__ h2 high(unsigned w) const { return __builtin_bit_cast(h2, (w & high_mask) | one); }
};
__device__ __forceinline__ h8 join4(h2 a, h2 b, h2 c, h2 d) {
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The largest of the four lanes that hold a column (lane % 16).
__device__ __forceinline__ float column_max(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace

// The launch for many columns (q8_kv4_wide.hip); p.tiles: of kWideCols columns.
constexpr int kWideCols = 128;
int kv4_attend_wide(int G, const AttendParams& p, const void* q, void* out, int type, hipStream_t stream);

}  // namespace q8
