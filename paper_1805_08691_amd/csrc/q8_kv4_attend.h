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
  t->seen = p.window > 0 ? max(0, max(pos0, 0) - p.window + 1) : 0;        // (rows in front of the first key see none)
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

// Parts that the keys are cut into where tiles are few: two for a compute unit.  (48 requests of up to 16384 tokens, 64 query
// heads on 8 of 128 channels, 107 us; for 384 parts 125, 640 114, 768 115.  One of 131071, 32 heads on 8: 44, 51, 49, 47.)
constexpr int kTarget = 512;
// A part is not shorter than a step for each wavefront, and than two of them where that makes kTarget / 2 parts.  (One
// request of 2000 tokens 11.6 us, never shorter than 8 or 16 steps 13.2 and 16.9; 8 of 4096, 64 channels, 14.0, with 4 14.8.)
constexpr int kShortest = 4;
constexpr int kMaxTiles = 256;         // beyond them nothing is cut: a thread each

// The split of the key axis.  The steps of all tiles and heads over kTarget are what a part should hold (`least` at
// least); a tile of more steps is cut into equal parts of no more.  Every workgroup works this out for itself from the
// lengths, a tile to a thread.  Parts of cut tiles have a place in the workspace, no more than 2 kTarget of them (a cut
// tile has more than `per` steps), and the cut tiles' heads, no more than kTarget, a counter.
struct Part {
  int head, part, parts;
  int slot, rank;                      // of a cut tile: its first part's place and its number, in units of H
  int step0, step1;
};

// The part of workgroup `id` (of MOST that a tile is cut into at most), and its tile; false: there is none.  `shared`: LDS
// that is free until then.
template <int COLS, int MOST>
__device__ __forceinline__ bool find_part(const AttendParams& p, int id, char* shared, Part* a, Tile* out) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int at = id / p.H;
  *a = Part{id - at * p.H, 0, 1, 0, 0, 0, 0};
  if (!p.parts) {
    if (at >= p.tiles || !find_tile<COLS>(p, at, out)) return false;
    a->step1 = out->steps;
    return true;
  }
  int* const found = reinterpret_cast<int*>(shared);
  unsigned* const low = reinterpret_cast<unsigned*>(found + 16);               // [kWaves], three times
  unsigned* const high = low + kWaves;
  unsigned* const sums = high + kWaves;
  int* const bases = reinterpret_cast<int*>(sums + kWaves);    // of the requests: first tiles,
  int* const lengths = bases + kMaxTiles;
  int* const rows = lengths + kMaxTiles;                       // rows, with the last one's end
  Tile t;
  bool is = false;
  if (!p.starts) {
    const int per = (p.ratio + COLS - 1) / COLS, b = tid / per;
    if (tid < p.tiles) is = set_tile<COLS>(p, tid, b, b * per, b, b + 1, p.lengths[b], &t);
  } else {
    for (int i = tid; i <= p.B; i += 256) {                    // (no more requests than tiles)
      const int start = request_start(p, i), length = i < p.B ? p.lengths[i] : 0;
      rows[i] = start;
      if (i < p.B) bases[i] = first_tile<COLS>(p, start, i), lengths[i] = length;
    }
    __syncthreads();
    int b = 0, hi = p.B - 1;
    while (b < hi) {
      const int mid = (b + hi + 1) >> 1;
      if (bases[mid] <= tid) b = mid; else hi = mid - 1;
    }
    if (tid < p.tiles) is = set_tile<COLS>(p, tid, b, bases[b], rows[b], rows[b + 1], lengths[b], &t);
  }
  // all tiles' steps, in two halves: less than 2^25 of each, 2^8 tiles
  const unsigned steps = is ? max(t.steps, 1) : 0;
  const unsigned lo = scan64(steps & 0xffffu), hi = scan64(steps >> 16);
  if (lane == 63) low[wave] = lo, high[wave] = hi;
  if (tid == 0) found[0] = 0;
  __syncthreads();
  const long total = ((long)((low[0] + low[1]) + (low[2] + low[3])) + ((long)((high[0] + high[1]) + (high[2] + high[3])) << 16)) * p.H;
  const long least = min(max((2 * total + kTarget - 1) / kTarget, (long)kShortest), 2l * kShortest);
  const unsigned per = (unsigned)max((total + kTarget - 1) / kTarget, least);
  // the sums before each tile: parts (kTarget + kMaxTiles at most); those of cut tiles (10 bits up); cut tiles (20 bits up)
  const unsigned n = steps ? min((steps + per - 1) / per, (unsigned)MOST) : 0, own = n > 1 ? n | n << 10 | 1u << 20 : n;
  unsigned v = scan64(own);
  if (lane == 63) sums[wave] = v;
  __syncthreads();
  for (int u = 0; u < wave; ++u) v += sums[u];
  // (the last tiles of a request see most keys: where tiles take longest they go first)
  const int place = COLS == kCols ? at : (int)(((sums[0] + sums[1]) + (sums[2] + sums[3])) & 0x3ffu) - 1 - at;
  const unsigned before = v - own;
  const int first = (int)(before & 0x3ffu), slot = (int)(before >> 10 & 0x3ffu), rank = (int)(before >> 20);
  if (place >= first && place < first + (int)n) {
    const int each = (t.steps + (int)n - 1) / (int)n, step0 = (place - first) * each;
    found[0] = 1, found[1] = place - first, found[2] = (int)n, found[3] = slot, found[4] = rank;
    found[5] = step0, found[6] = min(step0 + each, t.steps);
    found[7] = t.b, found[8] = t.row, found[9] = t.first, found[10] = t.cols, found[11] = t.len, found[12] = t.n;
    found[13] = t.seen, found[14] = t.lo, found[15] = t.steps;
  }
  __syncthreads();
  auto get = [&](int i) { return __builtin_amdgcn_readfirstlane(found[i]); };
  const bool there = get(0) != 0;
  *a = Part{a->head, get(1), get(2), get(3), get(4), get(5), get(6)};
  *out = Tile{get(7), get(8), get(9), get(10), get(11), get(12), get(13), get(14), get(15)};
  __syncthreads();                     // (LDS is free)
  return there;
}

// Two numbers of the workspace, between workgroups of different XCDs: written through and read past their caches.
typedef unsigned long word;
typedef float f2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put(word* to, float a, float b) {
  __hip_atomic_store(to, (word)__float_as_uint(a) | (word)__float_as_uint(b) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ f2 get(const word* from) {
  const word v = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  return f2{__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32))};
}

}  // namespace

// The launch for many columns (q8_kv4_wide.hip); p.tiles: of kWideCols columns.
constexpr int kWideCols = 128;
constexpr int kWideParts = 16;         // that a tile of them is cut into at most: the last workgroup adds them alone
int kv4_attend_wide(int G, const AttendParams& p, const void* q, void* out, int type, hipStream_t stream);

}  // namespace q8
