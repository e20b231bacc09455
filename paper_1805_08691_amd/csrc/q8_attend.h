// Shared by the kernels of attention over the paged caches: what a launch and a tile are, the split of the key axis, and
// how columns and parts are added.
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
  int all;                             // every row sees all of its request's keys (window 0)
  float scale_log2;                    // scale * log2(e)
};

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 64;              // keys of a wavefront's step
constexpr int kWaves = 4;
constexpr int kCols = 16;              // columns of an MFMA tile
constexpr int kWideTiles = 2;          // of them, of a wavefront of a workgroup for many columns
constexpr int kWideCols = kWaves * kWideTiles * kCols;         // and the workgroup's columns
constexpr int kWideParts = 16;         // that a tile of them is cut into at most: the last workgroup adds them alone

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

// The position up to which row `tok` of tile t's request sees keys.
__device__ __forceinline__ int row_position(const AttendParams& p, const Tile& t, int tok) {
  return p.all ? t.len - 1 : t.len - t.n + tok;
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
  const int pos0 = row_position(p, *t, tok0), pos1 = row_position(p, *t, tok1);
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

// Parts that the keys are cut into where tiles are few: two for a compute unit.  (Over the 4-bit cache, us: 48 requests of up to 16384
// tokens, 64 query heads on 8 of 128 channels, 107; for 384 parts 125, 640 114, 768 115.  One of 131071, 32 heads on 8: 44, 51,
// 49, 47.  Over the 8-bit one these take 151 and 58, at the memory's rate.)
constexpr int kTarget = 512;
// A part is not shorter than a step for each wavefront, and than two of them where that makes kTarget / 2 parts.  (Over the 4-bit
// cache: one request of 2000 tokens 11.6 us, never shorter than 8 or 16 steps 13.2 and 16.9; 8 of 4096, 64 channels, 14.0, with 4
// 14.8.)
constexpr int kShortest = 4;
constexpr int kMaxTiles = 256;         // beyond them nothing is cut: a thread each
constexpr int kManyTiles = 128;        // times heads: a workgroup for every second compute unit

// The split of the key axis.  The steps of all tiles and heads over kTarget are what a part should hold (`least` at
// least); a tile of more steps is cut into equal parts of no more.  Every workgroup works this out for itself from the
// lengths, a tile to a thread.  Parts of cut tiles have a place in the workspace, no more than 2 kTarget of them (a cut
// tile has more than `per` steps), and the cut tiles' heads, no more than kTarget, a counter.
//
// Parts of a tile are of equal numbers of steps, rounded up, but the last: that one has a step at least.  Where `most` keeps their
// number down, as many such parts may be fewer (65 steps in at most 16 parts: 13 of five).
__host__ __device__ constexpr unsigned parts_of(unsigned steps, unsigned per, unsigned most) {
  unsigned n = steps == 0 ? 0 : (steps + per - 1) / per;
  if (n > most) {
    const unsigned each = (steps + most - 1) / most;
    n = (steps + each - 1) / each;
  }
  return n;
}
constexpr bool no_part_is_empty(unsigned most) {
  for (unsigned per = kShortest; per <= 2 * kShortest; ++per)
    for (unsigned steps = 1; steps <= 512; ++steps) {
      const unsigned n = parts_of(steps, per, most), each = (steps + n - 1) / n;
      if (n > most || (n - 1) * each >= steps) return false;
    }
  return true;
}
static_assert(no_part_is_empty(kWideParts) && no_part_is_empty(kTarget), "the last part of a tile has a step at least");

struct Part {
  int head, part, parts;
  int slot, rank;                      // of a cut tile: its first part's place and its number, in units of H
  int step0, step1;
};

// The part of workgroup `id` (of MOST that a tile is cut into at most), and its tile; false: there is none.  SORTED: the
// longest tiles first.  LEAST: steps of the shortest part where tiles and heads are kManyTiles.  `shared`: LDS that is free until
// then.
template <int COLS, int MOST, bool SORTED = false, int LEAST = 0>
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
  auto tile = [&](int w) __attribute__((always_inline)) {
    int b = 0, hi = p.B - 1;
    while (b < hi) {
      const int mid = (b + hi + 1) >> 1;
      if (bases[mid] <= w) b = mid; else hi = mid - 1;
    }
    return w < p.tiles && set_tile<COLS>(p, w, b, bases[b], rows[b], rows[b + 1], lengths[b], &t);
  };
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
    is = tile(tid);
    if constexpr (SORTED) {            // (all keys differ: a tile's place is the number of larger ones)
      unsigned* const keys = reinterpret_cast<unsigned*>(rows + kMaxTiles + 4);
      unsigned char* const order = reinterpret_cast<unsigned char*>(keys + kMaxTiles);
      const unsigned key = (is ? (unsigned)min(max(t.steps, 1), 0xffffff) : 0u) << 8 | (255u - tid);
      keys[tid] = key;
      __syncthreads();
      int larger = 0;
      for (int i = 0; i < kMaxTiles; i += 4) {
        const uint4 k = *reinterpret_cast<const uint4*>(keys + i);
        larger += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
      }
      order[larger] = (unsigned char)tid;
      __syncthreads();
      is = tile(order[tid]);
    }
  }
  // all tiles' steps, in two halves: less than 2^25 of each, 2^8 tiles
  const unsigned steps = is ? max(t.steps, 1) : 0;
  const unsigned lo = scan64(steps & 0xffffu), hi = scan64(steps >> 16);
  if (lane == 63) low[wave] = lo, high[wave] = hi;
  if (tid == 0) found[0] = 0;
  __syncthreads();
  const long total = ((long)((low[0] + low[1]) + (low[2] + low[3])) + ((long)((high[0] + high[1]) + (high[2] + high[3])) << 16)) * p.H;
  long least = min(max((2 * total + kTarget - 1) / kTarget, (long)kShortest), 2l * kShortest);
  if (LEAST && p.tiles * p.H >= kManyTiles) least = LEAST;
  const unsigned per = (unsigned)max((total + kTarget - 1) / kTarget, least);
  // the sums before each tile: parts (kTarget + kMaxTiles at most); those of cut tiles (10 bits up); cut tiles (20 bits up)
  const unsigned n = parts_of(steps, per, MOST), own = n > 1 ? n | n << 10 | 1u << 20 : n;
  unsigned v = scan64(own);
  if (lane == 63) sums[wave] = v;
  __syncthreads();
  for (int u = 0; u < wave; ++u) v += sums[u];
  // (the last tiles of a request see most keys: where tiles take longest they go first)
  const int place = COLS == kCols || SORTED ? at : (int)(((sums[0] + sums[1]) + (sums[2] + sums[3])) & 0x3ffu) - 1 - at;
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

// The end of a workgroup of kCols columns whose wavefronts have seen keys of their own: lane (r, j) of each has channels
// 16 c + 4 j .. of column r in o[c], relative to 2^ref (as `sum`, of its four lanes).  The wavefronts' columns are added, and
// stored or put into the workspace; the last workgroup of a cut tile and head adds its parts.  D channels; `shared`: LDS,
// join_bytes(D, cut) of it.
template <int D>
struct Join {
  static constexpr int CT = D / 16;
  static constexpr int PITCH = D + 4;                   // of a column in LDS: eight lanes' quads meet different banks
  static constexpr size_t kPartWords = kCols * (D + 2) / 2;      // of a part: sums [16][D], then a maximum and a sum for each column
};
constexpr size_t join_bytes(int D, bool cut, int waves = kWaves) {
  const size_t columns = (size_t)waves * kCols * (D + 6) * 4, adding = 256 * 16 + (kTarget + 1) * kCols * sizeof(float);
  return cut && columns < adding ? adding : columns;
}
template <int D, int WAVES = kWaves, typename V>
__device__ __forceinline__ void join_columns(const AttendParams& p, const Part& a, const Tile& t, char* shared, V* __restrict__ out,
                                             const f4 (&o)[D / 16], float ref, float sum) {
  constexpr int CT = Join<D>::CT, PITCH = Join<D>::PITCH;
  constexpr size_t kPartWords = Join<D>::kPartWords;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, j = lane >> 4, head = a.head;
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  __syncthreads();                                      // LDS has been read: the columns take its place

  // ---- the wavefronts' columns together
  float* const cols = reinterpret_cast<float*>(shared);
  float* const refs = cols + WAVES * kCols * PITCH;
  float* const sums = refs + WAVES * kCols;
  if (j == 0) {
    refs[wave * kCols + r] = ref;
    sums[wave * kCols + r] = sum;
  }
  __syncthreads();
  float all = -__builtin_inff();
#pragma unroll
  for (int v = 0; v < WAVES; ++v) all = fmaxf(all, refs[v * kCols + r]);
  const float mine = ref == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(ref - all);
  float* const to = cols + (wave * kCols + r) * PITCH + 4 * j;
#pragma unroll
  for (int c = 0; c < CT; ++c) *reinterpret_cast<f4*>(to + 16 * c) = o[c] * mine;
  __syncthreads();
  const bool whole = a.parts == 1;
  const int valid = min(kCols, t.cols - t.first);
  for (int i = tid; i < valid * D / 4; i += 64 * WAVES) {
    const int c = i / (D / 4), d = i % (D / 4) * 4;
    f4 v = {0, 0, 0, 0};
    float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int u = 0; u < WAVES; ++u) m = fmaxf(m, refs[u * kCols + c]);
#pragma unroll
    for (int u = 0; u < WAVES; ++u) {
      v += *reinterpret_cast<const f4*>(cols + (u * kCols + c) * PITCH + d);
      const float ru = refs[u * kCols + c];
      l += ru == -__builtin_inff() ? 0.0f : sums[u * kCols + c] * __builtin_amdgcn_exp2f(ru - m);
    }
    if (whole) {
      const int oc = t.first + c;
      const float inv = l > 0.0f ? 1.0f / l : l;        // (no key: zeros; no number: none)
      const float y[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
      store_values<4, false>(out + (size_t)(t.row + oc / p.ratio) * p.o_stride +
                                 ((size_t)head * p.ratio + oc % p.ratio) * p.o_head + d, y);
    } else {
      // past this XCD's cache, for the workgroup that adds the parts
      word* part = reinterpret_cast<word*>(p.parts) + ((size_t)(a.slot + a.part) * p.H + head) * kPartWords;
      put(part + (c * D + d) / 2, v[0], v[1]);
      put(part + (c * D + d) / 2 + 1, v[2], v[3]);
      if (d == 0) put(part + kCols * D / 2 + c, m, l);
    }
  }
  if (whole) return;

  // ---- the parts of the tile and head: the workgroup that finishes last adds them, whichever it is in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's words have arrived
  __syncthreads();                                      // and the others'; LDS is free
  int* const flag = reinterpret_cast<int*>(shared);
  int* const counter = p.counters + a.rank * p.H + head;
  if (tid == 0) flag[0] = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  __syncthreads();
  if (flag[0] != a.parts - 1) return;
  __syncthreads();
  if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  const word* const parts = reinterpret_cast<const word*>(p.parts) + ((size_t)a.slot * p.H + head) * kPartWords;
  const size_t stride = (size_t)p.H * kPartWords;
  const int n = a.parts;
  f4* const quads = reinterpret_cast<f4*>(shared);      // 256
  float* const weights = reinterpret_cast<float*>(quads + 256);               // [n][16], then the columns' sums
  float* const totals = weights + (size_t)kTarget * kCols;
  for (int c = wave; c < valid; c += kWaves) {
    float most = -__builtin_inff(), l = 0.0f;
    f2 rs[kTarget / 64];
#pragma unroll
    for (int u = 0; u < kTarget / 64; ++u) {
      rs[u] = f2{-__builtin_inff(), 0.0f};
      if (u * 64 < n && u * 64 + lane < n) rs[u] = get(parts + (u * 64 + lane) * stride + kCols * D / 2 + c);
    }
#pragma unroll
    for (int u = 0; u < kTarget / 64; ++u) most = fmaxf(most, rs[u][0]);
    for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, 64));
#pragma unroll
    for (int u = 0; u < kTarget / 64; ++u)
      if (u * 64 + lane < n) {
        const float weight = rs[u][0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(rs[u][0] - most);
        weights[(u * 64 + lane) * kCols + c] = weight;
        l += weight * rs[u][1];
      }
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off, 64);
    if (lane == 0) totals[c] = l;
  }
  __syncthreads();
  // a thread takes four channels of a column, and where these are few, every so manieth part
  const int items = valid * (D / 4), groups = items >= 256 ? 1 : 256 / items, each = groups > 1 ? items : 256;
  for (int i0 = 0; i0 < items; i0 += 256) {
    const int group = groups > 1 ? tid / each : 0, i = i0 + (groups > 1 ? tid - group * each : tid);
    const int c = i / (D / 4), d = i % (D / 4) * 4;
    f4 v = {0, 0, 0, 0};
    // (as many parts on their way as there are, rounded up: the last is read again in the place of absent ones)
    auto add = [&](auto batch_c) __attribute__((always_inline)) {
      constexpr int kBatch = decltype(batch_c)::value;
      const word* from = parts + (c * D + d) / 2;
      for (int s0 = group; s0 < n; s0 += groups * kBatch) {
        f2 x[kBatch], y[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int s = min(s0 + u * groups, n - 1);
          x[u] = get(from + s * stride), y[u] = get(from + s * stride + 1);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (s0 + u * groups < n) v += weights[(s0 + u * groups) * kCols + c] * f4{x[u][0], x[u][1], y[u][0], y[u][1]};
      }
    };
    if (i < items && group < groups) {
      if (n <= 2 * groups) add(std::integral_constant<int, 2>{});
      else if (n <= 4 * groups) add(std::integral_constant<int, 4>{});
      else if (n <= 8 * groups) add(std::integral_constant<int, 8>{});
      else add(std::integral_constant<int, 16>{});
    }
    if (groups > 1) {
      quads[tid] = v;
      __syncthreads();
      if (group == 0)
        for (int g = 1; g < groups; ++g) v += quads[g * each + tid];
    }
    if (group == 0 && i < items) {
      const int oc = t.first + c;
      const float l = totals[c], inv = l > 0.0f ? 1.0f / l : l;
      const float y[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
      store_values<4, false>(out + (size_t)(t.row + oc / p.ratio) * p.o_stride +
                                 ((size_t)head * p.ratio + oc % p.ratio) * p.o_head + d, y);
    }
  }
}

// The same for workgroups of WAVES wavefronts that have all seen the same keys, each with TILES tiles of W columns: lane (r, j),
// r < W, of wavefront w has channels 256 / W i + 4 j .. of column (w TILES + c) W + r in o[c][i]; seen[c]: whether the column has
// seen a key.
template <int D, int WAVES, int W, int TILES, typename V>
__device__ __forceinline__ void join_wide(const AttendParams& p, const Part& a, const Tile& t, char* shared, V* __restrict__ out,
                                          const f4 (&o)[TILES][D * W / 256], const float (&ref)[TILES],
                                          float (&sum)[TILES], const bool (&seen)[TILES]) {
  constexpr int CT = D * W / 256, COLS = WAVES * TILES * W, NEXT = 256 / W;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane % W, j = lane / W, head = a.head;
  constexpr size_t kPartWords = (size_t)COLS * (D + 2) / 2;    // of a part: [tile][CT][2][lane], then maxima and sums
  word* const part = reinterpret_cast<word*>(p.parts) + ((size_t)(a.slot + a.part) * p.H + head) * kPartWords;
#pragma unroll
  for (int c = 0; c < TILES; ++c) {
    if constexpr (W == 16) sum[c] += __shfl_xor(sum[c], 16, 64);
    sum[c] += __shfl_xor(sum[c], 32, 64);
    const int of = (wave * TILES + c) * W + r, col = t.first + of;
    if (col >= t.cols) continue;
    const float l = sum[c];
    if (a.parts == 1) {
      const float inv = l > 0.0f ? 1.0f / l : l;                // (no key: zeros; no number: none)
      V* const to = out + (size_t)(t.row + col / p.ratio) * p.o_stride + ((size_t)head * p.ratio + col % p.ratio) * p.o_head + 4 * j;
#pragma unroll
      for (int i = 0; i < CT; ++i) {
        const float y[4] = {o[c][i][0] * inv, o[c][i][1] * inv, o[c][i][2] * inv, o[c][i][3] * inv};
        store_values<4, false>(to + NEXT * i, y);
      }
    } else {
      word* const to = part + (wave * TILES + c) * CT * 128 + lane;
#pragma unroll
      for (int i = 0; i < CT; ++i) {
        put(to + 128 * i, o[c][i][0], o[c][i][1]);
        put(to + 128 * i + 64, o[c][i][2], o[c][i][3]);
      }
      if (j == 0) put(part + COLS * D / 2 + of, seen[c] ? ref[c] : -__builtin_inff(), l);
    }
  }
  if (a.parts == 1) return;

  // ---- the parts of the tile and head: the workgroup that finishes last adds them, whichever it is in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's words have arrived
  __syncthreads();                                      // and the others'; LDS is free
  int* const flag = reinterpret_cast<int*>(shared);
  int* const counter = p.counters + a.rank * p.H + head;
  if (tid == 0) flag[0] = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  __syncthreads();
  if (flag[0] != a.parts - 1) return;
  __syncthreads();
  if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  const word* const parts = reinterpret_cast<const word*>(p.parts) + ((size_t)a.slot * p.H + head) * kPartWords;
  const size_t stride = (size_t)p.H * kPartWords;
  float* const weights = reinterpret_cast<float*>(shared);      // [16][COLS], then the columns' sums
  float* const totals = weights + kWideParts * COLS;
  if (tid < COLS) {
    f2 rs[kWideParts];
    float most = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int u = 0; u < kWideParts; ++u) {
      rs[u] = f2{-__builtin_inff(), 0.0f};
      if (u < a.parts && t.first + tid < t.cols) rs[u] = get(parts + u * stride + COLS * D / 2 + tid);
    }
#pragma unroll
    for (int u = 0; u < kWideParts; ++u) most = fmaxf(most, rs[u][0]);
#pragma unroll
    for (int u = 0; u < kWideParts; ++u) {
      const float weight = rs[u][0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(rs[u][0] - most);
      weights[u * COLS + tid] = weight;
      l += weight * rs[u][1];
    }
    totals[tid] = l;
  }
  __syncthreads();
  // a thread takes four channels of a column, as a lane had them, and several such, so that enough is on its way
  const int valid = t.cols - t.first, groups = min((valid + W - 1) / W, COLS / W) * CT;     // of 64 lanes' quads
  constexpr int kItems = 4, kBatch = 4;
  for (int g0 = wave; g0 < groups; g0 += WAVES * kItems) {
    f4 v[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) v[k] = f4{0, 0, 0, 0};
    for (int s0 = 0; s0 < a.parts; s0 += kBatch) {
      f2 x[kItems][kBatch][2];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
          const word* const from = parts + min(s0 + u, a.parts - 1) * stride + min(g0 + k * WAVES, groups - 1) * 128 + lane;
          x[k][u][0] = get(from), x[k][u][1] = get(from + 64);
        }
#pragma unroll
      for (int k = 0; k < kItems; ++k)
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (s0 + u < a.parts)
            v[k] += weights[(s0 + u) * COLS + min(g0 + k * WAVES, groups - 1) / CT * W + r] *
                    f4{x[k][u][0][0], x[k][u][0][1], x[k][u][1][0], x[k][u][1][1]};
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int g = g0 + k * WAVES, of = g / CT * W + r, col = t.first + of;
      if (g >= groups || col >= t.cols) continue;
      const float l = totals[of], inv = l > 0.0f ? 1.0f / l : l;
      const float y[4] = {v[k][0] * inv, v[k][1] * inv, v[k][2] * inv, v[k][3] * inv};
      store_values<4, false>(out + (size_t)(t.row + col / p.ratio) * p.o_stride + ((size_t)head * p.ratio + col % p.ratio) * p.o_head +
                                 g % CT * NEXT + 4 * j, y);
    }
  }
}

// ---- on the host
// Tiles of `cols` columns that T rows of B requests can have (find_tile).
inline size_t tiles_of(size_t T, int B, int ratio, bool starts, int cols = kCols) {
  return starts ? T * ratio / cols + B : (size_t)B * ((ratio + cols - 1) / cols);
}
// Whether keys of at most `longest` are cut: where tiles are so few that a part of the longest could keep compute units
// waiting, and two parts of 2 kShortest steps could be made.  (5 requests of up to 300 tokens: 7.3 us, and cut 10.4.)
inline bool cut(size_t tiles, size_t longest) { return tiles <= kMaxTiles && longest > (size_t)2 * kShortest * kStep; }
// Workspace: the counters (in one place for both kernels), then the parts.
constexpr size_t kCounterBytes = (kTarget + 15) / 16 * 16 * sizeof(int);
inline size_t split_bytes(int D, int cols = kCols) { return kCounterBytes + (size_t)2 * kTarget * cols * (D + 2) * 4; }

// Whether tiles of kWideCols columns are taken for T new tokens of B requests in runs of several (and then for more tokens of as
// many requests); cuts: they could be cut.
typedef bool WideFor(size_t T, int B, int H, int ratio, int D, size_t longest, bool cuts);

inline size_t attend_workspace_bytes(size_t T, int n_requests, int n_heads, int ratio, int D, size_t longest, WideFor* wide_for) {
  if (n_requests < 1 || n_heads < 1 || ratio < 1 || D < 32 || D > kMaxHead || T > 0x7fffffffu) return 0;
  // The most that any of up to T tokens is split with.  Tiles of 128 columns are cut if there are no more than kMaxTiles,
  // and the more there are, the sooner they are taken; tiles of 16 are fewest for a single token, or one of each request.
  const size_t B = (size_t)n_requests, columns = B <= kMaxTiles ? (kMaxTiles + 1 - B) * kWideCols - 1 : 0;
  const size_t few = columns / ratio < T ? columns / ratio : T;
  if (few > 0 && cut(tiles_of(few, n_requests, ratio, true, kWideCols), longest) &&
      wide_for(few, n_requests, n_heads, ratio, D, longest, true))
    return split_bytes(D, kWideCols);
  const bool rows = cut(tiles_of(1, n_requests, ratio, true), longest) || cut(tiles_of(B, n_requests, ratio, false), longest);
  return rows ? split_bytes(D) : 0;
}

// What a call runs as: tiles of kWideCols or of kCols columns, how many there can be, and whether keys may be split.  least: find_part's
// LEAST of the kernel for few columns.
struct Form {
  bool wide, split;
  size_t tiles;
};
inline Form form_of(size_t T, int B, int H, int ratio, int D, size_t longest, bool starts, size_t workspace_bytes, WideFor* wide_for,
                    int least) {
  const size_t wide_tiles = tiles_of(T, B, ratio, true, kWideCols), narrow_tiles = tiles_of(T, B, ratio, starts);
  const bool cuts = workspace_bytes >= split_bytes(D, kWideCols) && cut(wide_tiles, longest);
  if (starts && wide_for(T, B, H, ratio, D, longest, cuts)) return {true, cuts, wide_tiles};
  const bool whole = narrow_tiles * H >= (size_t)kManyTiles && longest <= (size_t)least * kStep;       // (none has two parts)
  return {false, workspace_bytes >= split_bytes(D) && cut(narrow_tiles, longest) && !whole, narrow_tiles};
}

// A call's arguments, checked, as *p, and whether it goes to the kernel for many columns.  p->T = 0: there is nothing to do.
inline int attend_params(const void* q_dev, int type, size_t T, int n_heads, int ratio, int D, size_t q_stride,
                         size_t q_head_stride, const void* cache_dev, size_t n_pages, int page, const int32_t* table_dev, int width,
                         size_t table_stride, const int32_t* lengths_dev, const int32_t* starts_dev, int n_requests, float scale,
                         int window, void* out_dev, size_t o_stride, size_t o_head_stride, void* workspace,
                         size_t workspace_bytes, WideFor* wide_for, AttendParams* out, bool* is_wide, int least = 0) {
  Q8_REQUIRE(type_ok(type) && n_heads >= 1 && ratio >= 1 && width >= 0 && window >= 0 && n_requests >= 0, Q8_EINVAL);
  Q8_REQUIRE(scale == scale && scale - scale == 0.0f, Q8_EINVAL);
  Q8_REQUIRE(type != Q8_F32 && kv4_shape_ok(D, page), Q8_EUNSUPPORTED);
  if (T == 0 || n_requests == 0) return Q8_OK;
  Q8_REQUIRE(q_dev && out_dev && cache_dev && n_pages >= 1 && lengths_dev && (table_dev || width == 0), Q8_EINVAL);
  Q8_REQUIRE(table_stride >= (size_t)width && (starts_dev || T == (size_t)n_requests), Q8_EINVAL);
  Q8_REQUIRE(T == 1 || (q_stride >= (size_t)D && o_stride >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(n_heads * ratio == 1 || (q_head_stride >= (size_t)D && o_head_stride >= (size_t)D), Q8_EINVAL);
  // (a table's places end far enough below 2^31 that the sixteens behind a tile's last key still have an int's numbers)
  Q8_REQUIRE(T <= 0x7fffffffu && n_pages <= 0x7fffffffu && (size_t)width * page <= 0x7fff0000u, Q8_EUNSUPPORTED);
  Q8_REQUIRE(q8_aligned(q_dev, 2) && q8_aligned(out_dev, 2) && q8_aligned(cache_dev, 64) && q8_aligned(table_dev, 4) &&
                 q8_aligned(lengths_dev, 4) && q8_aligned(starts_dev, 4) && q8_aligned(workspace, 16), Q8_EALIGN);
  const Form form = form_of(T, n_requests, n_heads, ratio, D, (size_t)width * page, starts_dev != nullptr,
                            workspace ? workspace_bytes : 0, wide_for, least);
  const bool split = form.split;
  const size_t tiles = form.tiles, longest = (size_t)width * page;
  Q8_REQUIRE(tiles * n_heads + kTarget <= most_blocks(256) && T * ratio <= 0x7fffffffu, Q8_EUNSUPPORTED);
  AttendParams& p = *out;
  p.cache = static_cast<const uint8_t*>(cache_dev);
  p.table = table_dev;
  p.lengths = lengths_dev;
  p.starts = starts_dev;
  p.counters = split ? static_cast<int*>(workspace) : nullptr;
  p.parts = split ? reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes) : nullptr;
  p.q_stride = q_stride, p.q_head = q_head_stride, p.o_stride = o_stride, p.o_head = o_head_stride;
  p.table_stride = table_stride;
  p.n_pages = (long)n_pages;
  p.T = (int)T, p.B = n_requests, p.H = n_heads, p.ratio = ratio, p.width = width;
  p.shift = __builtin_ctz(page) - 4;
  p.tiles = (int)tiles;
  p.window = (size_t)window >= longest ? 0 : window;      // (as long as a request: none; differences of positions fit an int)
  p.scale_log2 = scale * 1.4426950408889634f;
  *is_wide = form.wide;
  return Q8_OK;
}

}  // namespace

}  // namespace q8
