// The pages of a cache, whatever they hold: requests that go on, several times or not at all (q8_page_select), the pages in
// use moved to the front of the pool (q8_page_compact), and pages copied (q8_page_copy).
//
// Which pages are in use is one bit a page, set from the rows that are kept; every number that a page or a request gets is
// its rank among bits or flags, in ascending order, so that results do not depend on which block came first.
//
// Measured (us): 32 requests of up to 63 pages 6.1 and the copies 2.4, 1000 of up to 16 14.5; 4000 requests of up to 256 pages
// 19.4, in five launches of which the rows take 6.4 and the free pages 7.2.  All of them wait for their few dependent trips to memory.
// Every block of the last launch reads all rows' flags and all blocks' counts, so that beyond some ten thousand rows it grows
// with their product: 2^18 rows and 2^20 pages 290, 2^20 and 2^24 2200, 2^22 and 2^24 24500.
#include "q8_kv4.h"
#pragma clang fp contract(off)

namespace {

using namespace q8;

constexpr int kMostPages = 1 << 24, kMostRows = 1 << 24;
constexpr int kBlockWords = 64, kBlockPages = 32 * kBlockWords;        // words of 32 pages that a block lists

struct PagesParams {
  const int* __restrict__ parents;             // null: row c goes on as row c
  const int* __restrict__ lengths;
  const int* table;                            // (compact: may be out_table)
  int* out_table;
  int* __restrict__ out_lengths;
  int* __restrict__ free_pages;
  int* __restrict__ copies;                    // [n_copies][2]
  int* __restrict__ counts;
  uint8_t* __restrict__ marks;                 // of each page, up to whole blocks of them: whether a row holds it
  unsigned* __restrict__ used;                 // the same as bits, [blocks][kBlockWords]
  unsigned* __restrict__ counts_of;            // and their number in each block
  int* __restrict__ before;                    // compact: of each word, pages in use before it; select: parents' first rows
  uint8_t* __restrict__ flags;                 // select: of each new row, whether it needs a copy of its last page
  size_t stride, out_stride;
  int n, m, shift, width, pool, blocks, n_copies;          // old rows, new rows; shift: page = 1 << shift tokens
};

__device__ __forceinline__ int length_of(const PagesParams& p, int b) {
  return (int)min((long)max(p.lengths[b], 0), (long)p.width << p.shift);
}
__device__ __forceinline__ int pages_of(const PagesParams& p, int tokens) {
  return (int)(((long)tokens + (1 << p.shift) - 1) >> p.shift);
}

// Sums before a thread of a block of WAVES wavefronts, and of the block.
template <int WAVES>
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned (&sums)[WAVES], unsigned* total) {
  const unsigned upto = scan64(v), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  lds_barrier();                                           // the sums of a scan before have been read
  if (lane == 63) sums[wave] = upto;
  lds_barrier();
  const unsigned waves = scan64(lane < WAVES ? sums[lane] : 0u);
  *total = __builtin_amdgcn_readlane(waves, WAVES - 1);
  return upto - v + (wave ? __shfl(waves, wave - 1, 64) : 0u);
}

// The same of N numbers at once, in a block of 256: one trip through LDS.
template <int N>
__device__ __forceinline__ void block_scans(const unsigned (&v)[N], unsigned (&sums)[N][4], unsigned (&before)[N], unsigned (&total)[N]) {
  const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const unsigned upto = scan64(v[i]);
    if (lane == 63) sums[i][wave] = upto;
    before[i] = upto - v[i];
  }
  lds_barrier();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    total[i] = sums[i][0] + sums[i][1] + sums[i][2] + sums[i][3];
#pragma unroll
    for (unsigned w = 0; w < 3; ++w) before[i] += w < wave ? sums[i][w] : 0u;
  }
}

// A thread's share of the pages in use, of all blocks and of those in front of block `end`.
__device__ __forceinline__ void count_used(const PagesParams& p, int end, unsigned* all, unsigned* front) {
  *all = *front = 0;
  for (int i = threadIdx.x; i < p.blocks; i += 256) {
    const unsigned c = p.counts_of[i];
    *all += c;
    if (i < end) *front += c;
  }
}

__global__ __launch_bounds__(256) void pages_clear_kernel(uint4* marks, size_t n_marks, int* first, int n) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n_marks) marks[i] = uint4{0, 0, 0, 0};
  if (i < (size_t)n) first[i] = 0x7fffffff;
}
// Four bytes of 0 or 1 as four bits, in order.
__device__ __forceinline__ unsigned bits_of(unsigned w) { return (w & 0x01010101u) * 0x10204080u >> 28; }

// Marks to bits and their numbers: eight pages a thread.
__global__ __launch_bounds__(256) void pages_count_kernel(const PagesParams p) {
  __shared__ unsigned sums[4];
  const uint2 m = reinterpret_cast<const uint2*>(p.marks)[blockIdx.x * 256 + threadIdx.x];
  const unsigned bits = bits_of(m.x) | bits_of(m.y) << 4;
  unsigned word = bits << (8 * (threadIdx.x & 3)), total;
  word |= __shfl_xor(word, 1, 64);
  word |= __shfl_xor(word, 2, 64);
  if ((threadIdx.x & 3) == 0) p.used[blockIdx.x * kBlockWords + threadIdx.x / 4] = word;
  block_scan(__popc(bits), sums, &total);
  if (threadIdx.x == 0) p.counts_of[blockIdx.x] = total;
}

// The first new row of each parent, where rows are so many that looking through them all for every one takes longer.
__global__ __launch_bounds__(256) void select_first_kernel(const PagesParams p) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= p.m) return;
  const int parent = p.parents[c];
  if (parent >= 0 && parent < p.n) atomicMin(&p.before[parent], c);
}

__device__ __forceinline__ void mark(const PagesParams& p, int page) {
  if (page >= 0 && page < p.pool) p.marks[page] = 1;
}

// A wavefront takes a new row: its parent's places, whose pages are in use.  Of several rows of a parent, the first has its
// last page for itself; the others need a copy of it unless it is full.
__global__ __launch_bounds__(256) void select_rows_kernel(const PagesParams p) {
  const int c = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (c >= p.m) return;
  const int parent = p.parents[c];
  const bool given = parent >= 0 && parent < p.n;
  const int len = given ? length_of(p, parent) : 0, held = pages_of(p, len);
  const int* const from = p.table + (given ? parent : 0) * p.stride;
  int* const to = p.out_table + c * p.out_stride;
  constexpr int kAhead = 4;                                // places of a lane that are on their way during the search
  int page[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) page[u] = u * 64 + lane < held ? from[u * 64 + lane] : -1;
  bool again = false;
  if (given && p.before) {
    again = p.before[parent] < c;
  } else if (given) {
    constexpr int kBatch = 16;
    for (int i0 = 0; i0 < c; i0 += 64 * kBatch) {
      int v[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) v[u] = i0 + u * 64 + lane < c ? p.parents[i0 + u * 64 + lane] : -1;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) again |= v[u] == parent;
    }
    again = __any(again);
  }
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (u * 64 + lane < p.width) {
      to[u * 64 + lane] = page[u];
      if (!again) mark(p, page[u]);
    }
#pragma unroll 4
  for (int i = kAhead * 64 + lane; i < p.width; i += 64) {
    const int x = i < held ? from[i] : -1;
    to[i] = x;
    if (!again) mark(p, x);
  }
  if (lane == 0) {
    p.out_lengths[c] = len;
    p.flags[c] = again && (len & ((1 << p.shift) - 1));
  }
}

// Free pages in order: the first of them become copies, of the rows that need one in their order; the others are listed.  Rows
// that find none become empty.  A block lists kBlockPages pages; every block adds up all blocks and rows for itself.
__global__ __launch_bounds__(256) void select_free_kernel(const PagesParams p) {
  __shared__ __attribute__((aligned(16))) unsigned sums[4][4];
  __shared__ unsigned ranks[kBlockWords], words[kBlockWords];
  __shared__ int list[kBlockPages], rows[kBlockPages];
  const int tid = threadIdx.x, page0 = blockIdx.x * kBlockPages;
  // ---- rows that need a copy: those of this thread, one after the other
  const int each = (p.m + 4095) / 4096 * 16, row0 = tid * each, row1 = min(row0 + each, p.m);
  unsigned flags = 0;
  unsigned long which = 0;                                 // of the first 64
  for (int c = row0; c < row1; c += 16) {
    const uint4 w = *reinterpret_cast<const uint4*>(p.flags + c);
    const unsigned some = (bits_of(w.x) | bits_of(w.y) << 4 | bits_of(w.z) << 8 | bits_of(w.w) << 12) & (row1 - c < 16 ? (1u << (row1 - c)) - 1u : 0xffffu);
    flags += __popc(some);
    if (c - row0 < 64) which |= (unsigned long)some << (c - row0);
  }
  unsigned bits = tid < kBlockWords && blockIdx.x < p.blocks ? p.used[blockIdx.x * kBlockWords + tid] : 0xffffffffu;
  const int behind = page0 + 32 * (tid + 1) - p.pool;
  bits = behind >= 32 ? 0 : behind > 0 ? ~bits & 0xffffffffu >> behind : ~bits;
  unsigned v[4] = {0, 0, flags, (unsigned)__popc(bits)}, before[4], total[4];
  count_used(p, blockIdx.x, &v[0], &v[1]);
  block_scans(v, sums, before, total);
  const int n_needed = (int)total[2], n_free = p.pool - (int)total[0], taken = min(n_needed, n_free), first = page0 - (int)total[1];
  int rank = (int)before[2];
  // ---- this block's free pages
  if (tid < kBlockWords) ranks[tid] = before[3], words[tid] = bits;
  const int end = first + (int)total[3];
  lds_barrier();
#pragma unroll
  for (int i = tid; i < kBlockPages; i += 256) {
    const unsigned word = words[i >> 5], e = i & 31;
    if (!(word >> e & 1u)) continue;
    const int at = (int)ranks[i >> 5] + __popc(word & ((1u << e) - 1u)), page = page0 + i;
    if (first + at >= taken) p.free_pages[first + at - taken] = page;
    else list[at] = page;
  }
  lds_barrier();
  // ---- places behind the last of the lists
  for (int i = page0 + tid; i < min(page0 + kBlockPages, p.pool); i += 256)
    if (i >= n_free - taken) p.free_pages[i] = -1;
  for (int i = blockIdx.x * 256 + tid; i < p.m; i += gridDim.x * 256)
    if (i >= taken) p.copies[2 * i] = -1, p.copies[2 * i + 1] = -1;
  if (blockIdx.x == 0 && tid == 0)
    p.counts[0] = n_free - taken, p.counts[1] = taken, p.counts[2] = n_needed - taken, p.counts[3] = p.pool - n_free + taken;
  // ---- copies of rank first .. end - 1 are here, a row to a thread; rows behind the last free page are emptied, each by a wavefront
  // of one of the blocks
  const bool empties = n_needed > n_free;
  if (first >= taken && !empties) return;
  auto needs = [&](int i) { return i < 64 ? (which >> i & 1ul) != 0 : p.flags[row0 + i] != 0; };
  if (!empties) {
    for (int i = 0; flags && i < row1 - row0; ++i) {
      if (!needs(i)) continue;
      if (rank >= first && rank < end) rows[rank - first] = row0 + i;
      ++rank;
    }
  } else {
    for (int i = 0; i < each && __any(flags != 0); ++i) {
      const bool one = flags && i < row1 - row0 && needs(i);
      if (one && rank >= first && rank < min(end, n_free)) rows[rank - first] = row0 + i;
      for (unsigned long none = __ballot(one && rank >= n_free && (row0 + i) % gridDim.x == blockIdx.x); none; none &= none - 1) {
        const int c = __builtin_amdgcn_readlane(row0, __builtin_ctzl(none)) + i;
        for (int col = tid & 63; col < p.width; col += 64) p.out_table[c * p.out_stride + col] = -1;
        if ((tid & 63) == 0) p.out_lengths[c] = 0;
      }
      rank += one;
    }
  }
  lds_barrier();
  for (int i = tid; i < min(end, taken) - first; i += 256) {
    const int c = rows[i];
    int* const entry = p.out_table + c * p.out_stride + pages_of(p, p.out_lengths[c]) - 1;
    p.copies[2 * (first + i)] = *entry;
    *entry = p.copies[2 * (first + i) + 1] = list[i];
  }
}

// Both for tables of few places, in one launch of one block: a row to a thread, and kFewPlaces of the tables' places, of any
// row, which it keeps in registers.  Bound by three dependent trips to memory and the barriers of the sums, and by what one block
// writes where pages are many.  (us of select and of compact, 512 requests of 16 places, and 1025 of 15 in several launches: pools of
// 1000 pages 9.2, 8.3 and 12.5, 13.5; 8000 10.0, 10.1 and 12.2, 13.1; 16000 11.2, 12.0 and 12.4, 13.4; 24000 12.4, 13.5 and 12.6,
// 13.7; 32000 13.5, 15.3 and 12.3, 13.7; 131072 26.5, 34.8 and 12.4, 13.7.)
constexpr int kFewRows = 1024, kFewPlaces = 16, kFewPages = 24 << 10;
constexpr int kFewWords = 4096;                // of LDS: pages in use as bits, or parents
struct Few {
  int parent[kFewRows];                        // select: of new row c; -1: none, or none that holds pages
  int held[kFewRows];                          // pages of new row c, or (again) minus them
  unsigned used[kFewWords];
  int before[kFewWords];                       // pages in use before a word; select: at first, a parent's first new row
  int list[kFewRows * kFewPlaces];             // select: free pages for copies; compact: where pages go, by rank
  unsigned sums[16];
};
static_assert(kFewPages <= kFewWords * 32, "a bit for every page");
inline bool few(int rows, int parents, int width, size_t n_pages) {
  return rows <= kFewRows && parents <= kFewWords && (size_t)rows * width <= (size_t)kFewRows * kFewPlaces &&
         n_pages <= (size_t)kFewPages;
}

template <bool SELECT>
__global__ __launch_bounds__(1024) void pages_few_kernel(const PagesParams p) {
  extern __shared__ __attribute__((aligned(16))) char shared[];
  Few& s = *reinterpret_cast<Few*>(shared);
  const int tid = threadIdx.x;
  for (int i = tid; i < kFewWords; i += 1024) {
    s.used[i] = 0;
    if (SELECT) s.before[i] = 0x7fffffff;
  }
  int parent = -1, len = 0, held = 0;
  if (tid < p.m) {
    parent = SELECT ? p.parents[tid] : tid;
    if (parent < 0 || parent >= p.n) parent = -1;
    len = parent >= 0 ? length_of(p, parent) : 0;
    held = pages_of(p, len);
    s.parent[tid] = parent;
  }
  bool again = false;
  if constexpr (SELECT) {
    lds_barrier();
    if (parent >= 0) atomicMin(&s.before[parent], tid);
    lds_barrier();
    again = parent >= 0 && s.before[parent] < tid;
  }
  if (tid < p.m) s.held[tid] = again ? -held : held;
  lds_barrier();
  // ---- the places: what they name is in use (once for all rows of a parent)
  const int all = p.m * p.width;
  int page[kFewPlaces];
#pragma unroll
  for (int u = 0; u < kFewPlaces; ++u) {
    const int i = u * 1024 + tid, c = i / max(p.width, 1), col = i - c * p.width;
    page[u] = -1;
    if (i < all && col < abs(s.held[c])) page[u] = p.table[s.parent[c] * p.stride + col];
  }
#pragma unroll
  for (int u = 0; u < kFewPlaces; ++u) {
    const int i = u * 1024 + tid;
    if (page[u] >= 0 && page[u] < p.pool && s.held[i / max(p.width, 1)] > 0)
      atomicOr(&s.used[page[u] >> 5], 1u << (page[u] & 31));
  }
  lds_barrier();
  // ---- ranks: kFewWords / 1024 neighbouring words a thread
  constexpr int kWords = kFewWords / 1024;
  unsigned bits[kWords], n = 0, used;
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
    bits[u] = s.used[tid * kWords + u];
    n += __popc(bits[u]);
  }
  int rank = (int)block_scan(n, s.sums, &used);
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
    s.before[tid * kWords + u] = rank;
    rank += __popc(bits[u]);
  }
  lds_barrier();
  if constexpr (SELECT) {
    const bool flag = again && (len & ((1 << p.shift) - 1));
    unsigned needed;
    const int place = (int)block_scan(flag ? 1u : 0u, s.sums, &needed);
    const int n_free = p.pool - (int)used, taken = min((int)needed, n_free);
    // ---- free pages
    for (int i = tid; i < p.pool; i += 1024) {
      const unsigned word = s.used[i >> 5], e = i & 31;
      if (word >> e & 1u) continue;
      const int at = i - s.before[i >> 5] - __popc(word & ((1u << e) - 1u));
      if (at < taken) s.list[at] = i;
      else p.free_pages[at - taken] = i;
    }
    for (int i = n_free - taken + tid; i < p.pool; i += 1024) p.free_pages[i] = -1;
    for (int i = taken + tid; i < p.m; i += 1024) p.copies[2 * i] = -1, p.copies[2 * i + 1] = -1;
    lds_barrier();
    // ---- rows that need a copy: its place among them, or (behind the last free page) none of the row
    if (tid < p.m) {
      const bool out = flag && place >= taken;
      p.out_lengths[tid] = out ? 0 : len;
      s.held[tid] = out ? 0 : held;
      s.parent[tid] = flag && !out ? place : -1;
    }
    if (tid == 0) p.counts[0] = n_free - taken, p.counts[1] = taken, p.counts[2] = (int)needed - taken, p.counts[3] = p.pool - n_free + taken;
    lds_barrier();
#pragma unroll
    for (int u = 0; u < kFewPlaces; ++u) {
      const int i = u * 1024 + tid;
      if (i >= all) continue;
      const int c = i / p.width, col = i - c * p.width, place = s.parent[c];
      int x = col < s.held[c] ? page[u] : -1;
      if (place >= 0 && col == s.held[c] - 1) {
        p.copies[2 * place] = x;
        x = p.copies[2 * place + 1] = s.list[place];
      }
      p.out_table[c * p.out_stride + col] = x;
    }
  } else {
    const int k = (int)used;
    unsigned n_front = 0, stay;                            // in use in front of k: they stay
#pragma unroll
    for (int u = 0; u < kWords; ++u) {
      const int left = k - 32 * (tid * kWords + u);
      n_front += left >= 32 ? __popc(bits[u]) : left > 0 ? __popc(bits[u] & ((1u << left) - 1u)) : 0;
    }
    block_scan(n_front, s.sums, &stay);
    const int moves = k - (int)stay;
    for (int i = tid; i < p.pool; i += 1024) {
      const unsigned word = s.used[i >> 5], e = i & 31;
      const int before = s.before[i >> 5] + __popc(word & ((1u << e) - 1u));
      p.free_pages[i] = k + i < p.pool ? k + i : -1;
      if (word >> e & 1u) {
        if (i >= k) p.copies[2 * (before - (int)stay)] = i;
      } else if (i < k) {
        p.copies[2 * (i - before) + 1] = s.list[i - before] = i;
      }
    }
    for (int i = moves + tid; i < p.n_copies; i += 1024) p.copies[2 * i] = -1, p.copies[2 * i + 1] = -1;
    if (tid == 0) p.counts[0] = p.pool - k, p.counts[1] = moves, p.counts[2] = 0, p.counts[3] = k;
    lds_barrier();
#pragma unroll
    for (int u = 0; u < kFewPlaces; ++u) {
      const int i = u * 1024 + tid;
      if (i >= all) continue;
      const int c = i / p.width, col = i - c * p.width;
      int x = page[u];
      if (x >= k && x < p.pool) x = s.list[s.before[x >> 5] + __popc(s.used[x >> 5] & ((1u << (x & 31)) - 1u)) - (int)stay];
      p.out_table[c * p.out_stride + col] = x;
    }
  }
}

__global__ __launch_bounds__(256) void compact_mark_kernel(const PagesParams p) {
  const int b = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (b >= p.n) return;
  const int held = pages_of(p, length_of(p, b));
  for (int i = lane; i < held; i += 64) mark(p, p.table[b * p.stride + i]);
}

// Of the k pages in use, those at k and behind go to the free ones in front of k, both in ascending order.
__global__ __launch_bounds__(256) void compact_list_kernel(const PagesParams p) {
  __shared__ __attribute__((aligned(16))) unsigned sums[3][4], sums_of[2][4];
  __shared__ unsigned ranks[kBlockWords], words[kBlockWords];
  const int tid = threadIdx.x, page0 = blockIdx.x * kBlockPages;
  const unsigned bits = tid < kBlockWords && blockIdx.x < p.blocks ? p.used[blockIdx.x * kBlockWords + tid] : 0;
  unsigned v[3] = {0, 0, (unsigned)__popc(bits)}, before[3], total[3];
  count_used(p, blockIdx.x, &v[0], &v[1]);
  block_scans(v, sums, before, total);
  const int k = (int)total[0], rank0 = (int)(total[1] + before[2]);
  // in use in front of k: they stay
  const int of = k / kBlockPages, left = k - of * kBlockPages - 32 * tid;        // (of k's block, to this thread's word)
  unsigned in_front[2] = {0, 0}, front_before[2], front[2], all;
  count_used(p, of, &all, &in_front[0]);
  if (tid < kBlockWords && of < p.blocks && left > 0) {
    const unsigned n = p.used[of * kBlockWords + tid];
    in_front[1] = __popc(left >= 32 ? n : n & ((1u << left) - 1u));
  }
  block_scans(in_front, sums_of, front_before, front);
  const int stay = (int)(front[0] + front[1]), moves = k - stay;
  if (tid < kBlockWords) {
    if (blockIdx.x < p.blocks) p.before[blockIdx.x * kBlockWords + tid] = rank0;
    ranks[tid] = (unsigned)rank0, words[tid] = bits;
  }
  lds_barrier();
#pragma unroll
  for (int i = tid; i < kBlockPages; i += 256) {
    const unsigned word = words[i >> 5], e = i & 31;
    const int page = page0 + i, before = (int)ranks[i >> 5] + __popc(word & ((1u << e) - 1u));
    if (page >= p.pool) break;
    p.free_pages[page] = k + page < p.pool ? k + page : -1;
    if (word >> e & 1u) {
      if (page >= k) p.copies[2 * (before - stay)] = page;
    } else if (page < k) {
      p.copies[2 * (page - before) + 1] = page;
    }
  }
  for (int i = blockIdx.x * 256 + tid; i < p.n_copies; i += gridDim.x * 256)
    if (i >= moves) p.copies[2 * i] = -1, p.copies[2 * i + 1] = -1;
  if (blockIdx.x == 0 && tid == 0) p.counts[0] = p.pool - k, p.counts[1] = moves, p.counts[2] = 0, p.counts[3] = k;
}

__global__ __launch_bounds__(256) void compact_rows_kernel(const PagesParams p) {
  const int b = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (b >= p.n) return;
  const int held = pages_of(p, length_of(p, b)), k = p.counts[3], stay = k - p.counts[1];
  for (int i = lane; i < p.width; i += 64) {
    int page = i < held ? p.table[b * p.stride + i] : -1;
    if (page >= k && page < p.pool) {
      const int rank = p.before[page >> 5] + __popc(p.used[page >> 5] & ((1u << (page & 31)) - 1u));
      page = p.copies[2 * (rank - stay) + 1];
    }
    p.out_table[b * p.out_stride + i] = page;
  }
}

// A block copies 4 KB of a page at a time, 16 bytes a thread, from the pairs in turn.  (16 KB a block, four loads a thread behind a
// test each: 1500 pages of 17 KB 24 us instead of 10.)
constexpr size_t kCopyBytes = 4096;
constexpr unsigned kCopyBlocks = 8192;
__global__ __launch_bounds__(256) void page_copy_kernel(char* __restrict__ cache, size_t page_bytes, int pool,
                                                        const int2* __restrict__ pairs, size_t items, int chunks) {
  for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
    const size_t pair = item / (unsigned)chunks, at = (item - pair * chunks) * kCopyBytes + threadIdx.x * 16;
    const int2 of = pairs[pair];
    if (of.x < 0 || of.x >= pool || of.y < 0 || of.y >= pool || of.x == of.y || at >= page_bytes) continue;
    *reinterpret_cast<uint4*>(cache + of.y * page_bytes + at) = *reinterpret_cast<const uint4*>(cache + of.x * page_bytes + at);
  }
}

size_t round_up(size_t a, size_t b) { return (a + b - 1) / b * b; }
size_t blocks_of(size_t n_pages) { return (n_pages + kBlockPages - 1) / kBlockPages; }
// Workspace: marks, bits, numbers in front of words, of blocks; rows' flags, and their parents' first rows.
struct Space {
  size_t used, before, counts, flags, first, bytes;
  Space(size_t rows, size_t n_pages) {
    const size_t blocks = blocks_of(n_pages), words = blocks * kBlockWords * 4;
    used = blocks * kBlockPages, before = used + words, counts = before + words;
    flags = counts + round_up(blocks * 4, 256), first = flags + round_up(rows * 4, 256);
    bytes = first + round_up(rows * 4, 256);
  }
  void set(PagesParams* p, void* workspace) const {
    char* const at = static_cast<char*>(workspace);
    p->marks = reinterpret_cast<uint8_t*>(at);
    p->used = reinterpret_cast<unsigned*>(at + used);
    p->before = reinterpret_cast<int*>(at + before);
    p->counts_of = reinterpret_cast<unsigned*>(at + counts);
    p->flags = reinterpret_cast<uint8_t*>(at + flags);
  }
};

// More new rows than this have their parents' first ones found by a launch of its own.  (us with and without it, tables of up to 256
// places: 1200 rows 18.4 and 17.9, 2000 18.6 and 18.7, 2400 21.0 and 20.8, 3000 21.2 and 21.7, 4000 21.2 and 24.4, 9000 30 and 44.)
constexpr int kSearched = 2400;

template <bool SELECT>
int launch_few(const PagesParams& p, hipStream_t stream) {
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&pages_few_kernel<SELECT>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Few));
  if (attr != hipSuccess) return Q8_EHIP;
  pages_few_kernel<SELECT><<<1, 1024, sizeof(Few), stream>>>(p);
  return q8_launch_status();
}

// Memory from a table's first place to behind its last one, and whether two have any in common.
struct Span {
  const int *begin, *end;
  Span(const int* at, size_t rows, size_t stride, size_t width) : begin(at), end(rows && width ? at + (rows - 1) * stride + width : at) {}
  Span(const int* at, size_t n) : begin(at), end(at + n) {}
  bool meets(const Span& o) const { return begin < o.end && o.begin < end && begin != end && o.begin != o.end; }
};

}  // namespace

extern "C" size_t q8_page_workspace_bytes(int n_rows, size_t n_pages) {
  if (n_rows < 0 || n_pages > (size_t)kMostPages) return 0;
  return Space(n_rows, n_pages).bytes;
}

extern "C" int q8_page_select(const int32_t* parents_dev, int n_new, const int32_t* lengths_dev, const int32_t* table_dev,
                              size_t table_stride, int n_requests, int width, int page, size_t n_pages,
                              int32_t* out_table_dev, size_t out_stride, int32_t* out_lengths_dev, int32_t* free_pages_dev,
                              int32_t* copies_dev, int32_t* counts_dev, void* workspace, size_t workspace_bytes,
                              void* stream) {
  Q8_REQUIRE(n_new >= 0 && n_requests >= 0 && width >= 0, Q8_EINVAL);
  Q8_REQUIRE(kv4_page_ok(page) && n_pages <= (size_t)kMostPages && (size_t)width * page <= 0x7fff0000u &&
                 n_new <= kMostRows && n_requests <= kMostRows, Q8_EUNSUPPORTED);
  Q8_REQUIRE(counts_dev && (workspace || n_pages + n_new + n_requests == 0) && (n_pages == 0 || free_pages_dev), Q8_EINVAL);
  Q8_REQUIRE(n_new == 0 || (parents_dev && out_lengths_dev && copies_dev && (out_table_dev || width == 0)), Q8_EINVAL);
  Q8_REQUIRE(n_requests == 0 || (lengths_dev && (table_dev || width == 0)), Q8_EINVAL);
  Q8_REQUIRE(table_stride >= (size_t)width && out_stride >= (size_t)width, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(parents_dev, 4) && q8_aligned(lengths_dev, 4) && q8_aligned(table_dev, 4) &&
                 q8_aligned(out_table_dev, 4) && q8_aligned(out_lengths_dev, 4) && q8_aligned(free_pages_dev, 4) &&
                 q8_aligned(copies_dev, 4) && q8_aligned(counts_dev, 4) && q8_aligned(workspace, 16), Q8_EALIGN);
  Q8_REQUIRE(workspace_bytes >= q8_page_workspace_bytes(n_new > n_requests ? n_new : n_requests, n_pages), Q8_EWORKSPACE);
  const Span reads[] = {{parents_dev, (size_t)n_new}, {lengths_dev, (size_t)n_requests},
                        {table_dev, (size_t)n_requests, table_stride, (size_t)width}};
  for (const Span& in : reads)
    Q8_REQUIRE(!in.meets({out_table_dev, (size_t)n_new, out_stride, (size_t)width}) && !in.meets({out_lengths_dev, (size_t)n_new}) &&
                   !in.meets({free_pages_dev, n_pages}) && !in.meets({copies_dev, 2 * (size_t)n_new}) && !in.meets({counts_dev, 4}),
               Q8_EINVAL);
  PagesParams p{};
  p.parents = parents_dev, p.lengths = lengths_dev, p.table = table_dev, p.out_table = out_table_dev;
  p.out_lengths = out_lengths_dev, p.free_pages = free_pages_dev, p.copies = copies_dev, p.counts = counts_dev;
  const Space space(n_new > n_requests ? n_new : n_requests, n_pages);
  space.set(&p, workspace);
  p.before = n_new > kSearched ? reinterpret_cast<int*>(static_cast<char*>(workspace) + space.first) : nullptr;
  p.stride = table_stride, p.out_stride = out_stride;
  p.n = n_requests, p.m = n_new, p.shift = __builtin_ctz(page), p.width = width, p.pool = (int)n_pages;
  p.blocks = (int)blocks_of(n_pages), p.n_copies = n_new;
  const hipStream_t s = (hipStream_t)stream;
  if (few(n_new, n_requests, width, n_pages)) return launch_few<true>(p, s);
  const size_t marks = (size_t)p.blocks * kBlockPages / 16, first = p.before ? n_requests : 0;
  if (marks || first)
    pages_clear_kernel<<<(unsigned)(((marks > first ? marks : first) + 255) / 256), 256, 0, s>>>(
        reinterpret_cast<uint4*>(p.marks), marks, p.before, (int)first);
  if (p.before) select_first_kernel<<<(unsigned)(((size_t)n_new + 255) / 256), 256, 0, s>>>(p);
  if (n_new) select_rows_kernel<<<(unsigned)(((size_t)n_new + 3) / 4), 256, 0, s>>>(p);
  if (p.blocks) pages_count_kernel<<<p.blocks, 256, 0, s>>>(p);
  select_free_kernel<<<p.blocks ? p.blocks : 1, 256, 0, s>>>(p);
  return q8_launch_status();
}

extern "C" int q8_page_compact(const int32_t* lengths_dev, const int32_t* table_dev, size_t table_stride, int n_requests,
                               int width, int page, size_t n_pages, int32_t* out_table_dev, size_t out_stride,
                               int32_t* free_pages_dev, int32_t* copies_dev, int32_t* counts_dev, void* workspace,
                               size_t workspace_bytes, void* stream) {
  Q8_REQUIRE(n_requests >= 0 && width >= 0, Q8_EINVAL);
  Q8_REQUIRE(kv4_page_ok(page) && n_pages <= (size_t)kMostPages && (size_t)width * page <= 0x7fff0000u &&
                 n_requests <= kMostRows, Q8_EUNSUPPORTED);
  Q8_REQUIRE(counts_dev && (n_pages == 0 || (workspace && free_pages_dev)) && (n_pages < 2 || copies_dev), Q8_EINVAL);
  Q8_REQUIRE(n_requests == 0 || (lengths_dev && ((table_dev && out_table_dev) || width == 0)), Q8_EINVAL);
  Q8_REQUIRE(table_stride >= (size_t)width && out_stride >= (size_t)width, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(lengths_dev, 4) && q8_aligned(table_dev, 4) && q8_aligned(out_table_dev, 4) &&
                 q8_aligned(free_pages_dev, 4) && q8_aligned(copies_dev, 4) && q8_aligned(counts_dev, 4) &&
                 q8_aligned(workspace, 16), Q8_EALIGN);
  Q8_REQUIRE(workspace_bytes >= q8_page_workspace_bytes(0, n_pages), Q8_EWORKSPACE);
  const Span lengths{lengths_dev, (size_t)n_requests}, table{table_dev, (size_t)n_requests, table_stride, (size_t)width},
      out{out_table_dev, (size_t)n_requests, out_stride, (size_t)width};
  Q8_REQUIRE((table_dev == out_table_dev && (table_stride == out_stride || n_requests < 2)) || !table.meets(out), Q8_EINVAL);
  Q8_REQUIRE(!lengths.meets(out), Q8_EINVAL);
  for (const Span& in : {lengths, table})
    Q8_REQUIRE(!in.meets({free_pages_dev, n_pages}) && !in.meets({copies_dev, n_pages / 2 * 2}) && !in.meets({counts_dev, 4}), Q8_EINVAL);
  PagesParams p{};
  p.lengths = lengths_dev, p.table = table_dev, p.out_table = out_table_dev;
  p.free_pages = free_pages_dev, p.copies = copies_dev, p.counts = counts_dev;
  Space(0, n_pages).set(&p, workspace);
  p.stride = table_stride, p.out_stride = out_stride;
  p.n = p.m = n_requests, p.shift = __builtin_ctz(page), p.width = width, p.pool = (int)n_pages;
  p.blocks = (int)blocks_of(n_pages), p.n_copies = (int)(n_pages / 2);
  const hipStream_t s = (hipStream_t)stream;
  if (few(n_requests, 0, width, n_pages)) return launch_few<false>(p, s);
  const unsigned rows = (unsigned)(((size_t)n_requests + 3) / 4);
  const size_t marks = (size_t)p.blocks * kBlockPages / 16;
  if (marks) pages_clear_kernel<<<(unsigned)((marks + 255) / 256), 256, 0, s>>>(reinterpret_cast<uint4*>(p.marks), marks, nullptr, 0);
  if (rows) compact_mark_kernel<<<rows, 256, 0, s>>>(p);
  if (p.blocks) pages_count_kernel<<<p.blocks, 256, 0, s>>>(p);
  compact_list_kernel<<<p.blocks ? p.blocks : 1, 256, 0, s>>>(p);
  if (rows) compact_rows_kernel<<<rows, 256, 0, s>>>(p);
  return q8_launch_status();
}

extern "C" int q8_page_copy(void* cache_dev, size_t n_pages, size_t page_bytes, const int32_t* pairs_dev, int n_pairs,
                            void* stream) {
  Q8_REQUIRE(n_pairs >= 0, Q8_EINVAL);
  Q8_REQUIRE(n_pages <= 0x7fffffffu && page_bytes < (size_t)1 << 40, Q8_EUNSUPPORTED);
  if (n_pairs == 0 || n_pages == 0 || page_bytes == 0) return Q8_OK;
  Q8_REQUIRE(cache_dev && pairs_dev, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(cache_dev, 16) && page_bytes % 16 == 0 && q8_aligned(pairs_dev, 8), Q8_EALIGN);
  const size_t chunks = (page_bytes + kCopyBytes - 1) / kCopyBytes, items = chunks * n_pairs;
  page_copy_kernel<<<(unsigned)(items < kCopyBlocks ? items : kCopyBlocks), 256, 0, (hipStream_t)stream>>>(
      static_cast<char*>(cache_dev), page_bytes, (int)n_pages, reinterpret_cast<const int2*>(pairs_dev), items, (int)chunks);
  return q8_launch_status();
}
