// The pages of a cache, whatever they hold: requests that go on, several times or not at all (q8_page_select), the pages in
// use moved to the front of the pool (q8_page_compact), and pages copied (q8_page_copy).
//
// Which pages are in use is one bit a page, set from the rows that are kept; every number that a page or a request gets is
// its rank among bits or flags, in ascending order, so that results do not depend on which block came first.
#include "q8_kv4.h"
#pragma clang fp contract(off)

namespace {

using namespace q8;

constexpr int kMostPages = 1 << 24;
constexpr int kBlockWords = 256;               // words of 32 pages that a block lists

struct PagesParams {
  const int* __restrict__ parents;             // null: row c goes on as row c
  const int* __restrict__ lengths;
  const int* table;                            // (compact: may be out_table)
  int* out_table;
  int* __restrict__ out_lengths;
  int* __restrict__ free_pages;
  int* __restrict__ copies;                    // [n_copies][2]
  int* __restrict__ counts;
  unsigned* __restrict__ used;                 // [words]
  int* __restrict__ before;                    // compact: of each word, pages in use before it
  unsigned* __restrict__ flags;                // select: of each new row, whether it needs a copy of its last page
  size_t stride, out_stride;
  int n, m, shift, width, pool, words, n_copies;           // old rows, new rows; shift: page = 1 << shift tokens
};

__device__ __forceinline__ int length_of(const PagesParams& p, int b) {
  return (int)min((long)max(p.lengths[b], 0), (long)p.width << p.shift);
}
__device__ __forceinline__ int pages_of(const PagesParams& p, int tokens) {
  return (int)(((long)tokens + (1 << p.shift) - 1) >> p.shift);
}

// Sum over a block of 256.
__device__ __forceinline__ long block_sum(long v, long (&sums)[4]) {
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sums[0] + sums[1]) + (sums[2] + sums[3]);
}
// Sums before a thread, and of the block of 256.
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned (&sums)[4], unsigned* total) {
  const unsigned upto = scan64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = upto;
  __syncthreads();
  unsigned base = 0;
  for (unsigned w = 0; w < threadIdx.x >> 6; ++w) base += sums[w];
  *total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  return base + upto - v;
}

__global__ __launch_bounds__(256) void pages_clear_kernel(unsigned* used, int words) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < words) used[i] = 0;
}

__device__ __forceinline__ void mark(const PagesParams& p, int page) {
  if (page >= 0 && page < p.pool) atomicOr(&p.used[page >> 5], 1u << (page & 31));
}

// A wavefront takes a new row: its parent's places, whose pages are in use.  Of several rows of a parent, the first has its
// last page for itself; the others need a copy of it unless it is full.
__global__ __launch_bounds__(256) void select_rows_kernel(const PagesParams p) {
  const int c = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (c >= p.m) return;
  const int parent = p.parents[c];
  const bool given = parent >= 0 && parent < p.n;
  bool again = false;
  for (int i = 0; given && i < c && !again; i += 64) again = __any(i + lane < c && p.parents[i + lane] == parent);
  const int len = given ? length_of(p, parent) : 0, held = pages_of(p, len);
  const int* const from = p.table + (given ? parent : 0) * p.stride;
  int* const to = p.out_table + c * p.out_stride;
  for (int i = lane; i < p.width; i += 64) {
    const int page = i < held ? from[i] : -1;
    to[i] = page;
    if (!again) mark(p, page);
  }
  if (lane == 0) {
    p.out_lengths[c] = len;
    p.flags[c] = again && (len & ((1 << p.shift) - 1));
  }
}

// Free pages in order: the first of them become copies, of the rows that need one in their order; the others are listed.  Rows
// that find none become empty.
__global__ __launch_bounds__(256) void select_free_kernel(const PagesParams p) {
  __shared__ long sums[4];
  __shared__ unsigned scans[4];
  __shared__ int list[kBlockWords * 32];
  const int tid = threadIdx.x, word0 = blockIdx.x * kBlockWords;
  long all = 0, mine = 0, needed = 0;
  for (int i = tid; i < p.words; i += 256) {
    const int n = 32 - __popc(p.used[i]) - max(0, 32 * (i + 1) - p.pool);      // (bits behind the pool are never set)
    all += n;
    if (i < word0) mine += n;
  }
  for (int i = tid; i < p.m; i += 256) needed += p.flags[i];
  const int n_free = (int)block_sum(all, sums), first = (int)block_sum(mine, sums), n_needed = (int)block_sum(needed, sums);
  const int taken = min(n_needed, n_free);
  // ---- this block's free pages
  unsigned bits = 0;
  if (word0 + tid < p.words) {
    bits = ~p.used[word0 + tid];
    const int behind = 32 * (word0 + tid + 1) - p.pool;
    if (behind > 0) bits &= 0xffffffffu >> behind;
  }
  unsigned here;
  int at = (int)block_scan(__popc(bits), scans, &here);
  const int end = first + (int)here;
  for (; bits; bits &= bits - 1, ++at) {
    const int page = 32 * (word0 + tid) + __builtin_ctz(bits);
    list[at] = page;
    if (first + at >= taken) p.free_pages[first + at - taken] = page;
  }
  __syncthreads();
  // ---- places behind the last of the lists
  for (int i = word0 * 32 + tid; i < min((word0 + kBlockWords) * 32, p.pool); i += 256)
    if (i >= n_free - taken) p.free_pages[i] = -1;
  for (int i = blockIdx.x * 256 + tid; i < p.m; i += gridDim.x * 256)
    if (i >= taken) p.copies[2 * i] = -1, p.copies[2 * i + 1] = -1;
  if (blockIdx.x == 0 && tid == 0) {
    p.counts[0] = n_free - taken, p.counts[1] = taken, p.counts[2] = n_needed - taken, p.counts[3] = p.pool - n_free + taken;
  }
  // ---- rows that need a copy: of rank first .. end - 1 here; the last block empties those behind the last free page
  const bool empties = blockIdx.x == gridDim.x - 1 && n_needed > n_free;
  if (first >= taken && !empties) return;
  int rank0 = 0;
  for (int c0 = 0; c0 < p.m; c0 += 256) {
    const int c = c0 + tid;
    const unsigned flag = c < p.m ? p.flags[c] : 0;
    unsigned n;
    const int rank = rank0 + (int)block_scan(flag, scans, &n);
    if (flag && rank >= first && rank < end && rank < taken) {
      int* const entry = p.out_table + c * p.out_stride + pages_of(p, p.out_lengths[c]) - 1;
      p.copies[2 * rank] = *entry;
      *entry = p.copies[2 * rank + 1] = list[rank - first];
    }
    if (flag && empties && rank >= n_free) {
      for (int i = 0; i < p.width; ++i) p.out_table[c * p.out_stride + i] = -1;
      p.out_lengths[c] = 0;
    }
    rank0 += (int)n;
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
  __shared__ long sums[4];
  __shared__ unsigned scans[4];
  const int tid = threadIdx.x, word0 = blockIdx.x * kBlockWords;
  long all = 0, mine = 0;
  for (int i = tid; i < p.words; i += 256) {
    const int n = __popc(p.used[i]);
    all += n;
    if (i < word0) mine += n;
  }
  const int k = (int)block_sum(all, sums), first = (int)block_sum(mine, sums);
  long front = 0;                                          // in use in front of k: they stay
  for (int i = tid; i <= k >> 5 && i < p.words; i += 256)
    front += __popc(i < k >> 5 ? p.used[i] : p.used[i] & ((1u << (k & 31)) - 1u));
  const int stay = (int)block_sum(front, sums), moves = k - stay;
  const unsigned bits = word0 + tid < p.words ? p.used[word0 + tid] : 0;
  unsigned here;
  int rank = first + (int)block_scan(__popc(bits), scans, &here);
  if (word0 + tid < p.words) p.before[word0 + tid] = rank;
  for (int e = 0; e < 32; ++e) {
    const int page = 32 * (word0 + tid) + e;
    if (page >= p.pool) break;
    if (bits >> e & 1u) {
      if (page >= k) p.copies[2 * (rank - stay)] = page;
      ++rank;
    } else if (page < k) {
      p.copies[2 * (page - rank) + 1] = page;
    }
    p.free_pages[page] = k + page < p.pool ? k + page : -1;
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

// A block copies 16 KB of a page at a time, from the pairs in turn.
constexpr size_t kCopyBytes = 16384;
__global__ __launch_bounds__(256) void page_copy_kernel(char* __restrict__ cache, size_t page_bytes, int pool,
                                                        const int* __restrict__ pairs, size_t items, int chunks) {
  for (size_t item = blockIdx.x; item < items; item += gridDim.x) {
    const size_t pair = item / chunks;
    const size_t at = (item - pair * chunks) * kCopyBytes + threadIdx.x * 16;
    const int from = pairs[2 * pair], to = pairs[2 * pair + 1];
    if (from < 0 || from >= pool || to < 0 || to >= pool || from == to) continue;
    const char* const src = cache + from * page_bytes;
    char* const dst = cache + to * page_bytes;
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at + u * 4096 < page_bytes) v[u] = *reinterpret_cast<const uint4*>(src + at + u * 4096);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at + u * 4096 < page_bytes) *reinterpret_cast<uint4*>(dst + at + u * 4096) = v[u];
  }
}

size_t round_up(size_t a, size_t b) { return (a + b - 1) / b * b; }
size_t words_of(size_t n_pages) { return (n_pages + 31) / 32; }

// Whether two tables of n and m rows, `width` entries each, have places in common.
bool overlap(const int* a, int n, size_t a_stride, const int* b, int m, size_t b_stride, int width) {
  if (n == 0 || m == 0 || width == 0) return false;
  const int *a_end = a + (n - 1) * a_stride + width, *b_end = b + (m - 1) * b_stride + width;
  return a < b_end && b < a_end;
}

}  // namespace

extern "C" size_t q8_page_workspace_bytes(int n_rows, size_t n_pages) {
  if (n_rows < 0 || n_pages > (size_t)kMostPages) return 0;
  return round_up(words_of(n_pages) * 4, 256) + round_up((words_of(n_pages) > (size_t)n_rows ? words_of(n_pages) : n_rows) * 4, 256);
}

extern "C" int q8_page_select(const int32_t* parents_dev, int n_new, const int32_t* lengths_dev, const int32_t* table_dev,
                              size_t table_stride, int n_requests, int width, int page, size_t n_pages,
                              int32_t* out_table_dev, size_t out_stride, int32_t* out_lengths_dev, int32_t* free_pages_dev,
                              int32_t* copies_dev, int32_t* counts_dev, void* workspace, size_t workspace_bytes,
                              void* stream) {
  Q8_REQUIRE(n_new >= 0 && n_requests >= 0 && width >= 0, Q8_EINVAL);
  Q8_REQUIRE(kv4_page_ok(page) && n_pages <= (size_t)kMostPages && (size_t)width * page <= 0x7fff0000u, Q8_EUNSUPPORTED);
  Q8_REQUIRE(counts_dev && (workspace || n_pages + n_new == 0) && (n_pages == 0 || free_pages_dev), Q8_EINVAL);
  Q8_REQUIRE(n_new == 0 || (parents_dev && out_lengths_dev && copies_dev && (out_table_dev || width == 0)), Q8_EINVAL);
  Q8_REQUIRE(n_requests == 0 || (lengths_dev && (table_dev || width == 0)), Q8_EINVAL);
  Q8_REQUIRE(table_stride >= (size_t)width && out_stride >= (size_t)width, Q8_EINVAL);
  Q8_REQUIRE(!overlap(table_dev, n_requests, table_stride, out_table_dev, n_new, out_stride, width), Q8_EINVAL);
  Q8_REQUIRE(!overlap(lengths_dev, 1, 0, out_lengths_dev, 1, 0, n_requests < n_new ? n_requests : n_new), Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(parents_dev, 4) && q8_aligned(lengths_dev, 4) && q8_aligned(table_dev, 4) &&
                 q8_aligned(out_table_dev, 4) && q8_aligned(out_lengths_dev, 4) && q8_aligned(free_pages_dev, 4) &&
                 q8_aligned(copies_dev, 4) && q8_aligned(counts_dev, 4) && q8_aligned(workspace, 16), Q8_EALIGN);
  Q8_REQUIRE(workspace_bytes >= q8_page_workspace_bytes(n_new, n_pages), Q8_EWORKSPACE);
  PagesParams p{};
  p.parents = parents_dev, p.lengths = lengths_dev, p.table = table_dev, p.out_table = out_table_dev;
  p.out_lengths = out_lengths_dev, p.free_pages = free_pages_dev, p.copies = copies_dev, p.counts = counts_dev;
  p.used = static_cast<unsigned*>(workspace);
  p.flags = p.used + round_up(words_of(n_pages) * 4, 256) / 4;
  p.stride = table_stride, p.out_stride = out_stride;
  p.n = n_requests, p.m = n_new, p.shift = __builtin_ctz(page), p.width = width, p.pool = (int)n_pages;
  p.words = (int)words_of(n_pages), p.n_copies = n_new;
  const hipStream_t s = (hipStream_t)stream;
  if (p.words) pages_clear_kernel<<<(p.words + 255) / 256, 256, 0, s>>>(p.used, p.words);
  if (n_new) select_rows_kernel<<<(unsigned)(((size_t)n_new + 3) / 4), 256, 0, s>>>(p);
  select_free_kernel<<<p.words ? (p.words + kBlockWords - 1) / kBlockWords : 1, 256, 0, s>>>(p);
  return q8_launch_status();
}

extern "C" int q8_page_compact(const int32_t* lengths_dev, const int32_t* table_dev, size_t table_stride, int n_requests,
                               int width, int page, size_t n_pages, int32_t* out_table_dev, size_t out_stride,
                               int32_t* free_pages_dev, int32_t* copies_dev, int32_t* counts_dev, void* workspace,
                               size_t workspace_bytes, void* stream) {
  Q8_REQUIRE(n_requests >= 0 && width >= 0, Q8_EINVAL);
  Q8_REQUIRE(kv4_page_ok(page) && n_pages <= (size_t)kMostPages && (size_t)width * page <= 0x7fff0000u, Q8_EUNSUPPORTED);
  Q8_REQUIRE(counts_dev && (n_pages == 0 || (workspace && free_pages_dev)) && (n_pages < 2 || copies_dev), Q8_EINVAL);
  Q8_REQUIRE(n_requests == 0 || (lengths_dev && ((table_dev && out_table_dev) || width == 0)), Q8_EINVAL);
  Q8_REQUIRE(table_stride >= (size_t)width && out_stride >= (size_t)width, Q8_EINVAL);
  Q8_REQUIRE((table_dev == out_table_dev && (table_stride == out_stride || n_requests < 2)) ||
                 !overlap(table_dev, n_requests, table_stride, out_table_dev, n_requests, out_stride, width), Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(lengths_dev, 4) && q8_aligned(table_dev, 4) && q8_aligned(out_table_dev, 4) &&
                 q8_aligned(free_pages_dev, 4) && q8_aligned(copies_dev, 4) && q8_aligned(counts_dev, 4) &&
                 q8_aligned(workspace, 16), Q8_EALIGN);
  Q8_REQUIRE(workspace_bytes >= q8_page_workspace_bytes(0, n_pages), Q8_EWORKSPACE);
  PagesParams p{};
  p.lengths = lengths_dev, p.table = table_dev, p.out_table = out_table_dev;
  p.free_pages = free_pages_dev, p.copies = copies_dev, p.counts = counts_dev;
  p.used = static_cast<unsigned*>(workspace);
  p.before = static_cast<int*>(workspace) + round_up(words_of(n_pages) * 4, 256) / 4;
  p.stride = table_stride, p.out_stride = out_stride;
  p.n = p.m = n_requests, p.shift = __builtin_ctz(page), p.width = width, p.pool = (int)n_pages;
  p.words = (int)words_of(n_pages), p.n_copies = (int)(n_pages / 2);
  const hipStream_t s = (hipStream_t)stream;
  const unsigned rows = (unsigned)(((size_t)n_requests + 3) / 4);
  if (p.words) pages_clear_kernel<<<(p.words + 255) / 256, 256, 0, s>>>(p.used, p.words);
  if (rows) compact_mark_kernel<<<rows, 256, 0, s>>>(p);
  compact_list_kernel<<<p.words ? (p.words + kBlockWords - 1) / kBlockWords : 1, 256, 0, s>>>(p);
  if (rows) compact_rows_kernel<<<rows, 256, 0, s>>>(p);
  return q8_launch_status();
}

extern "C" int q8_page_copy(void* cache_dev, size_t n_pages, size_t page_bytes, const int32_t* pairs_dev, int n_pairs,
                            void* stream) {
  Q8_REQUIRE(n_pairs >= 0, Q8_EINVAL);
  Q8_REQUIRE(n_pages <= 0x7fffffffu && page_bytes < (size_t)1 << 40, Q8_EUNSUPPORTED);
  if (n_pairs == 0 || n_pages == 0 || page_bytes == 0) return Q8_OK;
  Q8_REQUIRE(cache_dev && pairs_dev, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(cache_dev, 16) && page_bytes % 16 == 0 && q8_aligned(pairs_dev, 4), Q8_EALIGN);
  const size_t chunks = (page_bytes + kCopyBytes - 1) / kCopyBytes, items = chunks * n_pairs;
  page_copy_kernel<<<(unsigned)(items < 4096 ? items : 4096), 256, 0, (hipStream_t)stream>>>(
      static_cast<char*>(cache_dev), page_bytes, (int)n_pages, pairs_dev, items, (int)chunks);
  return q8_launch_status();
}
