// The paged 4-bit cache of keys and values: block tables and slots from request lengths, tokens in, tokens out.
// (Attention over it: q8_kv4_attend.hip.)
//
// A group of 32 channels of one token's head is held by Eq. Q with p = 3 at the factor q = binary16(max|r| * fl(1/7)).
// Sixteen tokens of a head are 18 D bytes (q8_kv4.h): key codes by token, value codes by channel, so that both are
// operands of a matrix instruction as they lie.
#include "q8_kv4.h"
#include "q8_quant.h"
#pragma clang fp contract(off)

namespace {

using namespace q8;

// ---------------------------------------------------------------- block tables -----------
// A request with `len` tokens in the cache gets `add` more: its pages are counted and handed out in request order.
// One block walks over the requests, 1024 at a time, with the running sums of pages and of tokens.
struct PageParams {
  const int* __restrict__ lengths;
  const int* __restrict__ added;
  const int* __restrict__ free_pages;
  int* __restrict__ table;
  long* __restrict__ slots;
  int* __restrict__ positions;
  int* __restrict__ starts;
  int* __restrict__ grown;
  int* __restrict__ counts;
  int n, shift, n_free, width, n_slots;      // shift: page = 1 << shift tokens
  size_t table_stride;
};

__device__ __forceinline__ int pages_of(long tokens, int shift) { return (int)((tokens + (1 << shift) - 1) >> shift); }

__global__ __launch_bounds__(1024) void page_rows_kernel(const PageParams p) {
  __shared__ long tok_sum[16], page_sum[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  long tok_base = 0, page_base = 0, taken = 0;
  int refused = 0;
  auto inclusive = [&](long v, long* sums) {              // over the block
    for (int off = 1; off < 64; off <<= 1) {
      const long o = __shfl_up(v, off, 64);
      if (lane >= off) v += o;
    }
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += sums[w];
    return v;
  };
  for (int b0 = 0; b0 < p.n; b0 += 1024) {
    const int b = b0 + tid;
    const long len = b < p.n ? max(p.lengths[b], 0) : 0, add = b < p.n ? max(p.added[b], 0) : 0;
    const long end = tok_base + inclusive(add, tok_sum);
    const int have = pages_of(len, p.shift), total = pages_of(len + add, p.shift);
    const bool out = total > p.width || end > p.n_slots;
    const long need = out ? 0 : total - have;
    const long upto = page_base + inclusive(need, page_sum);
    const bool fits = !out && (need == 0 || upto <= p.n_free);
    if (b < p.n) {
      p.starts[b] = (int)(end - add);
      p.grown[b] = (int)(len + (fits ? add : 0));
      if (b == p.n - 1) p.starts[p.n] = (int)end;
      if (fits)
        for (int i = 0; i < need; ++i) p.table[b * p.table_stride + have + i] = p.free_pages[upto - need + i];
      taken += fits ? need : 0;
      refused += !fits;
    }
    __syncthreads();                                       // the sums are read before they are written again
    if (tid == 1023) tok_sum[0] = end, page_sum[0] = upto;
    __syncthreads();
    tok_base = tok_sum[0];
    page_base = page_sum[0];
    __syncthreads();
  }
  for (int off = 32; off > 0; off >>= 1) {
    taken += __shfl_xor(taken, off, 64);
    refused += __shfl_xor(refused, off, 64);
  }
  if (lane == 0) tok_sum[wave] = taken, page_sum[wave] = refused;
  __syncthreads();
  if (tid == 0) {
    long t = 0, r = 0;
    for (int w = 0; w < 16; ++w) t += tok_sum[w], r += page_sum[w];
    p.counts[0] = (int)t;
    p.counts[1] = (int)tok_base;
    p.counts[2] = (int)r;
    if (p.n == 0) p.starts[0] = 0;
  }
}

// A thread per slot: its request by bisection of the starts.
__global__ __launch_bounds__(256) void page_slots_kernel(const PageParams p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= p.n_slots) return;
  long slot = -1;
  int position = -1;
  if (p.n > 0 && i < p.starts[p.n]) {
    int lo = 0, hi = p.n - 1;                              // the last request that starts at i or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.starts[mid] <= i) lo = mid; else hi = mid - 1;
    }
    const int len = max(p.lengths[lo], 0);
    if (p.grown[lo] > len) {
      position = len + i - p.starts[lo];
      const int page = p.table[lo * p.table_stride + (position >> p.shift)];
      slot = ((long)page << p.shift) + (position & ((1 << p.shift) - 1));
    }
  }
  p.slots[i] = slot;
  p.positions[i] = position;
}

// ---------------------------------------------------------------- tokens in and out ------
struct Kv4Params {
  const long* __restrict__ slots;
  uint8_t* __restrict__ cache;
  size_t k_stride, k_head, v_stride, v_head;    // elements between tokens and between heads
  long n_slots;                                 // of the cache
  int T, H, G, shift;                           // shift: page = 1 << shift tokens
};

// Sixteen of a slot and head, and the token's place in it.
__device__ __forceinline__ uint8_t* sixteen_of(const Kv4Params& p, long slot, int head, int* t) {
  const long page = slot >> p.shift;
  const int in = (int)(slot & ((1 << p.shift) - 1));
  *t = in & 15;
  return p.cache + ((((size_t)page * p.H + head) << (p.shift - 4)) + (in >> 4)) * (size_t)(576 * p.G);
}

// A thread per group of 32 channels of a token's head, keys and values.
template <typename V, bool ALIGNED>
__global__ __launch_bounds__(256) void kv4_write_kernel(const Kv4Params p, const V* __restrict__ k,
                                                        const V* __restrict__ v, size_t n_groups) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_groups) return;
  const int g = (int)(i % p.G), head = (int)(i / p.G % p.H);
  const size_t token = i / p.G / p.H;
  const long slot = p.slots[token];
  if (slot < 0 || slot >= p.n_slots) return;
  int t;
  uint8_t* to = sixteen_of(p, slot, head, &t);
  const int G = p.G;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const V* from = which ? v + token * p.v_stride + head * p.v_head : k + token * p.k_stride + head * p.k_head;
    float r[32];
    load_values<32, ALIGNED>(from + 32 * g, r);
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e) m = fmaxf(m, finite_abs(r[e]));
    const _Float16 factor = kv4_factor(m);
    const float q = (float)factor;
    unsigned u[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) u[e] = (unsigned)(r[e] == r[e] ? quant1(r[e], q, -8.0f, 7.0f) : 0) + 8u;
    if (which == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        unsigned w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= u[8 * j + e] << (4 * e);
        *reinterpret_cast<unsigned*>(to + t * 16 * G + j * 4 * G + 4 * g) = w;
      }
      *reinterpret_cast<_Float16*>(to + 512 * G + 2 * (t * G + g)) = factor;
    } else {
#pragma unroll
      for (int c = 0; c < 16; ++c) to[256 * G + (g * 16 + c) * 16 + t] = (uint8_t)(u[c] | u[16 + c] << 4);
      *reinterpret_cast<_Float16*>(to + 544 * G + 2 * (g * 16 + kv4_place(t))) = factor;
    }
  }
}

template <typename V, bool ALIGNED>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4Params p, V* __restrict__ k, V* __restrict__ v,
                                                       size_t n_groups) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_groups) return;
  const int g = (int)(i % p.G), head = (int)(i / p.G % p.H);
  const size_t token = i / p.G / p.H;
  const long slot = p.slots[token];
  const bool in = slot >= 0 && slot < p.n_slots;
  int t;
  const uint8_t* from = sixteen_of(p, in ? slot : 0, head, &t);
  const int G = p.G;
  float r[32];
  const float qk = in ? (float)*reinterpret_cast<const _Float16*>(from + 512 * G + 2 * (t * G + g)) : 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const unsigned w = in ? *reinterpret_cast<const unsigned*>(from + t * 16 * G + j * 4 * G + 4 * g) : 0x88888888u;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[8 * j + e] = (float)((int)(w >> (4 * e) & 15u) - 8) * qk;
  }
  store_values<32, ALIGNED>(k + token * p.k_stride + head * p.k_head + 32 * g, r);
  const float qv = in ? (float)*reinterpret_cast<const _Float16*>(from + 544 * G + 2 * (g * 16 + kv4_place(t))) : 0.0f;
#pragma unroll
  for (int c = 0; c < 16; ++c) {
    const unsigned b = in ? from[256 * G + (g * 16 + c) * 16 + t] : 0x88u;
    r[c] = (float)((int)(b & 15u) - 8) * qv;
    r[16 + c] = (float)((int)(b >> 4) - 8) * qv;
  }
  store_values<32, ALIGNED>(v + token * p.v_stride + head * p.v_head + 32 * g, r);
}

int check_tokens(const void* k, const void* v, int type, size_t T, int H, int D, size_t k_stride, size_t k_head,
                 size_t v_stride, size_t v_head, const int64_t* slots, const void* cache, size_t n_pages, int page) {
  Q8_REQUIRE(type_ok(type) && H >= 1, Q8_EINVAL);
  Q8_REQUIRE(kv4_shape_ok(D, page) && T <= 0x7fffffffu && n_pages <= 0x7fffffffu, Q8_EUNSUPPORTED);
  Q8_REQUIRE(T == 0 || (k && v && slots && cache && n_pages >= 1), Q8_EINVAL);
  Q8_REQUIRE(H == 1 || (k_head >= (size_t)D && v_head >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(T <= 1 || (k_stride >= (size_t)D && v_stride >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(k, type_bytes(type)) && q8_aligned(v, type_bytes(type)) && q8_aligned(slots, 8) &&
                 q8_aligned(cache, 64), Q8_EALIGN);
  return Q8_OK;
}

}  // namespace

extern "C" int q8_page_tables(const int32_t* lengths_dev, const int32_t* added_dev, int n_requests, int page,
                              const int32_t* free_pages_dev, int n_free, int32_t* table_dev, int width,
                              size_t table_stride, int64_t* slots_dev, int32_t* positions_dev, int n_slots,
                              int32_t* starts_dev, int32_t* grown_dev, int32_t* counts_dev, void* stream) {
  Q8_REQUIRE(n_requests >= 0 && n_free >= 0 && width >= 0 && n_slots >= 0, Q8_EINVAL);
  Q8_REQUIRE(kv4_page_ok(page), Q8_EUNSUPPORTED);
  Q8_REQUIRE(starts_dev && counts_dev && table_stride >= (size_t)width, Q8_EINVAL);
  Q8_REQUIRE(n_requests == 0 || (lengths_dev && added_dev && grown_dev && (table_dev || width == 0)), Q8_EINVAL);
  Q8_REQUIRE((n_free == 0 || free_pages_dev) && (n_slots == 0 || (slots_dev && positions_dev)), Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(lengths_dev, 4) && q8_aligned(added_dev, 4) && q8_aligned(free_pages_dev, 4) &&
                 q8_aligned(table_dev, 4) && q8_aligned(slots_dev, 8) && q8_aligned(positions_dev, 4) &&
                 q8_aligned(starts_dev, 4) && q8_aligned(grown_dev, 4) && q8_aligned(counts_dev, 4), Q8_EALIGN);
  const PageParams p{lengths_dev, added_dev, free_pages_dev, table_dev, reinterpret_cast<long*>(slots_dev),
                     positions_dev, starts_dev, grown_dev, counts_dev, n_requests, __builtin_ctz(page), n_free, width,
                     n_slots, table_stride};
  page_rows_kernel<<<1, 1024, 0, (hipStream_t)stream>>>(p);
  if (n_slots) page_slots_kernel<<<(n_slots + 255) / 256, 256, 0, (hipStream_t)stream>>>(p);
  return q8_launch_status();
}

extern "C" size_t q8_kv4_cache_bytes(size_t n_pages, int n_heads, int page, int D) {
  if (n_heads < 1 || !kv4_shape_ok(D, page)) return 0;
  return n_pages * n_heads * (page / 16) * (18 * (size_t)D);
}

extern "C" int q8_kv4_write(const void* k_dev, const void* v_dev, int type, size_t T, int n_heads, int D,
                            size_t k_stride, size_t k_head_stride, size_t v_stride, size_t v_head_stride,
                            const int64_t* slots_dev, void* cache_dev, size_t n_pages, int page, void* stream) {
  const int rc = check_tokens(k_dev, v_dev, type, T, n_heads, D, k_stride, k_head_stride, v_stride, v_head_stride,
                              slots_dev, cache_dev, n_pages, page);
  if (rc != Q8_OK || T == 0) return rc;
  const Kv4Params p{reinterpret_cast<const long*>(slots_dev), static_cast<uint8_t*>(cache_dev), k_stride, k_head_stride,
                    v_stride, v_head_stride, (long)n_pages * page, (int)T, n_heads, D / 32, __builtin_ctz(page)};
  const size_t groups = T * n_heads * (D / 32), blocks = (groups + 255) / 256;
  Q8_REQUIRE(blocks <= 0x7fffffffu, Q8_EUNSUPPORTED);
  return with_type(type, [&](auto one) {
    using V = decltype(one);
    const V *k = static_cast<const V*>(k_dev), *v = static_cast<const V*>(v_dev);
    if (kv4_rows_aligned<V>(k_dev, v_dev, k_stride, k_head_stride, v_stride, v_head_stride))
      kv4_write_kernel<V, true><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(p, k, v, groups);
    else
      kv4_write_kernel<V, false><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(p, k, v, groups);
    return q8_launch_status();
  });
}

extern "C" int q8_kv4_read(const void* cache_dev, size_t n_pages, int page, const int64_t* slots_dev, size_t T,
                           int n_heads, int D, void* k_dev, void* v_dev, int type, size_t k_stride,
                           size_t k_head_stride, size_t v_stride, size_t v_head_stride, void* stream) {
  const int rc = check_tokens(k_dev, v_dev, type, T, n_heads, D, k_stride, k_head_stride, v_stride, v_head_stride,
                              slots_dev, cache_dev, n_pages, page);
  if (rc != Q8_OK || T == 0) return rc;
  const Kv4Params p{reinterpret_cast<const long*>(slots_dev), static_cast<uint8_t*>(const_cast<void*>(cache_dev)),
                    k_stride, k_head_stride, v_stride, v_head_stride, (long)n_pages * page, (int)T, n_heads, D / 32,
                    __builtin_ctz(page)};
  const size_t groups = T * n_heads * (D / 32), blocks = (groups + 255) / 256;
  Q8_REQUIRE(blocks <= 0x7fffffffu, Q8_EUNSUPPORTED);
  return with_type(type, [&](auto one) {
    using V = decltype(one);
    V *k = static_cast<V*>(k_dev), *v = static_cast<V*>(v_dev);
    if (kv4_rows_aligned<V>(k_dev, v_dev, k_stride, k_head_stride, v_stride, v_head_stride))
      kv4_read_kernel<V, true><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(p, k, v, groups);
    else
      kv4_read_kernel<V, false><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(p, k, v, groups);
    return q8_launch_status();
  });
}
