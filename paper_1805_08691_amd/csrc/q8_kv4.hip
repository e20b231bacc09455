// The paged 4-bit cache of keys and values: block tables and slots from request lengths, tokens in, tokens out.
// (Attention over it: q8_kv4_attend.hip.)
//
// A group of 32 channels of one token's head is held by Eq. Q with p = 3 at the factor q = binary16(max|r| * fl(1/7)).
// Sixteen tokens of a head are 18 D bytes (q8_kv4.h): key codes by token, value codes by channel, so that both are
// operands of a matrix instruction as they lie.
#include "q8_kv4.h"
#include "q8_quant.h"
#include <limits.h>
#pragma clang fp contract(off)

namespace {

using namespace q8;

// ---------------------------------------------------------------- block tables -----------
// A request with `len` tokens in the cache gets `add` more: its pages are counted and handed out in request order.
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

// Up to kFew requests, in one launch: every block sums up all of them for itself (up to four requests a thread; blocks
// of 256 threads for up to 256 requests, a shorter way through the sums: 33 requests 6.1 us in 1024 threads, 3.7 so), and a
// thread writes its tokens' slots by bisection of the starts in LDS.  The token that begins a new page writes its place in
// the table; no block needs what another one writes.  Bound by the two trips to memory and the sums' barriers (4000
// requests with 170 000 slots: 7.8 us).
constexpr int kFew = 4096, kFewest = 256;

template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void page_tables_kernel(const PageParams p) {
  constexpr int kPerThread = PER, kMost = THREADS * PER, kWaves = THREADS / 64;
  __shared__ int starts[kMost + 1], from[kMost];           // first new token; where free_pages[from + page number] is its page
  __shared__ int lengths[kMost];
  __shared__ unsigned sums[2][2][kWaves];
  __shared__ int took[kWaves], out[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), each = (p.n + THREADS - 1) / THREADS;
  int len[kPerThread], add[kPerThread];
  long tokens = 0;
#pragma unroll
  for (int e = 0; e < kPerThread; ++e) {
    const int b = tid * each + e;
    const bool in = e < each && b < p.n;
    len[e] = in ? max(p.lengths[b], 0) : 0;
    add[e] = in ? max(p.added[b], 0) : 0;
    tokens += add[e];
  }
  // The sum of the threads before, v < 2^33: its low 20 bits and the others by themselves, which 1024 threads' sums leave
  // in 32 bits each.
  auto before = [&](long v, unsigned (*sums)[kWaves]) {
    const unsigned own[2] = {(unsigned)v & 0xfffffu, (unsigned)(v >> 20)};
    unsigned upto[2], waves[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      upto[h] = scan64(own[h]);
      if (lane == 63) sums[h][wave] = upto[h];
    }
    lds_barrier();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      waves[h] = scan64(lane < kWaves ? sums[h][lane] : 0u);
      waves[h] = wave ? __builtin_amdgcn_readlane(waves[h], wave - 1) : 0u;
    }
    return (long)(waves[0] + upto[0] - own[0]) + ((long)(waves[1] + upto[1] - own[1]) << 20);
  };
  long at = before(tokens, sums[0]), need_all = 0;
  long begin[kPerThread], need[kPerThread];
  bool fits[kPerThread];
#pragma unroll
  for (int e = 0; e < kPerThread; ++e) {
    begin[e] = at;
    at += add[e];
    const int total = pages_of((long)len[e] + add[e], p.shift);
    fits[e] = total <= p.width && at <= p.n_slots;
    need[e] = fits[e] ? total - pages_of(len[e], p.shift) : 0;
    need_all += need[e];
  }
  long upto = before(need_all, sums[1]);
  int taken = 0, refused = 0;
#pragma unroll
  for (int e = 0; e < kPerThread; ++e) {
    const int b = tid * each + e;
    upto += need[e];
    fits[e] = fits[e] && (need[e] == 0 || upto <= p.n_free);
    if (e < each && b < p.n) {
      starts[b] = (int)begin[e];
      lengths[b] = len[e];
      from[b] = fits[e] ? (int)(upto - need[e]) - pages_of(len[e], p.shift) : INT_MIN;
      taken += fits[e] ? (int)need[e] : 0;
      refused += !fits[e];
      if (blockIdx.x == 0) {
        p.starts[b] = (int)begin[e];
        p.grown[b] = len[e] + (fits[e] ? add[e] : 0);
      }
    }
  }
  if (tid == THREADS - 1) starts[p.n] = (int)at;
  if (blockIdx.x == 0) {
    for (int off = 32; off > 0; off >>= 1) taken += __shfl_xor(taken, off, 64), refused += __shfl_xor(refused, off, 64);
    if (lane == 0) took[wave] = taken, out[wave] = refused;
  }
  lds_barrier();
  if (blockIdx.x == 0 && tid == 0) {
    int t = 0, r = 0;
    for (int w = 0; w < kWaves; ++w) t += took[w], r += out[w];
    p.starts[p.n] = starts[p.n];
    p.counts[0] = t, p.counts[1] = starts[p.n], p.counts[2] = r;
  }
  const int i = blockIdx.x * THREADS + tid;
  if (i < p.n_slots) {
    long slot = -1;
    int position = -1;
    if (i < starts[p.n]) {
      int lo = 0, hi = p.n - 1;                            // the last request that starts at i or before
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= i) lo = mid; else hi = mid - 1;
      }
      if (from[lo] != INT_MIN && i < starts[lo + 1]) {
        const int held = lengths[lo];
        position = held + i - starts[lo];
        const int number = position >> p.shift, in = position & ((1 << p.shift) - 1);
        int* const entry = p.table + lo * p.table_stride + number;
        int page;
        if (number >= pages_of(held, p.shift)) {
          page = p.free_pages[from[lo] + number];
          if (in == 0) *entry = page;
        } else {
          page = *entry;
        }
        slot = ((long)page << p.shift) + in;
      }
    }
    p.slots[i] = slot;
    p.positions[i] = position;
  }
}

// More requests: one block walks over them, 1024 at a time, with the running sums of pages and of tokens.  Bound by that one
// block's dependent trips to memory (5000 requests 25 us, 9000 37).
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

// ... and a thread per slot behind it: its request by bisection of the starts.
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
    if (p.grown[lo] > len && i < p.starts[lo + 1]) {
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

// A block takes 16 tokens and four groups of 32 channels (of the H G of a token); four lanes share a group, eight
// channels each, so that a wavefront reads and writes whole rows of the tokens' values.  Key codes are a word a lane as
// they lie in the cache.  Value codes lie by channel: they pass through LDS, where 16 tokens make rows of 16 bytes, and
// leave as words where four tokens' slots are neighbours (bytes elsewhere).  The floor is memory; what bounds it is
// vector instructions, so places are worked out once for a block.  16001 tokens of 8 heads of 128 channels in bf16, 84 MB: in
// 23 us (vector instructions in 95 % of the cycles), out 22 (80 %); 64 tokens 4 each, a launch.
constexpr int kTok = 16, kGroups = 4;

// The block's tokens, in LDS.
struct Places {
  long base[kTok];                 // where the token's sixteen of head 0 lies, -1: nowhere
  int t[kTok];                     // its place there
  // A row's bytes of the tokens, four to a lane: the first of them, whether they are one aligned word of the cache, and
  // how many of them are not first .. but the last tokens.  (In a run of neighbours that begins `off` places into a word,
  // three of the four lanes have whole words, and the first what is left in front of them and behind.)
  int first[4], word[4], tail[4];
};
__device__ __forceinline__ int place_of(const Places& s, int w, int e) {
  return e < 4 - s.tail[w] ? s.first[w] + e : kTok - 4 + e;
}

__device__ __forceinline__ void find_places(const Kv4Params& p, size_t token0, Places* s) {
  const int tid = threadIdx.x;
  if (tid < 64) {
    const size_t i = token0 + tid;
    const long slot = tid < kTok && i < (size_t)p.T ? p.slots[i] : -1;
    const bool in = slot >= 0 && slot < p.n_slots;
    const int place = (int)(slot & ((1 << p.shift) - 1));
    if (tid < kTok) {
      s->base[tid] = in ? ((((slot >> p.shift) * p.H) << (p.shift - 4)) + (place >> 4)) * (576 * p.G) : -1;
      s->t[tid] = place & 15;
    }
    const long first = __shfl(slot, 0, 64), before = __shfl_up(slot, 1, 64);
    const bool next = in && slot == before + 1;                 // one behind the token before
    const unsigned long chain = __ballot(next), held = __ballot(in);
    const bool run = (chain & 0xfffe) == 0xfffe && (held & 1);
    if (tid < 4) {
      const int off = run ? (int)(first & 3) : 0;
      s->first[tid] = 4 * tid - (tid ? off : 0);
      s->tail[tid] = tid == 0 ? off : 0;
      s->word[tid] = run ? tid > 0 || off == 0 : 0;
    }
    // outside a run: tokens 4 w .. + 3 are neighbours, and the first begins a word
    if (!run && tid < kTok && (tid & 3) == 0) s->word[tid >> 2] = in && (slot & 3) == 0 && (chain >> (tid + 1) & 7) == 7;
  }
  __syncthreads();
}

// Group `group` of the four that begin at group g0 of head0.
struct Group {
  int head, g;
  bool in;                         // there is such a group
  __device__ __forceinline__ Group(const Kv4Params& p, int head0, int g0, int group) {
    head = head0, g = g0 + group;
#pragma unroll
    for (int e = 1; e < kGroups; ++e)
      if (g >= p.G) g -= p.G, ++head;
    in = head < p.H;
  }
};

// The codes plus 8 of a lane's eight values, a byte each, and the factor f of its group, whose other 24 the three lanes
// beside it hold: Round(r / f) of each, on the correctly rounded quotient (a 16-bit r is often exactly between two codes:
// max / 7 is a binary16 number for one maximum in seven).  r * inv is off by a few units; a step t + (r - f t) inv, its
// remainder exact, ends within a unit of r / f, and on it where r / f is a number.  A 16-bit r (11 bits at most, as f) is
// either that at a tie or 2^-12 away from one, so a step and any inv near 1 / f will do; for fp32 two steps on the
// rounded 1 / f end on the rounded quotient (Markstein 1990; f is none of that theorem's exceptions).  A value that is not
// finite takes the division.
template <bool WIDE>
__device__ __forceinline__ void quad_codes(const float (&r)[8], _Float16* factor, unsigned (&u)[2]) {
  float m = 0.0f;
  bool none = false;               // one is no number
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    m = fmaxf(m, fmaxf(fabsf(r[e]), fabsf(r[e + 1])));
    none |= __builtin_isunordered(r[e], r[e + 1]);
  }
  const bool finite = !none && m < __builtin_inff();
  if (!finite) {
    m = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(r[e]));
  }
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0xb1, 0xf, 0xf, true)));        // lanes 1 0 3 2
  m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x4e, 0xf, 0xf, true)));        // lanes 2 3 0 1
  *factor = kv4_factor(m);
  const float f = (float)*factor, inv = WIDE ? __fdiv_rn(1.0f, f) : __builtin_amdgcn_rcpf(f), low = -8.0f * f, high = 7.0f * f;
  constexpr float kRound = 12582912.0f + 8.0f;            // 1.5 * 2^23: rounds half to even, the code plus 8 in the low byte
  unsigned z[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = __builtin_amdgcn_fmed3f(r[e], low, high);
    float t = __fmul_rn(x, inv);
    t = __builtin_fmaf(__builtin_fmaf(-f, t, x), inv, t);
    if constexpr (WIDE) t = __builtin_fmaf(__builtin_fmaf(-f, t, x), inv, t);
    z[e] = __float_as_uint(__fadd_rn(t, kRound));
  }
  if (!finite) {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = (unsigned)((r[e] == r[e] ? quant1(r[e], f, -8.0f, 7.0f) : 0) + 8);
  }
  u[0] = __builtin_amdgcn_perm(z[1], z[0], 0x0c0c0400u) | __builtin_amdgcn_perm(z[3], z[2], 0x04000c0cu);
  u[1] = __builtin_amdgcn_perm(z[5], z[4], 0x0c0c0400u) | __builtin_amdgcn_perm(z[7], z[6], 0x04000c0cu);
}

// `per` fours of groups one after the other, so that the tokens' places are worked out once; the next four's values are
// on their way meanwhile.
template <typename V, bool ALIGNED>
__global__ __launch_bounds__(256) void kv4_write_kernel(const Kv4Params p, const V* __restrict__ k,
                                                        const V* __restrict__ v, int group_blocks, int per) {
  __shared__ Places places;
  __shared__ __attribute__((aligned(4))) unsigned char rows[2][kGroups][16][kTok + 4];            // [group][channel pair][token]
  const int blocks = (group_blocks + per - 1) / per, first = (int)(blockIdx.x % blocks) * per, G = p.G;
  const size_t token0 = (size_t)(blockIdx.x / blocks) * kTok;
  const int end = min(first + per, group_blocks);
  int g0 = first * kGroups, head0 = g0 / G;
  g0 -= head0 * G;
  const int tid = threadIdx.x, q = tid & 3, group = tid >> 2 & 3, ti = tid >> 4;
  const size_t token = token0 + ti, in_k = token * p.k_stride, in_v = token * p.v_stride;
  const bool there = token < (size_t)p.T;
  V rk[8], rv[8];
  auto fetch = [&](const Group& a) __attribute__((always_inline)) {       // (of no group: any values, which go nowhere)
    const bool in = a.in && there;
    const V *fk = k + (in ? in_k + a.head * p.k_head + 32 * a.g + 8 * q : 0),
            *fv = v + (in ? in_v + a.head * p.v_head + 32 * a.g + 8 * q : 0);
    if constexpr (ALIGNED) {
      __builtin_memcpy(rk, __builtin_assume_aligned(fk, 16), sizeof(rk));
      __builtin_memcpy(rv, __builtin_assume_aligned(fv, 16), sizeof(rv));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) rk[e] = fk[e], rv[e] = fv[e];
    }
  };
  Group a(p, head0, g0, group);
  fetch(a);                                               // (its way does not depend on the slots)
  find_places(p, token0, &places);
  const size_t head_bytes = (size_t)(576 * G) << (p.shift - 4);
  const long base = places.base[ti];
  const int t = places.t[ti];
  uint8_t* const mine = p.cache + base;
  // rows out: four tokens of a channel pair
  const int out_group = tid >> 6, r = tid >> 2 & 15, w = tid & 3, i0 = places.first[w];
  const bool word = places.word[w] != 0;
  int byte_of[4];
  long byte_at[4];                                        // -1: nowhere
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    byte_of[e] = word ? i0 + e : place_of(places, w, e);
    const long at = places.base[byte_of[e]];
    byte_at[e] = at >= 0 ? at + places.t[byte_of[e]] + 256 * G + r * 16 : -1;
  }

  for (int block = first; block < end; ++block) {
    float nk[8], nv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) nk[e] = (float)rk[e], nv[e] = (float)rv[e];
    const Group now = a, leave(p, head0, g0, out_group);
    g0 += kGroups;
    while (g0 >= G) g0 -= G, ++head0;
    a = Group(p, head0, g0, group);
    if (block + 1 < end) fetch(a);
    unsigned char (*const to)[16][kTok + 4] = rows[block & 1];
    const bool held = now.in && base >= 0;
    uint8_t* const at = mine + now.head * head_bytes;
    _Float16 factor;
    unsigned u[2];
    quad_codes<sizeof(V) == 4>(nk, &factor, u);
    if (held) {
      // half byte e of the word is byte e of u
      const unsigned x = u[0] | u[0] >> 4, y = u[1] | u[1] >> 4;
      *reinterpret_cast<unsigned*>(at + t * 16 * G + q * 4 * G + 4 * now.g) = __builtin_amdgcn_perm(y, x, 0x06040200u);
      if (q == 0) *reinterpret_cast<_Float16*>(at + 512 * G + 2 * (t * G + now.g)) = factor;
    }
    quad_codes<sizeof(V) == 4>(nv, &factor, u);
    // lanes q and q + 2 hold the low and the high halves of the same eight bytes: each makes four of them
    const unsigned give = q < 2 ? u[1] : u[0];                       // what the other one needs
    const unsigned other = (unsigned)__builtin_amdgcn_mov_dpp((int)give, 0x4e, 0xf, 0xf, true);
    const unsigned bytes = q < 2 ? u[0] | other << 4 : other | u[1] << 4;
    const int r0 = 8 * (q & 1) + 4 * (q >> 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) to[group][r0 + e][ti] = (unsigned char)(bytes >> (8 * e));
    if (held && q == 0) *reinterpret_cast<_Float16*>(at + 544 * G + 2 * (now.g * 16 + kv4_place(t))) = factor;
    lds_barrier();
    if (leave.in) {
      const unsigned char* const b = to[out_group][r];
      const size_t beyond = leave.head * head_bytes + leave.g * 256;
      if (word) {
        *reinterpret_cast<unsigned*>(p.cache + byte_at[0] + beyond) =
            (unsigned)b[i0] | (unsigned)b[i0 + 1] << 8 | (unsigned)b[i0 + 2] << 16 | (unsigned)b[i0 + 3] << 24;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (byte_at[e] >= 0) p.cache[byte_at[e] + beyond] = b[byte_of[e]];
      }
    }
  }
}

template <typename V, bool ALIGNED>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4Params p, V* __restrict__ k, V* __restrict__ v,
                                                       int group_blocks, int per) {
  __shared__ Places places;
  __shared__ __attribute__((aligned(16))) unsigned char rows[2][kGroups][kTok][16];               // [group][token][channel pair]
  const int blocks = (group_blocks + per - 1) / per, first = (int)(blockIdx.x % blocks) * per, G = p.G;
  const size_t token0 = (size_t)(blockIdx.x / blocks) * kTok;
  const int end = min(first + per, group_blocks);
  int g0 = first * kGroups, head0 = g0 / G;
  g0 -= head0 * G;
  const size_t head_bytes = (size_t)(576 * G) << (p.shift - 4);
  find_places(p, token0, &places);
  const int tid = threadIdx.x, q = tid & 3, group = tid >> 2 & 3, ti = tid >> 4;
  const size_t token = token0 + ti, out_k = token * p.k_stride, out_v = token * p.v_stride;
  const bool there = token < (size_t)p.T;
  const long base = places.base[ti];
  const int t = places.t[ti];
  const uint8_t* const mine = p.cache + base;
  const int in_group = tid >> 6, r = tid >> 2 & 15, w = tid & 3, i0 = places.first[w];
  const bool word = places.word[w] != 0;
  int byte_of[4];
  long byte_at[4];                                        // -1: nowhere
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    byte_of[e] = word ? i0 + e : place_of(places, w, e);
    const long at = places.base[byte_of[e]];
    byte_at[e] = at >= 0 ? at + places.t[byte_of[e]] + 256 * G + r * 16 : -1;
  }

  // a four's bytes on their way: a row's word (or bytes), a key word and two factors
  unsigned row4 = 0, kc = 0;
  _Float16 kf = 0, vf = 0;
  auto fetch = [&](int head, int g) __attribute__((always_inline)) {
    const Group arrive(p, head, g, in_group), a(p, head, g, group);
    row4 = 0x88888888u, kc = 0x88888888u;
    kf = vf = 0;
    if (arrive.in) {
      const size_t beyond = arrive.head * head_bytes + arrive.g * 256;
      if (word) {
        row4 = *reinterpret_cast<const unsigned*>(p.cache + byte_at[0] + beyond);
      } else {
        row4 = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) row4 |= (byte_at[e] >= 0 ? (unsigned)p.cache[byte_at[e] + beyond] : 0x88u) << (8 * e);
      }
    }
    if (a.in && base >= 0) {
      const uint8_t* const at = mine + a.head * head_bytes;
      kc = *reinterpret_cast<const unsigned*>(at + t * 16 * G + q * 4 * G + 4 * a.g);
      kf = *reinterpret_cast<const _Float16*>(at + 512 * G + 2 * (t * G + a.g));
      vf = *reinterpret_cast<const _Float16*>(at + 544 * G + 2 * (a.g * 16 + kv4_place(t)));
    }
  };
  fetch(head0, g0);
  for (int block = first; block < end; ++block) {
    const unsigned bytes = row4, codes = kc;
    const float fk = (float)kf, fv = (float)vf;
    const Group a(p, head0, g0, group);
    g0 += kGroups;
    while (g0 >= G) g0 -= G, ++head0;
    if (block + 1 < end) fetch(head0, g0);
    unsigned char (*const to)[kTok][16] = rows[block & 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) to[in_group][byte_of[e]][r] = (unsigned char)(bytes >> (8 * e));
    lds_barrier();
    if (there && a.in) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)((int)(codes >> (4 * e) & 15u) - 8) * fk;
      store_values<8, ALIGNED>(k + out_k + a.head * p.k_head + 32 * a.g + 8 * q, x);
      // (the low half bytes of eight channel pairs, or their high ones)
      uint2 vc;
      __builtin_memcpy(&vc, __builtin_assume_aligned(&to[group][ti][8 * (q & 1)], 8), 8);
      const int high = 4 * (q >> 1);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)((int)((e < 4 ? vc.x : vc.y) >> (8 * (e & 3) + high) & 15u) - 8) * fv;
      store_values<8, ALIGNED>(v + out_v + a.head * p.v_head + 32 * a.g + 8 * q, x);
    }
  }
}

// Fours of groups that a block takes one after the other: as many as leave the compute units eight blocks each.
inline int fours_per_block(size_t blocks) { return (int)(blocks / 2048 < 1 ? 1 : blocks / 2048 > 8 ? 8 : blocks / 2048); }

// ... and launches of that: as many tokens as blocks reach.
template <typename F>
int launch_tokens(size_t T, size_t group_blocks, F launch) {
  const size_t all = (T + kTok - 1) / kTok * group_blocks;
  const int per = fours_per_block(all);
  const size_t blocks = (group_blocks + per - 1) / per, most = most_blocks(256) / blocks * kTok;
  Q8_REQUIRE(most > 0, Q8_EUNSUPPORTED);
  for (size_t t = 0; t < T; t += most) {
    const size_t n = T - t < most ? T - t : most;
    launch(t, (int)n, (unsigned)((n + kTok - 1) / kTok * blocks), per);
  }
  return q8_launch_status();
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
  if (n_requests <= kFew) {
    const int threads = n_requests <= kFewest ? 256 : 1024, blocks = n_slots > 0 ? (n_slots - 1) / threads + 1 : 1;
    if (threads == 256)
      page_tables_kernel<256, 1><<<blocks, 256, 0, (hipStream_t)stream>>>(p);
    else
      page_tables_kernel<1024, 4><<<blocks, 1024, 0, (hipStream_t)stream>>>(p);
    return q8_launch_status();
  }
  page_rows_kernel<<<1, 1024, 0, (hipStream_t)stream>>>(p);
  if (n_slots) page_slots_kernel<<<((unsigned)n_slots + 255) / 256, 256, 0, (hipStream_t)stream>>>(p);
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
  const size_t group_blocks = ((size_t)n_heads * (D / 32) + kGroups - 1) / kGroups;
  return with_type(type, [&](auto one) {
    using V = decltype(one);
    const V *const k = static_cast<const V*>(k_dev), *const v = static_cast<const V*>(v_dev);
    const bool aligned = kv4_rows_aligned<V>(k_dev, v_dev, k_stride, k_head_stride, v_stride, v_head_stride);
    return launch_tokens(T, group_blocks, [&](size_t t, int n, unsigned grid, int per) {
      Kv4Params part = p;
      part.slots = p.slots + t, part.T = n;
      if (aligned)
        kv4_write_kernel<V, true><<<grid, 256, 0, (hipStream_t)stream>>>(part, k + t * k_stride, v + t * v_stride, (int)group_blocks, per);
      else
        kv4_write_kernel<V, false><<<grid, 256, 0, (hipStream_t)stream>>>(part, k + t * k_stride, v + t * v_stride, (int)group_blocks, per);
    });
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
  const size_t group_blocks = ((size_t)n_heads * (D / 32) + kGroups - 1) / kGroups;
  return with_type(type, [&](auto one) {
    using V = decltype(one);
    V *const k = static_cast<V*>(k_dev), *const v = static_cast<V*>(v_dev);
    const bool aligned = kv4_rows_aligned<V>(k_dev, v_dev, k_stride, k_head_stride, v_stride, v_head_stride);
    return launch_tokens(T, group_blocks, [&](size_t t, int n, unsigned grid, int per) {
      Kv4Params part = p;
      part.slots = p.slots + t, part.T = n;
      if (aligned)
        kv4_read_kernel<V, true><<<grid, 256, 0, (hipStream_t)stream>>>(part, k + t * k_stride, v + t * v_stride, (int)group_blocks, per);
      else
        kv4_read_kernel<V, false><<<grid, 256, 0, (hipStream_t)stream>>>(part, k + t * k_stride, v + t * v_stride, (int)group_blocks, per);
    });
  });
}
