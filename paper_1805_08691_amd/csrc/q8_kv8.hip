// The paged 8-bit cache of keys and values: tokens in, tokens out.  (Attention over it: q8_kv8_attend.hip.)
//
// Sixteen tokens of a head are held by Eq. Q with p = 7 at one factor for their keys and one for their values (q8_kv8.h):
//   begun by this call (its first token is among the call's)   q = max|r| * fl(1/127), and places without a token are 0
//   else   q as it was where max|r| * fl(1/127) asks for no more, or the larger of that and 1.25 q;
//          what stood there becomes Round(z fl(q_old / q))
// A factor that grows takes half a step of the new one from every code that stands there: growing by a quarter at least, all
// that a code has lost is below 2.5 steps, however often it grows (by an eighth 4.5; the mean of the errors, over tokens
// whose sizes differ, is the same for any growth up to 1.25, a tenth larger for 1.5, and a third for 2).
#include "q8_kv8.h"
#include "q8_rows.h"
#pragma clang fp contract(off)

namespace {

using namespace q8;

constexpr float kGrowth = 1.25f;

struct Kv8Params {
  const long* __restrict__ slots;
  uint8_t* __restrict__ cache;
  size_t k_stride, k_head, v_stride, v_head;    // elements between tokens and between heads
  long n_slots;                                 // of the cache
  int T, H, D, shift;                           // shift: page = 1 << shift tokens
  int first;                                    // chunk of this launch's first block (read: token)
};

// Where the sixteen of a slot lies.
__device__ __forceinline__ size_t sixteen_of(const Kv8Params& p, long slot, int head) {
  return ((((size_t)(slot >> p.shift) * p.H + head) << (p.shift - 4)) + ((slot & ((1 << p.shift) - 1)) >> 4)) * kv8_sixteen(p.D);
}
__device__ __forceinline__ bool in_cache(const Kv8Params& p, long slot) { return slot >= 0 && slot < p.n_slots; }

// The tokens of one sixteen have to be written together, by whoever has the first of them.  Up to kScan tokens a call, a block
// looks through all slots for them; beyond, a launch before has left every token's number at its place in the cache.
// What stands there is taken for a token's number only if that token has this slot: nothing has to be cleared.
constexpr int kScan = 1024, kMostTokens = 1 << 24;
__device__ __forceinline__ uint8_t* number_at(const Kv8Params& p, long slot) {
  return p.cache + sixteen_of(p, slot, 0) + 32 * p.D + 16 + 3 * (slot & 15);
}

__global__ __launch_bounds__(256) void kv8_number_kernel(const Kv8Params p) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= p.T) return;
  const long slot = p.slots[t];
  if (!in_cache(p, slot)) return;
  uint8_t* const at = number_at(p, slot);
  at[0] = (uint8_t)t, at[1] = (uint8_t)(t >> 8), at[2] = (uint8_t)(t >> 16);
}

// The signed codes in four bytes that hold them plus 128, at factors whose quotient is `by`: Round(z by), plus 128.
__device__ __forceinline__ unsigned again4(unsigned w, float by) {
  unsigned out = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int z = (int)(w >> (8 * e) & 255u) - 128;
    out |= ((unsigned)((int)rintf(__fmul_rn((float)z, by)) + 128) & 255u) << (8 * e);
  }
  return out;
}

struct Factor {
  float q, by;                     // the new one; old over new where what stands there changes, 1 where not
};
__device__ __forceinline__ Factor new_factor(float most, float old, bool begun) {
  const float need = __fmul_rn(most, 1.0f / 127.0f);
  if (begun) return {need, 1.0f};
  if (need <= old) return {old, 1.0f};
  const float q = fmaxf(need, __fmul_rn(old, kGrowth));
  return {q, __fdiv_rn(old, q)};
}

// A block takes the sixteens of one head that its token begins (INDEXED: its 16 tokens), i.e. those of whose tokens in the
// call it is the first.  A thread has 8 channels of a token, twice beyond 128 channels.
template <typename V, bool ALIGNED, bool INDEXED>
__global__ __launch_bounds__(256) void kv8_write_kernel(const Kv8Params p, const V* __restrict__ k, const V* __restrict__ v) {
  constexpr int CHUNK = INDEXED ? 16 : 1;
  __shared__ int member[CHUNK][16];
  __shared__ int leads[CHUNK];
  __shared__ float most[2][4];
  __shared__ __attribute__((aligned(16))) unsigned char rows[kMaxHead][20];          // value codes [channel][token]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x % p.H, chunk = p.first + (int)(blockIdx.x / p.H), D = p.D;
  const int ti = tid >> 4, l = tid & 15;
  if constexpr (INDEXED) {
    const int t = chunk * 16 + ti;
    const long slot = t < p.T ? p.slots[t] : -1;
    const bool in = in_cache(p, slot);
    int e = -1;
    if (in) {
      const uint8_t* const at = number_at(p, (slot & ~15l) + l);
      const int n = at[0] | at[1] << 8 | at[2] << 16;
      if (n < p.T && p.slots[n] == (slot & ~15l) + l) e = n;
    }
    member[ti][l] = e;
    int first = e < 0 ? 0x7fffffff : e;
    for (int off = 8; off > 0; off >>= 1) first = min(first, __shfl_xor(first, off, 16));
    if (l == 0) leads[ti] = in && first == t;
  } else {
    const long slot = p.slots[chunk];
    if (!in_cache(p, slot)) return;
    if (tid < 16) member[0][tid] = -1;
    __syncthreads();
    for (int i = tid; i < p.T; i += 256) {
      const long s = p.slots[i];
      if (s >> 4 == slot >> 4) atomicMax(&member[0][s & 15], i);
    }
    __syncthreads();
    if (tid == 0) {
      int first = 0x7fffffff;
      for (int e = 0; e < 16; ++e) first = member[0][e] < 0 ? first : min(first, member[0][e]);
      leads[0] = first == chunk;
    }
  }
  __syncthreads();
  for (int i = 0; i < CHUNK; ++i) {
    if (!leads[i]) continue;
    const long slot = p.slots[chunk * CHUNK + i];
    uint8_t* const at = p.cache + sixteen_of(p, slot, head);
    const bool begun = member[i][0] >= 0;
    const int token = member[i][ti];
    float x[2][2][8];
    bool finite[2] = {true, true};
    float top[2] = {0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const V* const from = s ? v + (size_t)max(token, 0) * p.v_stride + head * p.v_head
                              : k + (size_t)max(token, 0) * p.k_stride + head * p.k_head;
      unsigned all = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[s][u][e] = 0.0f;
        if (token >= 0 && 8 * l + 128 * u < D) load_values<8, ALIGNED>(from + 8 * l + 128 * u, x[s][u]);
        all = row_bits8(x[s][u], all);
      }
      finite[s] = all < kNotFinite;
      top[s] = finite[s] ? __uint_as_float(all) : row_max8(x[s][1], row_max8(x[s][0], 0.0f));
      for (int off = 32; off > 0; off >>= 1) top[s] = fmaxf(top[s], __shfl_xor(top[s], off, 64));
      if (lane == 0) most[s][wave] = top[s];
    }
    const float2 old = *reinterpret_cast<const float2*>(at + 32 * D);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) top[s] = fmaxf(fmaxf(most[s][0], most[s][1]), fmaxf(most[s][2], most[s][3]));
    const Factor fk = new_factor(top[0], old.x, begun), fv = new_factor(top[1], old.y, begun);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = 8 * l + 128 * u;
      if (c >= D) continue;
      uint2* const to = reinterpret_cast<uint2*>(at + kv8_key(D, ti, c));
      if (token >= 0) {
        // (all zero: any factor)
        const float qk = fk.q > 0.0f ? fk.q : 1.0f, qv = fv.q > 0.0f ? fv.q : 1.0f;
        const uint2 zk = row_codes(x[0][u], qk, __fdiv_rn(1.0f, qk), finite[0]);
        *to = uint2{zk.x ^ 0x80808080u, zk.y ^ 0x80808080u};
        const uint2 zv = row_codes(x[1][u], qv, __fdiv_rn(1.0f, qv), finite[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) rows[c + e][ti] = (unsigned char)(((e < 4 ? zv.x : zv.y) >> (8 * (e & 3)) & 255u) ^ 128u);
      } else if (begun) {
        *to = uint2{0x80808080u, 0x80808080u};
      } else if (fk.by != 1.0f) {
        const uint2 z = *to;
        *to = uint2{again4(z.x, fk.by), again4(z.y, fk.by)};
      }
    }
    __syncthreads();
    if (tid < D) {
      uint4* const to = reinterpret_cast<uint4*>(at + 16 * D + 16 * tid);
      unsigned z[4] = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
      if (!begun) {
        const uint4 was = *to;
        z[0] = was.x, z[1] = was.y, z[2] = was.z, z[3] = was.w;
        if (fv.by != 1.0f) {
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = again4(z[e], fv.by);
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (member[i][e] >= 0) z[e >> 2] = (z[e >> 2] & ~(255u << (8 * (e & 3)))) | (unsigned)rows[tid][e] << (8 * (e & 3));
      *to = uint4{z[0], z[1], z[2], z[3]};
    }
    if (tid == 0) *reinterpret_cast<float2*>(at + 32 * D) = float2{fk.q, fv.q};
    __syncthreads();                                      // LDS has been read
  }
}

// A block takes 16 tokens of a head: key codes 8 a thread; value codes by the byte, 16 tokens of four channels a wavefront (whole
// lines where the tokens are neighbours), through LDS.
template <typename V, bool ALIGNED>
__global__ __launch_bounds__(256) void kv8_read_kernel(const Kv8Params p, V* __restrict__ k, V* __restrict__ v) {
  __shared__ long base[16];
  __shared__ int place[16];
  __shared__ __attribute__((aligned(8))) unsigned char codes[16][kMaxHead + 8];
  const int tid = threadIdx.x, head = blockIdx.x % p.H, D = p.D;
  const size_t token0 = (size_t)p.first + (size_t)(blockIdx.x / p.H) * 16;
  if (tid < 16) {
    const long slot = token0 + tid < (size_t)p.T ? p.slots[token0 + tid] : -1;
    base[tid] = in_cache(p, slot) ? (long)sixteen_of(p, slot, head) : -1;
    place[tid] = (int)(slot & 15);
  }
  __syncthreads();
  {
    const int t = tid & 15;
    const long at = base[t];
    for (int c = tid >> 4; c < D; c += 16) codes[t][c] = at >= 0 ? p.cache[at + 16 * D + 16 * c + place[t]] : (unsigned char)128;
  }
  __syncthreads();
  const int ti = tid >> 4, l = tid & 15;
  const size_t token = token0 + ti;
  if (token >= (size_t)p.T) return;
  const long at = base[ti];
  float2 q = {0.0f, 0.0f};
  if (at >= 0) q = *reinterpret_cast<const float2*>(p.cache + at + 32 * D);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int c = 8 * l + 128 * u;
    if (c >= D) continue;
    uint2 z[2] = {{0x80808080u, 0x80808080u}, {0, 0}};
    if (at >= 0) z[0] = *reinterpret_cast<const uint2*>(p.cache + at + kv8_key(D, place[ti], c));
    z[1] = *reinterpret_cast<const uint2*>(&codes[ti][c]);
    float x[8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)((int)((e < 4 ? z[s].x : z[s].y) >> (8 * (e & 3)) & 255u) - 128) * (s ? q.y : q.x);
      if (s) store_values<8, ALIGNED>(v + token * p.v_stride + head * p.v_head + c, x);
      else store_values<8, ALIGNED>(k + token * p.k_stride + head * p.k_head + c, x);
    }
  }
}

int check_tokens(const void* k, const void* v, int type, size_t T, int H, int D, size_t k_stride, size_t k_head,
                 size_t v_stride, size_t v_head, const int64_t* slots, const void* cache, size_t n_pages, int page) {
  Q8_REQUIRE(type_ok(type) && H >= 1, Q8_EINVAL);
  Q8_REQUIRE(kv4_shape_ok(D, page) && n_pages <= 0x7fffffffu && (size_t)H <= most_blocks(256), Q8_EUNSUPPORTED);
  Q8_REQUIRE(T == 0 || (k && v && slots && cache && n_pages >= 1), Q8_EINVAL);
  Q8_REQUIRE(H == 1 || (k_head >= (size_t)D && v_head >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(T <= 1 || (k_stride >= (size_t)D && v_stride >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(k, type_bytes(type)) && q8_aligned(v, type_bytes(type)) && q8_aligned(slots, 8) &&
                 q8_aligned(cache, 64), Q8_EALIGN);
  return Q8_OK;
}

// `chunks` blocks a head, in as many launches as they need.
template <typename F>
int launch_chunks(size_t chunks, int H, F launch) {
  const size_t most = most_blocks(256) / H;
  for (size_t c = 0; c < chunks; c += most) launch(c, (unsigned)((chunks - c < most ? chunks - c : most) * H));
  return q8_launch_status();
}

}  // namespace

extern "C" size_t q8_kv8_cache_bytes(size_t n_pages, int n_heads, int page, int D) {
  if (n_heads < 1 || !kv4_shape_ok(D, page)) return 0;
  return n_pages * n_heads * (page / 16) * (size_t)kv8_sixteen(D);
}

extern "C" int q8_kv8_write(const void* k_dev, const void* v_dev, int type, size_t T, int n_heads, int D,
                            size_t k_stride, size_t k_head_stride, size_t v_stride, size_t v_head_stride,
                            const int64_t* slots_dev, void* cache_dev, size_t n_pages, int page, void* stream) {
  const int rc = check_tokens(k_dev, v_dev, type, T, n_heads, D, k_stride, k_head_stride, v_stride, v_head_stride,
                              slots_dev, cache_dev, n_pages, page);
  if (rc != Q8_OK || T == 0) return rc;
  Q8_REQUIRE(T < (size_t)kMostTokens, Q8_EUNSUPPORTED);
  const Kv8Params p{reinterpret_cast<const long*>(slots_dev), static_cast<uint8_t*>(cache_dev), k_stride, k_head_stride,
                    v_stride, v_head_stride, (long)n_pages * page, (int)T, n_heads, D, __builtin_ctz(page), 0};
  const bool indexed = T > kScan;
  if (indexed) kv8_number_kernel<<<(unsigned)((T + 255) / 256), 256, 0, (hipStream_t)stream>>>(p);
  return with_type(type, [&](auto one) {
    using V = decltype(one);
    const V *const k = static_cast<const V*>(k_dev), *const v = static_cast<const V*>(v_dev);
    const bool aligned = kv4_rows_aligned<V>(k_dev, v_dev, k_stride, k_head_stride, v_stride, v_head_stride);
    return launch_chunks(indexed ? (T + 15) / 16 : T, n_heads, [&](size_t chunk, unsigned grid) {
      Kv8Params part = p;
      part.first = (int)chunk;
      auto go = [&](auto aligned_c, auto indexed_c) {
        kv8_write_kernel<V, decltype(aligned_c)::value, decltype(indexed_c)::value>
            <<<grid, 256, 0, (hipStream_t)stream>>>(part, k, v);
      };
      using T_ = std::true_type;
      using F_ = std::false_type;
      if (aligned && indexed) go(T_{}, T_{});
      else if (aligned) go(T_{}, F_{});
      else if (indexed) go(F_{}, T_{});
      else go(F_{}, F_{});
    });
  });
}

extern "C" int q8_kv8_read(const void* cache_dev, size_t n_pages, int page, const int64_t* slots_dev, size_t T,
                           int n_heads, int D, void* k_dev, void* v_dev, int type, size_t k_stride,
                           size_t k_head_stride, size_t v_stride, size_t v_head_stride, void* stream) {
  const int rc = check_tokens(k_dev, v_dev, type, T, n_heads, D, k_stride, k_head_stride, v_stride, v_head_stride,
                              slots_dev, cache_dev, n_pages, page);
  if (rc != Q8_OK || T == 0) return rc;
  Q8_REQUIRE(T <= 0x7fffffffu - 16, Q8_EUNSUPPORTED);
  const Kv8Params p{reinterpret_cast<const long*>(slots_dev), static_cast<uint8_t*>(const_cast<void*>(cache_dev)),
                    k_stride, k_head_stride, v_stride, v_head_stride, (long)n_pages * page, (int)T, n_heads, D,
                    __builtin_ctz(page), 0};
  return with_type(type, [&](auto one) {
    using V = decltype(one);
    V *const k = static_cast<V*>(k_dev), *const v = static_cast<V*>(v_dev);
    const bool aligned = kv4_rows_aligned<V>(k_dev, v_dev, k_stride, k_head_stride, v_stride, v_head_stride);
    return launch_chunks((T + 15) / 16, n_heads, [&](size_t chunk, unsigned grid) {
      Kv8Params part = p;
      part.first = (int)(chunk * 16);
      if (aligned)
        kv8_read_kernel<V, true><<<grid, 256, 0, (hipStream_t)stream>>>(part, k, v);
      else
        kv8_read_kernel<V, false><<<grid, 256, 0, (hipStream_t)stream>>>(part, k, v);
    });
  });
}
