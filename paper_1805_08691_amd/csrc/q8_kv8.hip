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

// The largest of half a wavefront's magnitudes, as bit patterns (whose order is theirs, and which need no care of what is no
// number).
__device__ __forceinline__ unsigned largest32(unsigned v) {
  auto turn = [&](auto ctrl_c) {
    constexpr int ctrl = decltype(ctrl_c)::value;            // (within 16 lanes, by 8, 4, 2, 1)
    v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, ctrl, 0xf, 0xf, true));
  };
  turn(std::integral_constant<int, 0x128>{});
  turn(std::integral_constant<int, 0x124>{});
  turn(std::integral_constant<int, 0x122>{});
  turn(std::integral_constant<int, 0x121>{});
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max((unsigned)a[0], (unsigned)a[1]);
}
// And of all of them.
__device__ __forceinline__ unsigned largest64(unsigned v) {
  v = largest32(v);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((unsigned)b[0], (unsigned)b[1]);
}

// 1 / q for row_codes, within 2^-23 of itself: a quotient of up to 127.1 is then off by 127.1 (2^-23 + 2^-24) = 2.3e-5, less
// than the 7e-5 from a tie within which it divides.
__device__ __forceinline__ float about_one_over(float q) { return __builtin_amdgcn_rcpf(q); }

struct Factor {
  float q, by;                     // the new one; old over new where what stands there changes, 1 where not
};
__device__ __forceinline__ Factor new_factor(unsigned most, float old, bool begun) {
  const float need = __fmul_rn(__uint_as_float(most), 1.0f / 127.0f);
  if (begun) return {need, 1.0f};
  if (need <= old) return {old, 1.0f};
  const float q = fmaxf(need, __fmul_rn(old, kGrowth));
  return {q, __fdiv_rn(old, q)};
}

// One token of a sixteen, of one head, by a wavefront: keys in its lower half, values in its upper half, 8 channels a lane.
// Nothing else of the sixteen is touched unless its factor begins or grows.  (A step's tokens, 8 heads of 128 channels, us with
// blocks for whole sixteens and so: 256 requests 9.7 and 6.7, 1000 25.7 and 16.8, 2000 48 and 20; its bytes are worth 1 to 4.
// Bound by the trips to memory: slots, then rows and factors, then what is stored by the byte.)
template <typename V, bool ALIGNED>
__device__ __forceinline__ void write_one(const Kv8Params& p, const V* k, const V* v, uint8_t* sixteen, int token, int head, int place) {
  const int lane = threadIdx.x & 63, l = lane & 31, D = p.D, c = 8 * l;
  const bool upper = lane >= 32, in = c < D, begun = place == 0;
  float* const factor = reinterpret_cast<float*>(sixteen + 32 * D) + upper;
  const V* const from = upper ? v + token * p.v_stride + head * p.v_head : k + token * p.k_stride + head * p.k_head;
  V raw[8];
  float old = 0.0f, x[8];
  if (in) {
    __builtin_memcpy(raw, __builtin_assume_aligned(from + c, ALIGNED ? 16 : sizeof(V)), sizeof(raw));
    if (!begun) old = *factor;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = in ? (float)raw[e] : 0.0f;
  const unsigned all = row_bits8(x, 0);
  const bool finite = all < kNotFinite;
  const Factor f = new_factor(largest32(finite ? all : __float_as_uint(row_max8(x, 0.0f))), old, begun);
  const float q = f.q > 0.0f ? f.q : 1.0f;               // (all zero: any factor)
  if (!in) return;
  uint2 z = row_codes(x, q, about_one_over(q), finite);
  z.x ^= 0x80808080u, z.y ^= 0x80808080u;
  if (l == 0) *factor = f.q;
  auto code = [&](int e) { return (e < 4 ? z.x : z.y) >> (8 * (e & 3)) & 255u; };
  if (!upper) {
    *reinterpret_cast<uint2*>(sixteen + kv8_key(D, place, c)) = z;
    if (begun || f.by != 1.0f)
#pragma unroll 1
      for (int t = 0; t < 16; ++t) {
        uint2* const at = reinterpret_cast<uint2*>(sixteen + kv8_key(D, t, c));
        if (t != place) *at = begun ? uint2{0x80808080u, 0x80808080u} : uint2{again4(at->x, f.by), again4(at->y, f.by)};
      }
  } else if (!begun && f.by == 1.0f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sixteen[16 * D + 16 * (c + e) + place] = (unsigned char)code(e);
  } else {
    const unsigned shift = 8 * (place & 3);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint4* const at = reinterpret_cast<uint4*>(sixteen + 16 * D + 16 * (c + e));
      unsigned w[4] = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
      if (!begun) {
        const uint4 was = *at;
        w[0] = again4(was.x, f.by), w[1] = again4(was.y, f.by), w[2] = again4(was.z, f.by), w[3] = again4(was.w, f.by);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i == place >> 2) w[i] = (w[i] & ~(255u << shift)) | code(e) << shift;
      *at = uint4{w[0], w[1], w[2], w[3]};
    }
  }
}

// A block takes, in `per` heads one after the other, the sixteens that its token begins (INDEXED: its 16 tokens), i.e. those of
// whose tokens in the call it is the first.  A thread has 8 channels of a token, twice beyond 128 channels (UNITS); the next
// head's values are on their way meanwhile, and barriers wait for LDS only: value codes change places there, so that both the
// token-major side and the cache's side are whole lines.  (16001 tokens, 8 heads of 128 channels: 29 us; bytes 20.  Bound by vector
// instructions, 76 % of the cycles, 20 a value: five for its code and for being sure of it, the others for its type, the maximum, and
// the way of a value's code through LDS by the byte, where half the cycles are conflicts between banks.)
template <typename V, bool ALIGNED, bool INDEXED, int UNITS>
__global__ __launch_bounds__(256, UNITS == 1 ? 5 : 3) void kv8_write_kernel(const Kv8Params p, const V* __restrict__ k, const V* __restrict__ v, int per) {
  constexpr int CHUNK = INDEXED ? 16 : 1;
  __shared__ int member[CHUNK][16];
  __shared__ int leads[CHUNK];                          // how many they are
  __shared__ long slots[CHUNK];
  __shared__ unsigned most[2][2][4];
  __shared__ __attribute__((aligned(16))) unsigned char rows[2][128 * UNITS][20];    // value codes [channel][token]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int groups = (p.H + per - 1) / per, head0 = (int)(blockIdx.x % groups) * per, head1 = min(head0 + per, p.H);
  const int chunk = p.first + (int)(blockIdx.x / groups), D = p.D;
  const int ti = tid >> 4, l = tid & 15;
  int members;                                          // of the sixteen that token `lane` (the only one) begins, or none
  long slot0 = 0;
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
    const int n = __popc((unsigned)(__ballot(e >= 0) >> (lane & 48)) & 0xffffu);
    if (l == 0) leads[ti] = in && first == t ? n : 0, slots[ti] = slot;
    lds_barrier();
    members = lane < CHUNK ? leads[lane] : 0;
  } else {
    const long slot = p.slots[chunk];
    long s[kScan / 256];
#pragma unroll
    for (int u = 0; u < kScan / 256; ++u) s[u] = u * 256 + tid < p.T ? p.slots[u * 256 + tid] : -1;
    if (!in_cache(p, slot)) return;
    if (tid < 16) member[0][tid] = -1;
    lds_barrier();
#pragma unroll
    for (int u = 0; u < kScan / 256; ++u)
      if (s[u] >> 4 == slot >> 4) atomicMax(&member[0][s[u] & 15], u * 256 + tid);
    lds_barrier();
    const int e = lane < 16 ? member[0][lane] : -1;
    if (__any(e >= 0 && e < chunk) || !__any(e == chunk)) return;
    members = __popcll(__ballot(e >= 0));
    slot0 = slot;
  }
  const size_t head_bytes = (size_t)kv8_sixteen(D) << (p.shift - 4);
  // ---- the only ones of their sixteens, a wavefront each
  for (unsigned ones = INDEXED ? (unsigned)__ballot(members == 1) : members == 1; ones; ones &= ones - 1) {
    const int i = INDEXED ? __builtin_ctz(ones) : 0, t = chunk * CHUNK + i;
    const long slot = INDEXED ? slots[i] : slot0;
    for (int head = head0 + ((wave - i) & 3); head < head1; head += 4)
      write_one<V, ALIGNED>(p, k, v, p.cache + sixteen_of(p, slot, head), t, head, (int)(slot & 15));
  }
  // ---- the others
  for (unsigned more = INDEXED ? (unsigned)__ballot(members > 1) : members > 1; more; more &= more - 1) {
    const int i = INDEXED ? __builtin_ctz(more) : 0;
    uint8_t* at = p.cache + sixteen_of(p, INDEXED ? slots[i] : slot0, head0);
    const int token = member[i][ti];
    const bool begun = member[i][0] >= 0;
    // which of the sixteen are tokens of the call, a byte of ones each
    unsigned given[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) given[e >> 2] |= member[i][e] >= 0 ? 255u << (8 * (e & 3)) : 0u;
    const V *from_k = k + (size_t)max(token, 0) * p.k_stride + head0 * p.k_head + 8 * l,
            *from_v = v + (size_t)max(token, 0) * p.v_stride + head0 * p.v_head + 8 * l;
    V raw[2][UNITS][8];
    float2 old = {0.0f, 0.0f};
    uint4 was = {0, 0, 0, 0};
    auto fetch = [&](const uint8_t* sixteen) __attribute__((always_inline)) {
      if (!begun) {
        old = *reinterpret_cast<const float2*>(sixteen + 32 * D);
        if (tid < D) was = *reinterpret_cast<const uint4*>(sixteen + 16 * D + 16 * tid);
      }
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const V* const from = (s ? from_v : from_k) + 128 * u;
          if (token >= 0 && 8 * l + 128 * u < D)
            __builtin_memcpy(raw[s][u], __builtin_assume_aligned(from, ALIGNED ? 16 : sizeof(V)), sizeof(raw[s][u]));
          else
#pragma unroll
            for (int e = 0; e < 8; ++e) raw[s][u][e] = (V)0.0f;
        }
    };
    fetch(at);
    for (int head = head0; head < head1; ++head) {
      const int turn = head & 1;
      float x[2][UNITS][8];
      unsigned top[2];
      bool finite[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        unsigned all = 0;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[s][u][e] = (float)raw[s][u][e];
          all = row_bits8(x[s][u], all);
        }
        finite[s] = all < kNotFinite;
        top[s] = all;
        if (!finite[s]) {
          float m = 0.0f;
#pragma unroll
          for (int u = 0; u < UNITS; ++u) m = row_max8(x[s][u], m);
          top[s] = __float_as_uint(m);
        }
      }
      const float2 q_old = old;
      const uint4 v_old = was;
      uint8_t* const sixteen = at;
      at += head_bytes, from_k += p.k_head, from_v += p.v_head;
      if (head + 1 < head1) fetch(at);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        top[s] = largest64(top[s]);
        if (lane == 0) most[turn][s][wave] = top[s];
      }
      lds_barrier();
#pragma unroll
      for (int s = 0; s < 2; ++s)
        top[s] = max(max(most[turn][s][0], most[turn][s][1]), max(most[turn][s][2], most[turn][s][3]));
      const Factor fk = new_factor(top[0], q_old.x, begun), fv = new_factor(top[1], q_old.y, begun);
      // (all zero: any factor)
      const float qk = fk.q > 0.0f ? fk.q : 1.0f, qv = fv.q > 0.0f ? fv.q : 1.0f;
      const float inv_k = about_one_over(qk), inv_v = about_one_over(qv);
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const int c = 8 * l + 128 * u;
        if (c >= D) continue;
        uint2* const to = reinterpret_cast<uint2*>(sixteen + kv8_key(D, ti, c));
        if (token >= 0) {
          const uint2 zk = row_codes(x[0][u], qk, inv_k, finite[0]);
          *to = uint2{zk.x ^ 0x80808080u, zk.y ^ 0x80808080u};
          const uint2 zv = row_codes(x[1][u], qv, inv_v, finite[1]);
#pragma unroll
          for (int e = 0; e < 8; ++e) rows[turn][c + e][ti] = (unsigned char)(((e < 4 ? zv.x : zv.y) >> (8 * (e & 3)) & 255u) ^ 128u);
        } else if (begun) {
          *to = uint2{0x80808080u, 0x80808080u};
        } else if (fk.by != 1.0f) {
          const uint2 z = *to;
          *to = uint2{again4(z.x, fk.by), again4(z.y, fk.by)};
        }
      }
      lds_barrier();
      if (tid < D) {
        unsigned z[4] = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
        if (!begun) {
          z[0] = v_old.x, z[1] = v_old.y, z[2] = v_old.z, z[3] = v_old.w;
          if (fv.by != 1.0f) {
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = again4(z[e], fv.by);
          }
        }
        // (bytes of places without a token are not read as such)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          z[e] = (z[e] & ~given[e]) | (*reinterpret_cast<const unsigned*>(&rows[turn][tid][4 * e]) & given[e]);
        *reinterpret_cast<uint4*>(sixteen + 16 * D + 16 * tid) = uint4{z[0], z[1], z[2], z[3]};
      }
      if (tid == 0) *reinterpret_cast<float2*>(sixteen + 32 * D) = float2{fk.q, fv.q};
    }
    lds_barrier();                                        // LDS has been read
  }
}

// A block takes 16 tokens of a head: key codes 8 a thread; value codes through LDS, a channel of a sixteen a thread where the
// tokens are one's, and by the byte where not.  (16001 tokens, 8 heads of 128 channels, bf16: 19 us, 5.2 TB/s; all by the byte 24.5.
// Bound by the memory's rate; values' codes are read from LDS by the byte, more than half of its cycles
// are conflicts.)
template <typename V, bool ALIGNED>
__global__ __launch_bounds__(256) void kv8_read_kernel(const Kv8Params p, V* __restrict__ k, V* __restrict__ v) {
  __shared__ long base[16];
  __shared__ int place[16];
  __shared__ __attribute__((aligned(16))) unsigned char rows[kMaxHead][20];          // value codes [channel][token]
  const int tid = threadIdx.x, head = blockIdx.x % p.H, D = p.D;
  const size_t token0 = (size_t)p.first + (size_t)(blockIdx.x / p.H) * 16;
  if (tid < 16) {
    const long slot = token0 + tid < (size_t)p.T ? p.slots[token0 + tid] : -1;
    base[tid] = in_cache(p, slot) ? (long)sixteen_of(p, slot, head) : -1;
    place[tid] = (int)(slot & 15);
  }
  __syncthreads();
  const int ti = tid >> 4, l = tid & 15;
  const long at = base[ti];
  float2 q = {0.0f, 0.0f};
  uint2 zk[2] = {{0x80808080u, 0x80808080u}, {0x80808080u, 0x80808080u}};
  if (at >= 0) {
    q = *reinterpret_cast<const float2*>(p.cache + at + 32 * D);
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (8 * l + 128 * u < D) zk[u] = *reinterpret_cast<const uint2*>(p.cache + at + kv8_key(D, place[ti], 8 * l + 128 * u));
  }
  {
    const long from = base[l];
    if (__all(from >= 0 && from == base[0] && place[l] == l)) {
      if (tid < D) {
        const uint4 w = *reinterpret_cast<const uint4*>(p.cache + from + 16 * D + 16 * tid);
        unsigned* const to = reinterpret_cast<unsigned*>(rows[tid]);
        to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
      }
    } else {
      for (int c = ti; c < D; c += 16) rows[c][l] = from >= 0 ? p.cache[from + 16 * D + 16 * c + place[l]] : (unsigned char)128;
    }
  }
  __syncthreads();
  const size_t token = token0 + ti;
  if (token >= (size_t)p.T) return;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int c = 8 * l + 128 * u;
    if (c >= D) continue;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)((int)((e < 4 ? zk[u].x : zk[u].y) >> (8 * (e & 3)) & 255u) - 128) * q.x;
    store_values<8, ALIGNED>(k + token * p.k_stride + head * p.k_head + c, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)((int)rows[c + e][ti] - 128) * q.y;
    store_values<8, ALIGNED>(v + token * p.v_stride + head * p.v_head + c, x);
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

// `chunks` blocks a group of heads, in as many launches as they need.
template <typename F>
int launch_chunks(size_t chunks, int groups, F launch) {
  const size_t most = most_blocks(256) / groups;
  for (size_t c = 0; c < chunks; c += most) launch(c, (unsigned)((chunks - c < most ? chunks - c : most) * groups));
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
    // (heads of a block: as many as leave the compute units eight blocks each)
    const size_t chunks = indexed ? (T + 15) / 16 : T, all = chunks * n_heads / 2048;
    const int per = (int)(all < 1 ? 1 : all > 8 ? 8 : all);
    return launch_chunks(chunks, (n_heads + per - 1) / per, [&](size_t chunk, unsigned grid) {
      Kv8Params part = p;
      part.first = (int)chunk;
      auto go = [&](auto aligned_c, auto indexed_c) {
        if (D <= 128)
          kv8_write_kernel<V, decltype(aligned_c)::value, decltype(indexed_c)::value, 1>
              <<<grid, 256, 0, (hipStream_t)stream>>>(part, k, v, per);
        else
          kv8_write_kernel<V, decltype(aligned_c)::value, decltype(indexed_c)::value, 2>
              <<<grid, 256, 0, (hipStream_t)stream>>>(part, k, v, per);
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
