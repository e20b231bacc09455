// Attention over the paged 8-bit cache where a request has many columns (prompts, in pieces or whole; a decoder's rows over an
// encoder's states): the mathematics of q8_kv8_attend.hip, on v_mfma_f32_32x32x16_f16.
//
// A workgroup owns 32 columns of each of its wavefronts, which share a key head, and walks over the keys they see, 64 at a
// time.  The codes go from memory to registers, a share to a wavefront, and become operands of the matrix instruction in
// LDS, in the order in which a wavefront reads them; all wavefronts multiply all of them.
//   S^T[key][column]     = K Q^T   two tiles of 32 keys, 2 G products each
//   O^T[channel][column] = V^T P^T G tiles of 32 channels, four products each
// Lane (r, h) of S has 16 keys of sixteens h and 2 + h for column r, so that a factor is one number of a lane, and probabilities
// are operands as they come.
//
// Measured: 2048 tokens of each of three requests over up to 8192 keys, 32 query heads on 4 of 128 channels, 356 us, 0.83 PFLOP/s
// (in a window of 1024 116); matrix instructions in 39 %, vector instructions in 53 % of the cycles, at 1.85 GHz, of 1.6 wavefronts a
// SIMD where two have room: workgroups of whole tiles, of which there are barely two for each place, end at different times.  The order
// below, exponentials between key products and unpacking between value products, took it from 383 to 354; a reference of each column
// of its own costs 1 % of that.  Eight wavefronts that share keys, products of 16 x 16, and two groups that multiply in turn were no
// faster; 64 columns a wavefront, which halve what is read from LDS, need 493 registers and lose it in moves between their halves (504).
#include "q8_kv8_attend.h"

namespace {

using namespace q8;

typedef float f16v __attribute__((ext_vector_type(16)));

// Products of probabilities and values' factors are made relative to a column's largest so that this is 2^kTop, and again where
// their sum over a lane's keys of a sixteen passes 2^kMost: binary16 numbers, off by 2^-11 of themselves, or by 2^-32 of the
// largest.  Probabilities' sums have a reference of their own, made and left alike.  The factor is part of the exponent (its
// logarithm is added to the score), and taken out of the probabilities' sums again, in fp32, so that what an exponent loses
// beside a large score is the score's error alone.  A factor that is 2^-kFar of what matters to the column or less counts as that: its
// product is as good as 0 in binary16, and its probability is still an fp32 number.  All of it is a column's own: what others of
// the tile see has no effect.
[[maybe_unused]] constexpr float kTop = 7.0f, kMost = 15.0f, kFar = 40.0f;
constexpr int kRing = 128;                      // steps whose sixteens' places and factors are in LDS

template <int G>
struct Wide {
  static constexpr int OPERANDS = 4096 * G;     // of a step's keys, and of its values; two steps of each
  static constexpr int V_AT = 2 * OPERANDS, RING_AT = 4 * OPERANDS, FACTORS_AT = RING_AT + kRing * 4 * 4;
  static constexpr int HOLE_AT = FACTORS_AT + kRing * 4 * 8, LDS = HOLE_AT + 16;
};

// Product n of a key tile: lane half h has eight channels from here on, 16 neighbours in two products (q8_kv8.h).
template <int G>
__device__ __forceinline__ constexpr int channel_of(int n, int h) {
  return n < G / 2 * 4 ? n / 4 * 64 + 16 * (2 * (n >> 1 & 1) + h) + 8 * (n & 1) : 32 * (G - 1) + 8 * (2 * (n & 1) + h);
}

template <int G, typename V>
__global__ __launch_bounds__(256, G <= 4 ? 2 : 1) void kv8_wide_kernel(const AttendParams p, const V* __restrict__ q,
                                                                       V* __restrict__ out) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int D = 32 * G, SIXTEEN = kv8_sixteen(D);
  constexpr int PAIRS = (2 * G + kWaves - 1) / kWaves;      // of operands that a wavefront makes, of keys and of values
  using W = Wide<G>;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 31, h = lane >> 5;
  const Codes codes;
  Part a;
  Tile t;
  // (whole tiles: the last of a request see most keys, so they go before its others; requests are not ordered by their lengths)
  const int id = p.parts ? (int)blockIdx.x : (p.tiles - 1 - (int)blockIdx.x / p.H) * p.H + (int)blockIdx.x % p.H;
  if (!find_part<kWideCols, kWideParts, true>(p, id, shared, &a, &t)) return;
  const int head = a.head, start = t.lo + a.step0 * kStep, steps = a.step1 - a.step0;
  const int last = min(t.lo + t.steps * kStep, t.len);

  // ---- where sixteens lie, as numbers of them in the cache, and their factors.  One that is not there is read as the cache's
  // first, and its keys' factor is -1; the values' factor of one that no row sees, which may be anything, counts as zero.
  const int* __restrict__ table = p.table + t.b * p.table_stride;
  unsigned* const places = reinterpret_cast<unsigned*>(shared + W::RING_AT);
  float2* const factors = reinterpret_cast<float2*>(shared + W::FACTORS_AT);
  int* const hole = reinterpret_cast<int*>(shared + W::HOLE_AT);        // whether one that should be there is not
  auto find_sixteens = [&](int i0, int n) {           // i0: of the part's, four to a step
    for (int i = i0 + tid; i < i0 + n; i += 256) {
      const int at = (start >> 4) + i;
      int page = -1;
      if (at * 16 < last) page = table[at >> p.shift];
      const bool in = page >= 0 && page < p.n_pages;
      const unsigned place = in ? (unsigned)((((long)page * p.H + head) << p.shift) + (at & ((1 << p.shift) - 1))) : 0u;
      float2 f = {-1.0f, 0.0f};
      if (in) f = *reinterpret_cast<const float2*>(p.cache + (size_t)place * SIXTEEN + 32 * D);
      if (at * 16 + 15 < t.seen) f.y = 0.0f;
      places[i & (4 * kRing - 1)] = place;
      factors[i & (4 * kRing - 1)] = f;
      if (!in && at * 16 < last) *hole = 1;
    }
  };
  if (tid == 0) *hole = 0;
  lds_barrier();
  find_sixteens(0, min(4 * (steps + 3), 4 * kRing));
  lds_barrier();
  bool holes = __builtin_amdgcn_readfirstlane(*hole) != 0;
  auto slot_of = [&](int s, int c) { return (4 * s + c) & (4 * kRing - 1); };

  // ---- loads.  Pair u of a step's keys: products 2 m and 2 m + 1 of tile u / G, m = u % G, whose row r is token 4 (r / 8) + r % 4
  // of the tile's sixteen (r / 4) % 2; of the values: channel tile u / 2, keys of sixteens 2 (u % 2) and the next.
  uint4 kc[PAIRS], vc[PAIRS];
  unsigned key_place[PAIRS], value_place[PAIRS];      // of the next loads
  auto find_pair = [&](int s, int i) __attribute__((always_inline)) {           // keys of s + 1, values of s
    const int u = wave + i * kWaves;
    if (2 * G % kWaves != 0 && u >= 2 * G) return;
    key_place[i] = places[slot_of(s + 1, 2 * (u / G) + (r >> 2 & 1))];
    value_place[i] = places[slot_of(s, 2 * (u & 1) + h)];
  };
  auto issue_keys = [&](int i) __attribute__((always_inline)) {
    const int u = wave + i * kWaves, m = u % G;
    if (2 * G % kWaves != 0 && u >= 2 * G) return;
    const uint8_t* const from = p.cache + (size_t)key_place[i] * SIXTEEN + (r >> 3) * 4 * D + (m >> 1) * 256;
    if (m < G / 2 * 2) {
      kc[i] = *reinterpret_cast<const uint4*>(from + ((2 * (m & 1) + h) * 4 + (r & 3)) * 16);
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(from + (h * 4 + (r & 3)) * 8);
      const uint2 y = *reinterpret_cast<const uint2*>(from + ((2 + h) * 4 + (r & 3)) * 8);
      kc[i] = uint4{x.x, x.y, y.x, y.y};
    }
  };
  auto issue_values = [&](int i) __attribute__((always_inline)) {
    const int u = wave + i * kWaves;
    if (2 * G % kWaves != 0 && u >= 2 * G) return;
    vc[i] = *reinterpret_cast<const uint4*>(p.cache + (size_t)value_place[i] * SIXTEEN + 16 * D + (32 * (u >> 1) + r) * 16);
  };
  // Operands of step s: codes.
  auto unpack_key = [&](int s, auto k_c) __attribute__((always_inline)) {        // half k % 2 of pair k / 2
    constexpr int k = decltype(k_c)::value, i = k / 2;
    const int u = wave + i * kWaves;
    if (2 * G % kWaves != 0 && u >= 2 * G) return;
    char* const to = shared + (s & 1) * W::OPERANDS + u * 2048 + k % 2 * 1024 + lane * 16;
    *reinterpret_cast<h8*>(to) = k % 2 ? codes.eight(kc[i].z, kc[i].w) : codes.eight(kc[i].x, kc[i].y);
  };
  float2 next[2];                                     // factors of a step's sixteens h and 2 + h
  float ref = 0.0f;                                   // of a column's products, as a power of two
  float above = 0.0f;                                 // and how far it is above that of its probabilities' sum
  float factor[2], weight[2], offset[2];              // log2 of the values' factors; what they count as; the same less `ref`
  auto find_factors = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 2; ++b) next[b] = factors[slot_of(s, 2 * b + h)];
  };
  auto weigh = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      factor[b] = log2_of(next[b].y);
      weight[b] = fmaxf(factor[b], above - kFar);
      offset[b] = weight[b] - ref;
    }
  };
  auto unpack_value = [&](int s, auto k_c) __attribute__((always_inline)) {
    constexpr int k = decltype(k_c)::value, i = k / 2;
    const int u = wave + i * kWaves;
    if (2 * G % kWaves != 0 && u >= 2 * G) return;
    char* const to = shared + W::V_AT + (s & 1) * W::OPERANDS + u * 2048 + k % 2 * 1024 + lane * 16;
    *reinterpret_cast<h8*>(to) = k % 2 ? codes.eight(vc[i].z, vc[i].w) : codes.eight(vc[i].x, vc[i].y);
  };
  constexpr std::integral_constant<int, PAIRS> kPairs{};
  auto all_of = [&](auto n_c, auto f) __attribute__((always_inline)) {
    auto each = [&](auto self, auto k_c) __attribute__((always_inline)) -> void {
      constexpr int k = decltype(k_c)::value;
      if constexpr (k < decltype(n_c)::value) {
        f(k_c);
        self(self, std::integral_constant<int, k + 1>{});
      }
    };
    each(each, std::integral_constant<int, 0>{});
  };
  all_of(kPairs, [&](auto i_c) { find_pair(-1, decltype(i_c)::value), issue_keys(decltype(i_c)::value); });

  // ---- the column of this lane
  const int col = t.first + wave * 32 + r, in = min(col, t.cols - 1), tok = in / p.ratio;
  const int pos = col < t.cols ? row_position(p, t, tok) : -1;
  h8 qf[2 * G];
  float rest;                                         // scores are products times `rest` and the keys' factor
  {
    const V* qr = q + (size_t)(t.row + tok) * p.q_stride + ((size_t)head * p.ratio + in % p.ratio) * p.q_head;
    float v[2 * G][8], top = 0.0f;
#pragma unroll
    for (int n = 0; n < 2 * G; ++n) {
      load_values<8, false>(qr + channel_of<G>(n, h), v[n]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[n][e]));
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const unsigned e2 = min(max(__float_as_uint(top) >> 23, 1u), 253u);
    const float down = copysignf(__uint_as_float((254u - e2) << 23), p.scale_log2);
    rest = fmaxf(fabsf(p.scale_log2) * __uint_as_float(e2 << 23), 1e-30f);    // (no 0 times infinity)
#pragma unroll
    for (int n = 0; n < 2 * G; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[n][e] = (_Float16)(v[n][e] * down);
  }
  float sum = 0.0f;
  bool begun = col >= t.cols;                         // (a column that there is not: it has no maximum to find)
  f16v o[G];
#pragma unroll
  for (int i = 0; i < G; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
  // steps whose every key is seen by every column of the tile
  const int pos0 = row_position(p, t, t.first / p.ratio), pos1 = row_position(p, t, (min(t.first + kWideCols, t.cols) - 1) / p.ratio);
  const int clear0 = p.window > 0 ? pos1 - p.window : -1, clear1 = pos0;

  // ---- products, register e of s2[b] being token e of sixteen 2 b + h: kProducts of a step's keys, and of its values, one after
  // the other, with what is to be done beside the i-th; operands are read kAhead products before.  (Four before: 128
  // channels spill ten registers, 386 us for the three requests instead of 367.)
  constexpr int kProducts = 4 * G, kAhead = 2;
  using std::integral_constant;
  f16v s2[2], x[2];
  h8 pr[2][2];
  auto products = [&](const char* from, auto multiply, auto beside) __attribute__((always_inline)) {
    h8 operand[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) operand[i] = *reinterpret_cast<const h8*>(from + i * 1024 + lane * 16);
    __builtin_amdgcn_sched_barrier(0);
    auto each = [&](auto self, auto i_c) __attribute__((always_inline)) -> void {
      constexpr int i = decltype(i_c)::value;
      if constexpr (i < kProducts) {
        multiply(i_c, operand[i % kAhead]);
        if constexpr (i + kAhead < kProducts) operand[i % kAhead] = *reinterpret_cast<const h8*>(from + (i + kAhead) * 1024 + lane * 16);
        beside(i_c);
        __builtin_amdgcn_sched_barrier(0);
        self(self, integral_constant<int, i + 1>{});
      }
    };
    each(each, integral_constant<int, 0>{});
  };
  auto nothing = [&](auto) {};
  auto scores = [&](int s, auto beside) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s2[0][e] = s2[1][e] = 0.0f;
    products(shared + (s & 1) * W::OPERANDS, [&](auto i_c, const h8& k8) __attribute__((always_inline)) {
      constexpr int i = decltype(i_c)::value, b = i / (2 * G), n = i % (2 * G);
      s2[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k8, qf[n], s2[b], 0, 0, 0);
    }, beside);
  };
  auto add_values = [&](int s, auto beside) __attribute__((always_inline)) {
    products(shared + W::V_AT + (s & 1) * W::OPERANDS, [&](auto i_c, const h8& v8) __attribute__((always_inline)) {
      constexpr int i = decltype(i_c)::value;
      o[i / 4] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v8, pr[i / 2 % 2][i % 2], o[i / 4], 0, 0, 0);
    }, beside);
  };
  // The share of N things that is done beside product i.
  auto share = [&](auto i_c, auto n_c, auto f) __attribute__((always_inline)) {
    constexpr int i = decltype(i_c)::value, N = decltype(n_c)::value, first = N * i / kProducts, end = N * (i + 1) / kProducts;
    auto each = [&](auto self, auto k_c) __attribute__((always_inline)) -> void {
      constexpr int k = decltype(k_c)::value;
      if constexpr (k < end) {
        f(k_c);
        self(self, integral_constant<int, k + 1>{});
      }
    };
    each(each, integral_constant<int, first>{});
  };
  // Scores 2 k and 2 k + 1 relative to `ref`, as powers of two, with their values' factor; none of keys that the column does not see.
  float by[2];
  auto scale_two = [&](auto k_c) __attribute__((always_inline)) {
    constexpr int k = decltype(k_c)::value, b = k / 8, e = k % 8 * 2;
    x[b][e] = __builtin_fmaf(s2[b][e], by[b], offset[b]);
    x[b][e + 1] = __builtin_fmaf(s2[b][e + 1], by[b], offset[b]);
    float pinned[2] = {x[b][e], x[b][e + 1]};
    asm volatile("" : "+v"(pinned[0]), "+v"(pinned[1]));        // (here, beside the product, not where they are used)
    x[b][e] = pinned[0], x[b][e + 1] = pinned[1];
  };
  auto hide = [&](int s) __attribute__((always_inline)) {
    const int key0 = start + s * kStep;
    if (key0 > clear0 && key0 + kStep - 1 <= clear1 && !holes) return;
    const bool there[2] = {factors[slot_of(s, h)].x >= 0.0f, factors[slot_of(s, 2 + h)].x >= 0.0f};
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int at = pos + 1 - (key0 + 16 * (2 * b + h));
      unsigned see = token_bits(p.window > 0 ? at - p.window : 0, there[b] ? at : 0);
      asm volatile("" : "+v"(see));                   // (a branch, not selects in every step)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[b][e] = see >> e & 1u ? x[b][e] : -__builtin_inff();
    }
  };
  float part[2];                                      // sums of a lane's products of a sixteen
  auto probabilities = [&]() __attribute__((always_inline)) {          // what they are the sums of, without the factors
    return part[0] * __builtin_amdgcn_exp2f(above - weight[0]) + part[1] * __builtin_amdgcn_exp2f(above - weight[1]);
  };
  float raised[2];
  auto raise_two = [&](auto k_c) __attribute__((always_inline)) {
    constexpr int k = decltype(k_c)::value, b = k / 8, e = k % 8 * 2;
    raised[0] = __builtin_amdgcn_exp2f(x[b][e]);
    raised[1] = __builtin_amdgcn_exp2f(x[b][e + 1]);
  };
  auto keep_two = [&](auto k_c) __attribute__((always_inline)) {
    constexpr int k = decltype(k_c)::value, b = k / 8, e = k % 8 * 2;
    unsigned both = __builtin_bit_cast(unsigned, h2{(_Float16)raised[0], (_Float16)raised[1]});
    asm volatile("" : "+v"(both));                    // (here, not behind the branch in which it may be made again)
    const h2 two = __builtin_bit_cast(h2, both);
    part[b] += raised[0];
    part[b] += raised[1];
    pr[b][e >> 3][e & 7] = two[0], pr[b][e >> 3][(e & 7) + 1] = two[1];
  };
  constexpr integral_constant<int, 16> kTwos{};

  // ---- step s multiplies keys of s + 1 beside the exponentials of s, and values of s beside the unpacking of keys s + 2 and
  // values s + 1, whose codes were loaded a step before.  (What is done for steps behind the last goes nowhere.)
  constexpr integral_constant<int, 2 * PAIRS> kHalves{};
  all_of(kHalves, [&](auto k_c) { unpack_key(0, k_c); });
  all_of(kPairs, [&](auto i_c) {
    constexpr int i = decltype(i_c)::value;
    find_pair(0, i), issue_keys(i), issue_values(i);
  });
  lds_barrier();
  scores(0, nothing);
  find_factors(0);
  weigh();
  all_of(kHalves, [&](auto k_c) { unpack_key(1, k_c), unpack_value(0, k_c); });
  by[0] = next[0].x * rest, by[1] = next[1].x * rest;
  all_of(kTwos, scale_two);
  hide(0);
  all_of(kPairs, [&](auto i_c) {
    constexpr int i = decltype(i_c)::value;
    find_pair(1, i), issue_keys(i), issue_values(i);
  });
  lds_barrier();
  for (int s = 0; s < steps; ++s) {
    if ((s & 63) == 0 && s > 0) find_sixteens((s + 64) * 4, 256);
    if ((s & 63) == 1) holes = __builtin_amdgcn_readfirstlane(*hole) != 0;
    part[0] = part[1] = 0.0f;
    scores(s + 1, [&](auto i_c) __attribute__((always_inline)) {
      constexpr int i = decltype(i_c)::value;
      share(i_c, kTwos, [&](auto k_c) __attribute__((always_inline)) {
        constexpr int k = decltype(k_c)::value;
        if constexpr (k > 0) keep_two(integral_constant<int, k - 1>{});
        raise_two(k_c);
      });
      if constexpr (i == 0) find_factors(s + 1);
      if constexpr (i == kProducts / 2) {
        all_of(kPairs, [&](auto i_c) __attribute__((always_inline)) { find_pair(s + 2, decltype(i_c)::value); });
        by[0] = next[0].x * rest, by[1] = next[1].x * rest;
      }
    });
    keep_two(integral_constant<int, 15>{});
    // the first keys that a column sees, and where products or probabilities grow
    float all = probabilities();
    bool again = !begun || fmaxf(all, fmaxf(part[0], part[1])) > 32768.0f;
    if (__any(again)) {
      again |= __shfl_xor((int)again, 32, 64) != 0;
      float most[2] = {x[0][0], x[1][0]};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 1; e < 16; ++e) most[b] = fmaxf(most[b], x[b][e]);
      float top = fmaxf(most[0] + (factor[0] - weight[0]), most[1] + (factor[1] - weight[1]));
      float m = fmaxf(most[0] + (above - weight[0]), most[1] + (above - weight[1]));
      top = fmaxf(top, __shfl_xor(top, 32, 64)), m = fmaxf(m, __shfl_xor(m, 32, 64));
      const bool seen = m > -__builtin_inff();
      // (a sum of 32 that is 2^15 has a term of 2^10)
      again &= seen;
      const float more = again && (!begun || top > kMost - 5.0f) ? top - kTop : 0.0f;
      const float more_sum = again && (!begun || m > kMost - 5.0f) ? m - kTop : 0.0f;
      const float shrink = begun ? __builtin_amdgcn_exp2f(-more) : 1.0f;
      sum *= begun ? __builtin_amdgcn_exp2f(-more_sum) : 1.0f;
      begun |= seen;
      ref += more;
      above += more - more_sum;
#pragma unroll
      for (int i = 0; i < G; ++i) o[i] *= shrink;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float was = weight[b];
        weight[b] = fmaxf(factor[b], above - kFar);
        x[b] += weight[b] - was - more;
      }
      part[0] = part[1] = 0.0f;
      all_of(kTwos, [&](auto k_c) { raise_two(k_c), keep_two(k_c); });
      all = probabilities();
    }
    asm volatile("" : "+v"(above));                   // (what depends on it is not made twice: 128 channels would spill 50 registers)
    sum += all;
    add_values(s, [&](auto i_c) __attribute__((always_inline)) {
      if constexpr (decltype(i_c)::value == 0) weigh();
      share(i_c, integral_constant<int, 4 * PAIRS>{}, [&](auto k_c) __attribute__((always_inline)) {
        constexpr int k = decltype(k_c)::value;
        if constexpr (k < 2 * PAIRS) {
          unpack_key(s + 2, integral_constant<int, k>{});
          if constexpr (k % 2 == 1) issue_keys(k / 2);
        } else {
          unpack_value(s + 1, integral_constant<int, k - 2 * PAIRS>{});
          if constexpr (k % 2 == 1) issue_values((k - 2 * PAIRS) / 2);
        }
      });
      share(i_c, kTwos, scale_two);
    });
    hide(s + 1);
    lds_barrier();
  }
  const float back = __builtin_amdgcn_exp2f(0.5f * above);      // (twice: the power itself may be no normal number)
  f4 all[1][D / 8];
#pragma unroll
  for (int i = 0; i < G; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) all[0][4 * i + (e >> 2)][e & 3] = o[i][e] * back * back;
  const float refs[1] = {ref - above};
  float sums[1] = {sum};
  const bool seen[1] = {begun};
  __syncthreads();
  join_wide<D, kWaves, 32, 1>(p, a, t, shared, out, all, refs, sums, seen);
#endif
}

template <int G, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  constexpr size_t kJoin = (kWideParts + 1) * kWideCols * 4, kLds = Wide<G>::LDS > kJoin ? Wide<G>::LDS : kJoin;
  if constexpr (kLds > 65536) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_wide_kernel<G, V>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    if (attr != hipSuccess) return Q8_EHIP;
  }
  kv8_wide_kernel<G, V><<<(unsigned)(p.tiles * p.H) + (p.parts ? kTarget : 0), 256, kLds, stream>>>(p, q, out);
  return q8_launch_status();
}

template <typename V>
int launch_any(int G, const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  switch (G) {
    case 1: return launch<1>(p, q, out, stream);
    case 2: return launch<2>(p, q, out, stream);
    case 3: return launch<3>(p, q, out, stream);
    case 4: return launch<4>(p, q, out, stream);
    case 5: return launch<5>(p, q, out, stream);
    case 6: return launch<6>(p, q, out, stream);
    case 7: return launch<7>(p, q, out, stream);
    case 8: return launch<8>(p, q, out, stream);
  }
  return Q8_EUNSUPPORTED;
}

}  // namespace

namespace q8 {

int kv8_attend_wide(int G, const AttendParams& p, const void* q, void* out, int type, hipStream_t stream) {
  if (type == Q8_F16)
    return launch_any(G, p, static_cast<const _Float16*>(q), static_cast<_Float16*>(out), stream);
  return launch_any(G, p, static_cast<const __bf16*>(q), static_cast<__bf16*>(out), stream);
}

}  // namespace q8
