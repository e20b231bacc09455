// Attention of new tokens over the paged 4-bit cache (q8_kv4.h):
//   s[j] = scale q . D(k_j),   o = sum_j exp(s[j] - max s) D(v_j) / sum_j exp(s[j] - max s)
// over the keys j <= position (and > position - window) of the token's request; 0 where there are none.  One pass
// over the keys with the running maximum and sum of the softmax in fp32.
//
// A column is a query head of a token; the columns of a request that share a key head are taken 16 at a time, and a
// wavefront multiplies 64 keys by them per step on v_mfma_f32_16x16x32_f16:
//   S^T[key][column]     = K Q^T      four tiles of 16 keys, G products each
//   O^T[channel][column] = V^T P^T    2 G tiles of 16 channels, two products each
// Codes are multiplied as they are: four become binary16 in five instructions (1024 + u is its own bit pattern; u and 16 u
// are taken out of the bytes as they lie), and what they have too much is taken from the keys by a second product, from the
// values before theirs.  A key's factor goes into the fp32 sum of its group, a value's into its token's probability, whose
// product, formed in fp32, is rounded to binary16 (by 2^-11 of it at most).  Outputs are off by, in parts of their norm, where
// scores spread by 1 to 32: fp16 1.8 to 2.7e-4 (their own rounding alone: 2.1e-4), bf16 1.5 to 1.8e-3 (alone: the same).
// Which 16 keys a tile of S takes is chosen so that a lane's 16 probabilities belong to the 16 tokens whose value codes it
// loads: nothing is exchanged between lanes but the maximum.
// The key axis is split over workgroups where columns are few; the last of them to finish adds the parts, in their order.
// Bound by memory while it loops (48 requests of up to 16384 tokens, 64 query heads on 8 of 128 channels: 415 MB in 100 us,
// 70 to 80 of them in the loop at 5 to 5.5 TB/s; 2000 cycles of vector instructions a step beside 1000 of the matrix
// cores) and by dependent trips to memory at both ends (5 us in front of the first keys' products of a split, 4 to 7 behind:
// one request of 131071 tokens, 151 MB, 43 us; 5 short ones 6.7).  One step in LDS a wavefront: with three workgroups a
// compute unit that is 110 KB on their way, and a second would leave room for fewer of them.
#include "q8_kv4_attend.h"
#pragma clang fp contract(fast)

namespace {

using namespace q8;

// A wavefront's step in LDS, 64 keys: the codes of its four sixteens' keys (32 bytes between them: the four rows that one
// LDS access serves then meet different banks), of their values, and their factors.
template <int G>
struct Stage {
  static constexpr int SIXTEEN = 576 * G, CODES = 256 * G, FACTORS = 64 * G;
  static constexpr int K_PITCH = CODES + 32, V_AT = 4 * K_PITCH, F_AT = V_AT + 4 * CODES, SIZE = F_AT + 4 * FACTORS;
  static constexpr int LOADS = 4 * (2 * ((CODES + 1023) / 1024) + 1);                      // of 16 bytes a lane
};

[[maybe_unused]] constexpr float kLift = 10.0f;      // probabilities times 2^10 / (a power of two above the values' factors)

template <int G, typename V>
__global__ __launch_bounds__(256, G <= 4 ? 3 : 1) void kv4_attend_kernel(const AttendParams p, const V* __restrict__ q,
                                                                         V* __restrict__ out) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int D = 32 * G, CT = 2 * G;                 // channels, tiles of 16 of them
  using St = Stage<G>;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, j = lane >> 4;
  Part a;
  Tile t;
  if (!find_part<kCols, kTarget>(p, blockIdx.x, shared, &a, &t)) return;
  const int head = a.head, step0 = a.step0, step1 = a.step1;
  const Unpack un;
  const int last = min(t.lo + t.steps * kStep, t.len);         // keys of the tile end here
  const int iterations = step0 + wave < step1 ? (step1 - step0 - wave + kWaves - 1) / kWaves : 0;

  // ---- the column of this lane
  const int col = t.first + r;
  const bool given = col < t.cols;
  const int tok = min(col, t.cols - 1) / p.ratio, qh = min(col, t.cols - 1) % p.ratio;
  const int pos = given ? row_position(p, t, tok) : -1;  // (no key is at or before -1)
  const int from = p.window > 0 ? pos - p.window : -1;  // keys behind this one
  float v[G][8];
  {
    const V* qr = q + (size_t)(t.row + tok) * p.q_stride + ((size_t)head * p.ratio + qh) * p.q_head + 8 * j;
#pragma unroll
    for (int g = 0; g < G; ++g) load_values<8, false>(qr + 32 * g, v[g]);
  }

  // ---- loads: lane l holds where sixteen l % 4 of iteration l / 4 (of 16) lies, bit l of `held` whether it is there
  const int* __restrict__ table = p.table + t.b * p.table_stride;
  long where = 0;
  unsigned long held = 0;
  auto find_sixteens = [&](int it0) {
    const int s = step0 + wave + (it0 + (lane >> 2)) * kWaves, at = (t.lo >> 4) + s * 4 + (lane & 3);
    int page = -1;
    if (s < step1 && at * 16 < last) page = table[at >> p.shift];
    const bool in = page >= 0 && page < p.n_pages;
    where = in ? (((((long)page * p.H + head) << p.shift) + (at & ((1 << p.shift) - 1))) * St::SIXTEEN) : 0;
    held = __ballot(in);
  };
  char* const stage = shared + wave * St::SIZE;
  auto load = [&](__amdgpu_buffer_rsrc_t from, int at, int bytes, char* to) __attribute__((always_inline)) {
#pragma unroll
    for (int l = 0; l < (bytes + 1023) / 1024; ++l)
      if (l * 1024 + 1024 <= bytes || lane * 16 < bytes - l * 1024)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + l * 1024), 16,
                                                 lane * 16 + at + l * 1024, 0, 0, 0);
  };
  unsigned there = 0;                                          // the iteration's sixteens that there are
  auto issue = [&](int it) __attribute__((always_inline)) {
    if (it > 0 && (it & 15) == 0) find_sixteens(it);
    there = (unsigned)(held >> ((it & 15) * 4)) & 15u;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int l = (it & 15) * 4 + c;
      const unsigned lo = __builtin_amdgcn_readlane((int)where, l), hi = __builtin_amdgcn_readlane((int)(where >> 32), l);
      const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(
          (void*)(p.cache + ((size_t)hi << 32 | lo)), 0, there >> c & 1u ? St::SIXTEEN : 0, 0x00020000);
      load(from, 0, St::CODES, stage + c * St::K_PITCH);
      load(from, 2 * St::CODES, St::FACTORS, stage + St::F_AT + c * St::FACTORS);
      load(from, St::CODES, St::CODES, stage + St::V_AT + c * St::CODES);
    }
  };

  find_sixteens(0);
  if (iterations > 0) issue(0);

  // ---- its queries as the right operand, scaled to [1, 2) by a power of two and turned so that scores grow with the
  // products.  The high half bytes come 16 times as large: their queries are a 16th.
  h8 qf[G];
  float scale;
  {
    float top = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[g][e]));
    top = column_max(top);
    const unsigned e2 = min(max(__float_as_uint(top) >> 23, 1u), 253u);
    const float down = copysignf(__uint_as_float((254u - e2) << 23), p.scale_log2);
    scale = fmaxf(fabsf(p.scale_log2) * __uint_as_float(e2 << 23), 1e-30f);    // (no 0 times infinity)
    constexpr int kKeyOrder[8] = {0, 4, 2, 6, 1, 5, 3, 7};
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[g][e] = (_Float16)(v[g][kKeyOrder[e]] * (e < 4 ? down : down * 0.0625f));
  }
  // steps whose every key is seen by every column: behind `clear0`, up to `clear1`
  const int pos0 = row_position(p, t, t.first / p.ratio), pos1 = row_position(p, t, (min(t.first + kCols, t.cols) - 1) / p.ratio);
  const int clear0 = p.window > 0 ? pos1 - p.window : -1, clear1 = pos0;

  f4 o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f4{0, 0, 0, 0};
  float top = -__builtin_inff(), ref = -__builtin_inff(), sum = 0.0f;     // ref: what sum and o are relative to, as a power of 2
  float lift = kLift, limit = 0.0f;                     // kLift - log2 of the factors' power, and where it has to grow
  constexpr _Float16 kLow = -1032.0f16, kHigh = -1152.0f16;
  const h8 key_off = {kLow, kLow, kLow, kLow, kHigh, kHigh, kHigh, kHigh};

  for (int it = 0; it < iterations; ++it) {
    const int key0 = t.lo + (step0 + wave + it * kWaves) * kStep;
    const bool more = it + 1 < iterations;
    wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    const bool clear = key0 > clear0 && key0 + kStep - 1 <= clear1 && there == 15u;
    const char* const factors = stage + St::F_AT + j * St::FACTORS;

    // ---- S^T, keys 16 j + 4 tile + i in register i of tile `tile`
    float x[4][4];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
      unsigned kc[G];
      _Float16 kf[4][G];
      __builtin_memcpy(kc, __builtin_assume_aligned(stage + (r >> 2) * St::K_PITCH + (4 * tile + (r & 3)) * 16 * G + j * 4 * G, 4), 4 * G);
      __builtin_memcpy(kf, __builtin_assume_aligned(factors + tile * 8 * G, 8), 8 * G);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[tile][i] = 0.0f;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const unsigned w8 = kc[g] >> 8;
        f4 s = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_off, qf[g], f4{0, 0, 0, 0}, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(un.low(kc[g]), un.low(w8), un.high(kc[g]), un.high(w8)), qf[g], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[tile][i] = __builtin_fmaf(s[i], (float)kf[i][g], x[tile][i]);
      }
    }
    if (!clear) {
      const int base = key0 + 16 * j;
      unsigned see = token_bits(from + 1 - base, (there >> j & 1u) ? pos + 1 - base : 0);
      asm volatile("" : "+v"(see));                     // (a branch, not selects in every step)
#pragma unroll
      for (int tile = 0; tile < 4; ++tile)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[tile][i] = see >> (4 * tile + i) & 1u ? x[tile][i] : -__builtin_inff();
    }
    // ---- the values' factors.  What lies outside the keys that the rows see may be no number: it counts as zero.
    // (Read twice, for their largest and for use: they would not fit the registers of three wavefronts a SIMD.)
    const bool edge = key0 < t.seen || key0 + kStep > last;
    unsigned keep[8] = {};                              // of the factors as they lie, two each
    if (edge) {
      unsigned in = token_bits(t.seen - (key0 + 16 * j), last - (key0 + 16 * j));
      asm volatile("" : "+v"(in));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t0 = 4 * (e >> 1) + (e & 1);
        keep[e] = (in >> t0 & 1u) * 0xffffu | (in >> (t0 + 2) & 1u) * 0xffff0000u;
      }
    }
    auto value_factors = [&](int g, h2 (&vf)[8]) __attribute__((always_inline)) {
      __builtin_memcpy(vf, __builtin_assume_aligned(factors + 32 * G + g * 32, 16), 32);
      if (edge) {
#pragma unroll
        for (int e = 0; e < 8; ++e) vf[e] = __builtin_bit_cast(h2, __builtin_bit_cast(unsigned, vf[e]) & keep[e]);
      }
    };
    s2 most = {0, 0};                                   // (none is negative: their patterns order as numbers)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      h2 vf[8];
      value_factors(g, vf);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(s2, vf[e]));
    }
    asm volatile("" ::: "memory");
    const h2 both = __builtin_bit_cast(h2, most);
    const float big = fmaxf((float)both[0], (float)both[1]);
    if (__any(big > limit)) {                           // (the first step, and where factors grow beyond 32 times)
      const float all = column_max(big);
      const int e = (int)(__float_as_uint(all) >> 23) - 126;                  // all < 2^e
      lift = kLift - (float)e;
      limit = __uint_as_float((unsigned)(min(e + 5, 126) + 127) << 23);
    }
    // ---- running maximum and sum
    float m = x[0][0];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = fmaxf(m, x[tile][i]);
    top = fmaxf(top, column_max(m));
    const float now = top == -__builtin_inff() ? 0.0f : __builtin_fmaf(top, scale, -lift);
    const float shrink = __builtin_amdgcn_exp2f(ref - now);
    ref = top == -__builtin_inff() ? top : now;
    sum *= shrink;
    if (__any(shrink != 1.0f)) {
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c] *= shrink;
    }
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[tile][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[tile][i], scale, -now));
        sum += x[tile][i];
      }
    // ---- O^T: a probability times its token's factor is the right operand.  What the codes have too much is taken from them
    // here, not by a product as for the keys: the matrix instruction cuts what it adds at the largest, always downwards, and
    // products of 1032 would leave 7e-6 of a value in every output, more than a fp16 output's rounding over long contexts.
#pragma unroll
    for (int g = 0; g < G; ++g) {
      h2 vf[8];
      value_factors(g, vf);
      unsigned vc[4];
      __builtin_memcpy(vc, __builtin_assume_aligned(stage + St::V_AT + j * St::CODES + (g * 16 + r) * 16, 16), 16);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        h8 pr;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tile = 2 * h + (e >> 1), i = e & 1;
          // (in fp32, rounded once: a probability alone is up to 2^lift, beyond binary16 where the factors are small.  Rounded
          // first and multiplied in binary16, bf16 took 41.6 us for one request of 131071 tokens instead of 42.9)
          pr[2 * e] = (_Float16)__builtin_fmaf(x[tile][i], (float)vf[2 * tile + i][0], 0.0f);
          pr[2 * e + 1] = (_Float16)__builtin_fmaf(x[tile][i + 2], (float)vf[2 * tile + i][1], 0.0f);
        }
        const unsigned c = vc[2 * h], d = vc[2 * h + 1];
        auto low = [&](unsigned w) { return un.low(w) + h2{kLow, kLow}; };
        auto high = [&](unsigned w) { return un.high(w) + h2{kHigh, kHigh}; };
        o[2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(low(c), low(c >> 8), low(d), low(d >> 8)), pr, o[2 * g], 0, 0, 0);
        o[2 * g + 1] =
            __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(high(c), high(c >> 8), high(d), high(d >> 8)), pr, o[2 * g + 1], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);                 // the stage has been read
    asm volatile("" ::: "memory");
    if (more) issue(it + 1);
  }
#pragma unroll
  for (int g = 0; g < G; ++g) o[2 * g + 1] *= 0.0625f;
  join_columns<D>(p, a, t, shared, out, o, ref, sum);
#endif
}

template <int G, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  const size_t stages = (size_t)kWaves * Stage<G>::SIZE, joining = join_bytes(32 * G, p.parts != nullptr);
  const size_t lds = stages > joining ? stages : joining;
  if (lds > 65536) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_attend_kernel<G, V>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (attr != hipSuccess) return Q8_EHIP;
  }
  const unsigned blocks = (unsigned)(p.tiles * p.H) + (p.parts ? kTarget : 0);
  kv4_attend_kernel<G, V><<<blocks, 256, lds, stream>>>(p, q, out);
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

// Whether tiles of 128 columns, which unpack a key once for all of them, are taken for new tokens in runs of several: where
// requests have that many columns and the tiles are a workgroup for every compute unit, or can be cut, and parts of them
// are long enough for what adding them costs.  (3 pieces of 2048 tokens over 8192 keys, 32 query heads on 4 of 128 channels:
// 752 us in tiles of 16 columns, 395 so; 512 tokens of one request, 32 on 8, over 4096, 8192, 32768 keys: 91, 163, 591
// and, cut, 68, 108, 321; but 128 tokens over 8192 keys 60 and 71, and with 256 channels, 2 times 256 tokens over 16384
// keys, 179 and 226.)
bool wide_for(size_t T, int B, int H, int ratio, int D, size_t longest, bool cuts) {
  const size_t tiles = tiles_of(T, B, ratio, true, kWideCols) * H;
  if (T * ratio < (size_t)B * (kWideCols / 2)) return false;
  return tiles >= 256 || (cuts && tiles >= 32 && tiles * (longest / kStep) / kTarget >= (D <= 128 ? 32u : 64u));
}

}  // namespace

extern "C" size_t q8_kv4_attend_workspace_bytes(size_t T, int n_requests, int n_heads, int ratio, int D,
                                                size_t longest) {
  return attend_workspace_bytes(T, n_requests, n_heads, ratio, D, longest, wide_for);
}

extern "C" int q8_kv4_attend(const void* q_dev, int type, size_t T, int n_heads, int ratio, int D, size_t q_stride,
                             size_t q_head_stride, const void* cache_dev, size_t n_pages, int page,
                             const int32_t* table_dev, int width, size_t table_stride, const int32_t* lengths_dev,
                             const int32_t* starts_dev, int n_requests, float scale, int window, void* out_dev,
                             size_t o_stride, size_t o_head_stride, void* workspace, size_t workspace_bytes,
                             void* stream) {
  AttendParams p{};
  bool wide = false;
  const int rc = attend_params(q_dev, type, T, n_heads, ratio, D, q_stride, q_head_stride, cache_dev, n_pages, page, table_dev,
                               width, table_stride, lengths_dev, starts_dev, n_requests, scale, window, out_dev, o_stride,
                               o_head_stride, workspace, workspace_bytes, wide_for, &p, &wide);
  if (rc != Q8_OK || p.T == 0) return rc;
  if (wide) return kv4_attend_wide(D / 32, p, q_dev, out_dev, type, (hipStream_t)stream);
  if (type == Q8_F16)
    return launch_any(D / 32, p, static_cast<const _Float16*>(q_dev), static_cast<_Float16*>(out_dev),
                      (hipStream_t)stream);
  return launch_any(D / 32, p, static_cast<const __bf16*>(q_dev), static_cast<__bf16*>(out_dev), (hipStream_t)stream);
}
