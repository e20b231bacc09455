// Attention of new tokens over the paged 8-bit cache (q8_kv8.h):
//   s[j] = scale q . D(k_j),   o = sum_j exp(s[j] - max s) D(v_j) / sum_j exp(s[j] - max s)
// over the keys j <= position (and > position - window) of the token's request, or over all of them; 0 where there are none.
// One pass over the keys with the running maximum and sum of the softmax in fp32.
//
// A column is a query head of a token; the columns of a request that share a key head are taken 16 at a time, and a
// wavefront multiplies 64 keys (four sixteens) by them per step on v_mfma_f32_16x16x32_f16:
//   S^T[key][column]     = K Q^T      four tiles of 16 keys, G products each
//   O^T[channel][column] = V^T P^T    2 G tiles of 16 channels, two products each
// Codes are multiplied as they are: whole numbers up to 128 are binary16 numbers.  Lane (r, j) of S has 16 keys of sixteen j
// and loads the values of the same 16: a score meets its sixteen's factor as one fp32 number of the lane.  A probability times the
// values' factor is rounded to binary16 once, relative to the largest such product that the column itself has met (kLift below):
// whatever other columns of the tile see has no effect.
// The key axis is split over workgroups where columns are few; the last of them to finish adds the parts, in their order.
//
// Measured: 48 rows of 64 query heads on 8 of 128 channels over up to 16384 keys 151 us, 4.85 TB/s, which bounds it (without LDS
// and with the next step's codes on their way, two wavefronts a SIMD are enough), in a window of 1024 23.3; one row over 131071
// keys 58 us, of which six are the split and the adding, in a window of 4096 11.9; 9 x 448 rows of 16 heads of 64 channels over up
// to 1500 keys 28.4 us, bound by vector instructions (three quarters of the cycles), unpacking for 16 columns above all.  Tiles of two
// times 16 columns a wavefront need more registers and were slower nearly everywhere (20 rows of 128 requests over 400 keys 23.4
// and 27.0 us).
#include "q8_kv8_attend.h"
#pragma clang fp contract(fast)

namespace {

using namespace q8;

// Steps of the shortest part that keys are cut into where tiles and heads are many: adding parts takes as long as eight
// steps of a wavefront.  (us with no such limit, 16, 24 and 32 steps, 32 query heads on 8 of 128 channels, one row a request: 64 of
// up to 2048 keys 35.6, 35.6, 33.6, 31.4; 16 of 4096 24.7, 22.0, 22.4, 20.7; 32 of 1000 15.7, 12.0, 12.0, 11.8.)
[[maybe_unused]] constexpr int kLeast = 32;
// Products of probabilities and values' factors are made relative to a column's largest so far so that this is 2^kLift, and again
// where one is 2^kSlack times that: binary16 numbers, off by 2^-11 of themselves, or by 2^-35 of the largest.  The factor is part
// of the exponent (its logarithm is added to the score), and taken out of the probabilities' sum again, in fp32, so that what an
// exponent loses beside a large score is the score's error alone.  A factor that is 2^-kFar of what matters to the column or
// less counts as that in its sums: its product is 0 in binary16, and its probability is still an fp32 number.
[[maybe_unused]] constexpr float kLift = 10.0f, kSlack = 5.0f, kFar = 60.0f;
[[maybe_unused]] constexpr float kNothing = -300.0f;          // the logarithm of no product so far

template <int G, int WAVES, typename V>
__global__ __launch_bounds__(64 * WAVES, G <= 4 ? 2 : 1) void kv8_attend_kernel(const AttendParams p, const V* __restrict__ q,
                                                                         V* __restrict__ out) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int D = 32 * G, CT = 2 * G, CHUNKS = (G + 1) / 2, SIXTEEN = kv8_sixteen(D);
  extern __shared__ __attribute__((aligned(16))) char shared[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, j = lane >> 4;
  Part a;
  Tile t;
  if (!find_part<kCols, kTarget, false, kLeast>(p, blockIdx.x, shared, &a, &t)) return;
  const int head = a.head, step0 = a.step0, step1 = a.step1;
  const Codes codes;
  const int last = min(t.lo + t.steps * kStep, t.len);         // keys of the tile end here
  const int iterations = step0 + wave < step1 ? (step1 - step0 - wave + WAVES - 1) / WAVES : 0;

  // ---- the column of this lane
  const int col = t.first + r;
  const bool given = col < t.cols;
  const int tok = min(col, t.cols - 1) / p.ratio, qh = min(col, t.cols - 1) % p.ratio;
  const int pos = given ? row_position(p, t, tok) : -1;        // (no key is at or before -1)
  const int from = p.window > 0 ? pos - p.window : -1;         // keys behind this one
  float v[G][8];
  {
    const V* qr = q + (size_t)(t.row + tok) * p.q_stride + ((size_t)head * p.ratio + qh) * p.q_head;
#pragma unroll
    for (int g = 0; g < G; ++g) load_values<8, false>(qr + key_channel<G>(g, j), v[g]);
  }

  // ---- loads: lane l holds where sixteen l % 4 of iteration l / 4 (of 16) lies, bit l of `held` whether it is there.  One that
  // is not is read as the cache's first, and its factors count as zeros.
  const int* __restrict__ table = p.table + t.b * p.table_stride;
  long where = 0;
  unsigned long held = 0;
  auto find_sixteens = [&](int it0) {
    const int s = step0 + wave + (it0 + (lane >> 2)) * WAVES, at = (t.lo >> 4) + s * 4 + (lane & 3);
    int page = -1;
    if (s < step1 && at * 16 < last) page = table[at >> p.shift];
    const bool in = page >= 0 && page < p.n_pages;
    where = in ? (((((long)page * p.H + head) << p.shift) + (at & ((1 << p.shift) - 1))) * SIXTEEN) : 0;
    held = __ballot(in);
  };
  uint4 kc[4][CHUNKS], vc[CT];
  float2 factors = {0.0f, 0.0f};
  const uint8_t* values = p.cache;                             // of this lane's sixteen, in the next iteration
  unsigned there = 0, next_there = 0;                          // the iteration's sixteens that there are
  auto issue_keys = [&](int it) __attribute__((always_inline)) {
    if (it > 0 && (it & 15) == 0) find_sixteens(it);
    next_there = (unsigned)(held >> ((it & 15) * 4)) & 15u;
    const uint8_t* const keys = p.cache + __shfl(where, (it & 15) * 4 + (r >> 2), 64);
    values = p.cache + __shfl(where, (it & 15) * 4 + j, 64);
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const uint8_t* const at = keys + tile * 4 * D + c * 256;
        if (c < G / 2) kc[tile][c] = *reinterpret_cast<const uint4*>(at + (j * 4 + (r & 3)) * 16);
        else __builtin_memcpy(&kc[tile][c], __builtin_assume_aligned(at + (j * 4 + (r & 3)) * 8, 8), 8);
      }
    factors = *reinterpret_cast<const float2*>(values + 32 * D);
  };
  auto issue_values = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CT; ++c) vc[c] = *reinterpret_cast<const uint4*>(values + 16 * D + (16 * c + r) * 16);
  };
  find_sixteens(0);
  if (iterations > 0) {
    issue_keys(0);
    issue_values();
  }

  // ---- its queries as the right operand, scaled to [1, 2) by a power of two and turned so that scores grow with the products: binary16,
  // so that the matrix instruction takes them.  fp16 and bf16 values down to 2^-14 and 2^-17 of their row's largest are exact,
  // others off by 2^-25 of it at most.
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
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[g][e] = (_Float16)(v[g][e] * down);
  }
  // steps whose every key is seen by every column: behind `clear0`, up to `clear1`
  const int pos0 = row_position(p, t, t.first / p.ratio), pos1 = row_position(p, t, (min(t.first + kCols, t.cols) - 1) / p.ratio);
  const int clear0 = p.window > 0 ? pos1 - p.window : -1, clear1 = pos0;

  f4 o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f4{0, 0, 0, 0};
  float ref = -__builtin_inff(), sum = 0.0f;            // what sum and o are relative to, as a power of 2
  float products = kNothing;                            // o is relative to 2^(ref + products - kLift)

  for (int it = 0; it < iterations; ++it) {
    const int key0 = t.lo + (step0 + wave + it * WAVES) * kStep;
    const bool more = it + 1 < iterations;
    there = next_there;
    const bool clear = key0 > clear0 && key0 + kStep - 1 <= clear1 && there == 15u;
    const int base = key0 + 16 * j;

    // ---- S^T, keys 16 j + 4 tile + i in register i of tile `tile`
    float x[4][4];
    const float fk = factors.x * scale;
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
      f4 s = {0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint4& w = kc[tile][g / 2];
        const h8 k8 = g & 1 ? codes.eight(w.z, w.w) : codes.eight(w.x, w.y);
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, qf[g], s, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[tile][i] = s[i] * fk;
    }
    float fv = factors.y;
    if (!clear) {
      unsigned see = token_bits(from + 1 - base, (there >> j & 1u) ? pos + 1 - base : 0);
      asm volatile("" : "+v"(see));                     // (a branch, not selects in every step)
#pragma unroll
      for (int tile = 0; tile < 4; ++tile)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[tile][i] = see >> (4 * tile + i) & 1u ? x[tile][i] : -__builtin_inff();
      // (a sixteen that no row sees: its factor may be anything)
      if (!(there >> j & 1u) || base + 15 < t.seen || base >= last) fv = 0.0f;
    }
    // ---- running maximum and sum
    float m = x[0][0];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = fmaxf(m, x[tile][i]);
    const float top = fmaxf(ref, column_max(m));
    const float now = top == -__builtin_inff() ? 0.0f : top;
    const float kept = ref == -__builtin_inff() ? 0.0f : ref - now;
    const float factor = log2_of(fv), before = products + kept, own = m - now + factor;
    products = fmaxf(before, kNothing);
    if (__any(own > before + kSlack || before < kNothing)) {
      const float most = column_max(own);
      if (most > before + kSlack) products = most;
      const float shrink = __builtin_amdgcn_exp2f(before - products);
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c] *= shrink;
    }
    // ---- O^T: a probability times its sixteen's factor is the right operand
    const float raise = fmaxf(factor - products, -kFar) + kLift;
    float beside = now - raise;
    if (m - beside > kLift + kSlack + 0.5f) beside = m;    // (rounded beside a large score: no infinity)
    float all = 0.0f;
    h8 pr[2];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(x[tile][i] - beside);
        all += e;
        pr[tile >> 1][(tile & 1) * 4 + i] = (_Float16)e;
      }
    sum = sum * __builtin_amdgcn_exp2f(kept) + all * __builtin_amdgcn_exp2f(-raise);
    ref = top;
    if (more) issue_keys(it + 1);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes.eight(vc[c].x, vc[c].y), pr[0], o[c], 0, 0, 0);
      o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes.eight(vc[c].z, vc[c].w), pr[1], o[c], 0, 0, 0);
    }
    if (more) issue_values();
  }
  const float back = __builtin_amdgcn_exp2f(0.5f * (products - kLift));      // (twice: the power itself may be no normal number)
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = o[c] * back * back;
  join_columns<D, WAVES>(p, a, t, shared, out, o, ref, sum);
#endif
}

template <int G, int WAVES, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  const size_t lds = join_bytes(32 * G, p.parts != nullptr, WAVES);
  if (lds > 65536) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv8_attend_kernel<G, WAVES, V>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)join_bytes(32 * G, WAVES == kWaves, WAVES));
    if (attr != hipSuccess) return Q8_EHIP;
  }
  const unsigned blocks = (unsigned)(p.tiles * p.H) + (p.parts ? kTarget : 0);
  kv8_attend_kernel<G, WAVES, V><<<blocks, 64 * WAVES, lds, stream>>>(p, q, out);
  return q8_launch_status();
}
template <int G, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  // Whole tiles, fewer than compute units, of many steps: eight wavefronts share them.  (us with four and eight, 16 requests of up to
  // 1500 keys, 12 heads of 64 channels 9.9 and 9.2, 8 of 128 12.8 and 12.2; but 256 tiles and heads of up to 1000 keys 11.1 and
  // 11.8, 60 of up to 300 6.0 and 6.5.)
  if constexpr (G <= 4)
    if (!p.parts && p.tiles * p.H <= 224 && ((long)p.width << p.shift) > 64) return launch<G, 8>(p, q, out, stream);
  return launch<G, kWaves>(p, q, out, stream);
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

// Whether tiles of 128 columns, whose keys and values are unpacked once for all of them, are taken for new tokens in runs of
// several: where requests fill most of a tile, and the tiles are workgroups enough, or can be cut and the parts are long enough
// for what adding them costs.  us in tiles of 16 and of 128 columns, 32 query heads on 8: of 64 channels 16 x 300 tokens 35
// and 26, 32 pieces of up to 100 tokens over up to 2000 63 and 70, 512 over 8192 91 and 72; of 128 channels 512 tokens 17
// and 21, 2 x 1000 47 and 41, 64 pieces of up to 30 81 and 85, 128 over 8192 48 and 69, 512 over 8192 148 and 105; of 256
// channels 512 tokens 40 and 34, 2048 293 and 162, 64 pieces of up to 30 225 and 173, 128 over 8192 117 and 146.
bool wide_for(size_t T, int B, int H, int ratio, int D, size_t longest, bool cuts) {
  const size_t tiles = tiles_of(T, B, ratio, true, kWideCols) * H;
  if (T * ratio < (size_t)B * (D <= 128 ? 96 : 64)) return false;
  if (tiles >= (D <= 64 ? 768 : D <= 128 ? 256 : 96)) return true;
  return cuts && tiles >= 32 && tiles * (longest / kStep) / kTarget >= (D <= 128 ? 32u : 16u);
}

}  // namespace

extern "C" size_t q8_kv8_attend_workspace_bytes(size_t T, int n_requests, int n_heads, int ratio, int D,
                                                size_t longest) {
  return attend_workspace_bytes(T, n_requests, n_heads, ratio, D, longest, wide_for);
}

extern "C" int q8_kv8_attend_call_form(size_t T, int n_requests, int n_heads, int ratio, int D, size_t longest, int ragged,
                                       size_t workspace_bytes) {
  if (n_requests < 1 || n_heads < 1 || ratio < 1 || T < 1 || T > 0x7fffffffu || D < 32 || D > kMaxHead || D % 32 != 0) return 0;
  const Form form = form_of(T, n_requests, n_heads, ratio, D, longest, ragged != 0, workspace_bytes, wide_for, kLeast);
  return (form.wide ? kWideCols : kCols) + form.split;
}

extern "C" int q8_kv8_attend(const void* q_dev, int type, size_t T, int n_heads, int ratio, int D, size_t q_stride,
                             size_t q_head_stride, const void* cache_dev, size_t n_pages, int page,
                             const int32_t* table_dev, int width, size_t table_stride, const int32_t* lengths_dev,
                             const int32_t* starts_dev, int n_requests, float scale, int window, int causal, void* out_dev,
                             size_t o_stride, size_t o_head_stride, void* workspace, size_t workspace_bytes,
                             void* stream) {
  Q8_REQUIRE((causal == 0 || causal == 1) && (causal || window == 0), Q8_EINVAL);
  AttendParams p{};
  bool wide = false;
  const int rc = attend_params(q_dev, type, T, n_heads, ratio, D, q_stride, q_head_stride, cache_dev, n_pages, page, table_dev,
                               width, table_stride, lengths_dev, starts_dev, n_requests, scale, window, out_dev, o_stride,
                               o_head_stride, workspace, workspace_bytes, wide_for, &p, &wide, kLeast);
  if (rc != Q8_OK || p.T == 0) return rc;
  p.all = !causal;
  if (wide) return kv8_attend_wide(D / 32, p, q_dev, out_dev, type, (hipStream_t)stream);
  if (type == Q8_F16)
    return launch_any(D / 32, p, static_cast<const _Float16*>(q_dev), static_cast<_Float16*>(out_dev),
                      (hipStream_t)stream);
  return launch_any(D / 32, p, static_cast<const __bf16*>(q_dev), static_cast<__bf16*>(out_dev), (hipStream_t)stream);
}
