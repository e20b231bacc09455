// Attention of new tokens over the paged 4-bit cache (q8_kv4.h):
//   s[j] = scale q . D(k_j),   o = sum_j exp(s[j] - max s) D(v_j) / sum_j exp(s[j] - max s)
// over the keys j <= position (and > position - window) of the token's request; 0 where there are none.  One pass
// over the keys with the running maximum and sum of the softmax in fp32.
//
// A column is a query head of a token; the columns of a request that share a key head are taken 16 at a time, and a
// wavefront multiplies 64 keys by them per step on v_mfma_f32_16x16x32_f16:
//   S^T[key][column]     = K Q^T      four tiles of 16 keys, G products each
//   O^T[channel][column] = V^T P^T    2 G tiles of 16 channels, two products each
// Four codes become binary16 in five instructions (1024 + u is its own bit pattern; u and 16 u are taken out of the
// bytes as they lie), times their factor exact to half a unit of binary16.  Which 16 keys a tile of S takes is chosen
// so that a lane's 16 probabilities belong to the 16 tokens whose value codes it loads: nothing is exchanged
// between lanes but the maximum.
// The key axis is split over workgroups where columns are few; kv4_join_kernel adds the parts.
#include "q8_kv4.h"
#pragma clang fp contract(fast)

namespace {

using namespace q8;

typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kCols = 16;              // columns of a tile
constexpr int kStep = 64;              // keys of a wavefront's step
constexpr int kWaves = 4;

struct AttendParams {
  const uint8_t* __restrict__ cache;
  const int* __restrict__ table;
  const int* __restrict__ lengths;
  const int* __restrict__ starts;      // null: request b is row b
  float* __restrict__ parts;           // workspace of the split, null: one part
  size_t q_stride, q_head, o_stride, o_head, table_stride;
  long n_pages;
  int T, B, H, ratio, width, shift;    // shift: page = 16 << shift tokens
  int tiles, splits, window;
  float scale_log2;                    // scale * log2(e)
};

// What a workgroup works on: the 16 columns of tile `tile` of request b, whose row 0 is q row `row`.
struct Tile {
  int b, row, first, cols, len, n;     // first column, columns of the request, keys, new tokens
  int seen, lo, steps;                 // first key that a row sees, that key's step's first one, and steps of kStep keys
};

__device__ __forceinline__ bool find_tile(const AttendParams& p, int w, Tile* t) {
  int b = 0, base = 0;
  if (!p.starts) {
    const int per = (p.ratio + kCols - 1) / kCols;
    b = w / per;
    base = b * per;
    t->row = b;
    t->n = 1;
  } else {
    // request b's tiles begin at floor(starts[b] ratio / 16) + b: none overlap, and those behind its last are empty
    auto start = [&](int i) { return min(max(p.starts[i], 0), p.T); };
    auto first = [&](int i) { return (int)((long)start(i) * p.ratio / kCols) + i; };
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first(mid) <= w) lo = mid; else hi = mid - 1;
    }
    b = lo;
    base = first(b);
    t->row = start(b);
    t->n = start(b + 1) - t->row;
  }
  if (b >= p.B) return false;
  t->b = b;
  t->first = (w - base) * kCols;
  t->cols = t->n * p.ratio;
  if (t->first < 0 || t->first >= t->cols) return false;
  const long longest = (long)p.width << (p.shift + 4);
  t->len = (int)min((long)max(p.lengths[b], 0), longest);
  const int tok0 = t->first / p.ratio, tok1 = (min(t->first + kCols, t->cols) - 1) / p.ratio;
  const int pos0 = t->len - t->n + tok0, pos1 = t->len - t->n + tok1;
  t->seen = p.window > 0 ? max(0, pos0 - p.window + 1) : 0;
  t->lo = t->seen & ~(kStep - 1);
  t->steps = pos1 < t->lo ? 0 : (pos1 - t->lo) / kStep + 1;
  return true;
}

// Steps of a part, and how many parts hold any (at least one: it writes the zeros of empty rows).
__device__ __forceinline__ int steps_per_part(const Tile& t, int splits) {
  return max((t.steps + splits - 1) / splits, kWaves);
}

// Four half bytes of each half of w, in the order 0 4 2 6 (from = the low half bytes) or 1 5 3 7, as binary16 codes.
__device__ __forceinline__ h2 codes_low(unsigned w) {
  const unsigned b = (w & 0x000f000fu) | 0x64006400u;              // 1024 + u
  return __builtin_bit_cast(h2, b) - h2{1032.0f16, 1032.0f16};
}
__device__ __forceinline__ h2 codes_high(unsigned w) {
  const unsigned b = (w & 0x00f000f0u) | 0x64006400u;              // 1024 + 16 u
  return __builtin_elementwise_fma(__builtin_bit_cast(h2, b), h2{0.0625f16, 0.0625f16}, h2{-72.0f16, -72.0f16});
}

__device__ __forceinline__ h8 join4(h2 a, h2 b, h2 c, h2 d) {
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int G, typename V>
__global__ __launch_bounds__(256) void kv4_attend_kernel(const AttendParams p, const V* __restrict__ q,
                                                         V* __restrict__ out) {
  constexpr int D = 32 * G, CT = 2 * G;                 // channels, tiles of 16 of them
  extern __shared__ float shared[];                     // [4 waves][16 columns][D], then maxima and sums
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, j = lane >> 4;
  const int head = blockIdx.x % p.H, w = blockIdx.x / p.H % p.tiles, split = blockIdx.x / p.H / p.tiles;
  Tile t;
  if (!find_tile(p, w, &t)) return;
  const int per = steps_per_part(t, p.splits);
  const int step0 = split * per, step1 = min(step0 + per, t.steps);
  if (split > 0 && step0 >= t.steps) return;

  // ---- the column of this lane: its queries as the right operand, scaled to [1, 2) by a power of two
  const int col = t.first + r;
  const bool given = col < t.cols;
  const int tok = min(col, t.cols - 1) / p.ratio, qh = min(col, t.cols - 1) % p.ratio;
  const int pos = given ? t.len - t.n + tok : -1;       // (no key is at or before -1)
  const int from = p.window > 0 ? pos - p.window : -1;  // keys behind this one
  const size_t q_head = (size_t)head * p.ratio + qh;
  h8 qf[G];
  float col_scale;
  {
    const V* qr = q + (size_t)(t.row + tok) * p.q_stride + q_head * p.q_head + 8 * j;
    float v[G][8], top = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      load_values<8, false>(qr + 32 * g, v[g]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[g][e]));
    }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const unsigned e2 = min(max(__float_as_uint(top) >> 23, 1u), 253u);
    const float down = __uint_as_float((254u - e2) << 23);
    col_scale = p.scale_log2 * __uint_as_float(e2 << 23);
    constexpr int kOrder[8] = {0, 4, 2, 6, 1, 5, 3, 7};
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[g][e] = (_Float16)(v[g][kOrder[e]] * down);
  }

  f4 o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f4{0, 0, 0, 0};
  float top = -__builtin_inff(), sum = 0.0f;

  const int* __restrict__ table = p.table + t.b * p.table_stride;
  const int last = min(t.lo + t.steps * kStep, t.len);         // keys of the tile end here
  for (int s = step0 + wave; s < step1; s += kWaves) {
    const int key0 = t.lo + s * kStep;
    // ---- the sixteens: lane (r, j) loads keys of sixteen r / 4 and values of sixteen j
    const int mine = (key0 >> 4) + (r >> 2);
    int page = -1;
    if (mine * 16 < last) page = table[mine >> p.shift];
    const bool held = page >= 0 && page < p.n_pages;
    const size_t at = (((size_t)(held ? page : 0) * p.H + head) << p.shift) + (mine & ((1 << p.shift) - 1));
    const uint8_t* kb = p.cache + at * (576 * G);
    const int other = j * 4;                                   // a lane whose sixteen is j
    const bool v_held = __shfl((int)held, other, 64) != 0;
    const size_t v_at = (size_t)__shfl((long)at, other, 64);
    const uint8_t* vb = p.cache + v_at * (576 * G);

    // ---- S^T, keys 16 j + 4 tile + i in register i of tile `tile`
    float x[4][4];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
      const int tk = 4 * tile + (r & 3);
      unsigned kc[G];
      _Float16 kf[G];
      __builtin_memcpy(kc, __builtin_assume_aligned(kb + tk * 16 * G + j * 4 * G, 4), 4 * G);
      __builtin_memcpy(kf, __builtin_assume_aligned(kb + 512 * G + tk * 2 * G, 2), 2 * G);
      f4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const h2 f = {kf[g], kf[g]};
        const unsigned w8 = kc[g] >> 8;
        const h8 a = join4(codes_low(kc[g]) * f, codes_low(w8) * f, codes_high(kc[g]) * f, codes_high(w8) * f);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, qf[g], acc, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 16 * j + 4 * tile + i;
        const bool seen = v_held && key <= pos && key > from;
        x[tile][i] = seen ? acc[i] * col_scale : -__builtin_inff();
      }
    }
    // ---- running maximum and sum
    float m = top;
#pragma unroll
    for (int tile = 0; tile < 4; ++tile)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = fmaxf(m, x[tile][i]);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const float base = m == -__builtin_inff() ? 0.0f : m;
    const float shrink = __builtin_amdgcn_exp2f(top - base);
    top = m;
    sum *= shrink;
    h2 pr[4][2];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[tile][i] = __builtin_amdgcn_exp2f(x[tile][i] - base);
        sum += x[tile][i];
      }
      pr[tile][0] = h2{(_Float16)x[tile][0], (_Float16)x[tile][2]};
      pr[tile][1] = h2{(_Float16)x[tile][1], (_Float16)x[tile][3]};
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) o[c] *= shrink;
    // ---- O^T.  What lies outside the keys that the rows see, or in a page that the request has not, may be no
    // number: its factors count as zeros.
    const h8 p0 = join4(pr[0][0], pr[0][1], pr[1][0], pr[1][1]), p1 = join4(pr[2][0], pr[2][1], pr[3][0], pr[3][1]);
    const int before = t.seen - (key0 + 16 * j), behind = v_held ? last - (key0 + 16 * j) : 0;   // of 16 tokens
    const bool edge = key0 < t.seen || key0 + kStep > last || !__all(v_held);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      unsigned vc[4];
      h2 vf[8];
      __builtin_memcpy(vc, __builtin_assume_aligned(vb + 256 * G + (g * 16 + r) * 16, 16), 16);
      __builtin_memcpy(vf, __builtin_assume_aligned(vb + 544 * G + g * 32, 16), 32);
      if (edge) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t0 = 4 * (e >> 1) + (e & 1), t2 = t0 + 2;  // tokens t0 and t0 + 2
          vf[e] = h2{t0 >= before && t0 < behind ? vf[e][0] : 0.0f16, t2 >= before && t2 < behind ? vf[e][1] : 0.0f16};
        }
      }
      h2 low[8], high[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        low[2 * e] = codes_low(vc[e]) * vf[2 * e];
        low[2 * e + 1] = codes_low(vc[e] >> 8) * vf[2 * e + 1];
        high[2 * e] = codes_high(vc[e]) * vf[2 * e];
        high[2 * e + 1] = codes_high(vc[e] >> 8) * vf[2 * e + 1];
      }
      o[2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(low[0], low[1], low[2], low[3]), p0, o[2 * g], 0, 0, 0);
      o[2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(low[4], low[5], low[6], low[7]), p1, o[2 * g], 0, 0, 0);
      o[2 * g + 1] =
          __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(high[0], high[1], high[2], high[3]), p0, o[2 * g + 1], 0, 0, 0);
      o[2 * g + 1] =
          __builtin_amdgcn_mfma_f32_16x16x32_f16(join4(high[4], high[5], high[6], high[7]), p1, o[2 * g + 1], 0, 0, 0);
    }
  }
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);

  // ---- the four wavefronts' columns together
  float* const tops = shared + kWaves * kCols * D;
  float* const sums = tops + kWaves * kCols;
  if (j == 0) {
    tops[wave * kCols + r] = top;
    sums[wave * kCols + r] = sum;
  }
  __syncthreads();
  float all = -__builtin_inff();
#pragma unroll
  for (int v = 0; v < kWaves; ++v) all = fmaxf(all, tops[v * kCols + r]);
  const float mine = top == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top - all);
  float* const to = shared + (wave * kCols + r) * D + 4 * j;
#pragma unroll
  for (int c = 0; c < CT; ++c) *reinterpret_cast<f4*>(to + 16 * c) = o[c] * mine;
  __syncthreads();
  const bool whole = p.splits == 1 || per >= t.steps;
  for (int i = tid; i < kCols * D / 4; i += 256) {
    const int c = i / (D / 4), d = i % (D / 4) * 4;
    f4 v = {0, 0, 0, 0};
    float m = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int u = 0; u < kWaves; ++u) m = fmaxf(m, tops[u * kCols + c]);
#pragma unroll
    for (int u = 0; u < kWaves; ++u) {
      v += *reinterpret_cast<const f4*>(shared + (u * kCols + c) * D + d);
      const float tu = tops[u * kCols + c];
      l += tu == -__builtin_inff() ? 0.0f : sums[u * kCols + c] * __builtin_amdgcn_exp2f(tu - m);
    }
    if (whole) {
      const int oc = t.first + c;
      if (oc < t.cols) {
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        const float y[4] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
        store_values<4, false>(out + (size_t)(t.row + oc / p.ratio) * p.o_stride +
                                   ((size_t)head * p.ratio + oc % p.ratio) * p.o_head + d, y);
      }
    } else {
      float* part = p.parts + (((size_t)w * p.H + head) * p.splits + split) * (kCols * (D + 2));
      *reinterpret_cast<f4*>(part + c * D + d) = v;
      if (d == 0) {
        part[kCols * D + c] = m;
        part[kCols * D + kCols + c] = l;
      }
    }
  }
}

// The parts of a tile and head, one after the other in their order.
template <typename V>
__global__ __launch_bounds__(256) void kv4_join_kernel(const AttendParams p, int D, V* __restrict__ out) {
  const int head = blockIdx.x % p.H, w = blockIdx.x / p.H;
  Tile t;
  if (!find_tile(p, w, &t)) return;
  const int per = steps_per_part(t, p.splits);
  if (per >= t.steps) return;                            // (one part: it has written the output)
  const int n = (t.steps + per - 1) / per;
  const float* part = p.parts + ((size_t)w * p.H + head) * p.splits * (kCols * (D + 2));
  const size_t stride = kCols * (D + 2);
  for (int i = threadIdx.x; i < kCols * D; i += 256) {
    const int c = i / D, d = i % D, oc = t.first + c;
    if (oc >= t.cols) return;
    float m = -__builtin_inff(), l = 0.0f, v = 0.0f;
    for (int s = 0; s < n; ++s) m = fmaxf(m, part[s * stride + kCols * D + c]);
    for (int s = 0; s < n; ++s) {
      const float ms = part[s * stride + kCols * D + c];
      const float f = ms == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(ms - m);
      l += f * part[s * stride + kCols * D + kCols + c];
      v += f * part[s * stride + c * D + d];
    }
    out[(size_t)(t.row + oc / p.ratio) * p.o_stride + ((size_t)head * p.ratio + oc % p.ratio) * p.o_head + d] =
        (V)(l > 0.0f ? v / l : 0.0f);
  }
}

template <int G, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  const size_t lds = (size_t)kWaves * kCols * (32 * G + 2) * 4;
  if (lds > 65536) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_attend_kernel<G, V>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (attr != hipSuccess) return Q8_EHIP;
  }
  kv4_attend_kernel<G, V><<<(unsigned)(p.tiles * p.H * p.splits), 256, lds, stream>>>(p, q, out);
  if (p.splits > 1) kv4_join_kernel<V><<<(unsigned)(p.tiles * p.H), 256, 0, stream>>>(p, 32 * G, out);
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

// Tiles of 16 columns that T rows of B requests can have (find_tile), and the parts that they are split into for
// keys of at most `longest`: four workgroups for a compute unit, a part of 512 keys at least.
size_t tiles_of(size_t T, int B, int ratio, bool starts) {
  return starts ? T * ratio / kCols + B : (size_t)B * ((ratio + kCols - 1) / kCols);
}
size_t splits_of(size_t tiles, int H, size_t longest) {
  const size_t want = 1024 / (tiles * H ? tiles * H : 1), most = longest / 512;
  const size_t s = want < most ? want : most;
  return s < 1 ? 1 : s;
}
size_t part_bytes(size_t tiles, int H, int D) { return tiles * H * kCols * (D + 2) * 4; }

}  // namespace

extern "C" size_t q8_kv4_attend_workspace_bytes(size_t T, int n_requests, int n_heads, int ratio, int D,
                                                size_t longest) {
  if (n_requests < 1 || n_heads < 1 || ratio < 1 || D < 32 || D > kMaxHead || T > 0x7fffffffu) return 0;
  // (whether the rows' starts are given is not known here: the more tiles, the fewer splits)
  const size_t a = tiles_of(T, n_requests, ratio, false), b = tiles_of(T, n_requests, ratio, true);
  const size_t sa = splits_of(a, n_heads, longest), sb = splits_of(b, n_heads, longest);
  const size_t na = sa > 1 ? sa * part_bytes(a, n_heads, D) : 0, nb = sb > 1 ? sb * part_bytes(b, n_heads, D) : 0;
  return na > nb ? na : nb;
}

extern "C" int q8_kv4_attend(const void* q_dev, int type, size_t T, int n_heads, int ratio, int D, size_t q_stride,
                             size_t q_head_stride, const void* cache_dev, size_t n_pages, int page,
                             const int32_t* table_dev, int width, size_t table_stride, const int32_t* lengths_dev,
                             const int32_t* starts_dev, int n_requests, float scale, int window, void* out_dev,
                             size_t o_stride, size_t o_head_stride, void* workspace, size_t workspace_bytes,
                             void* stream) {
  Q8_REQUIRE(type_ok(type) && n_heads >= 1 && ratio >= 1 && width >= 0 && window >= 0 && n_requests >= 0, Q8_EINVAL);
  Q8_REQUIRE(scale == scale && scale - scale == 0.0f, Q8_EINVAL);
  Q8_REQUIRE(type != Q8_F32 && kv4_shape_ok(D, page), Q8_EUNSUPPORTED);
  if (T == 0 || n_requests == 0) return Q8_OK;
  Q8_REQUIRE(q_dev && out_dev && cache_dev && n_pages >= 1 && lengths_dev && (table_dev || width == 0), Q8_EINVAL);
  Q8_REQUIRE(table_stride >= (size_t)width && (starts_dev || T == (size_t)n_requests), Q8_EINVAL);
  Q8_REQUIRE(T == 1 || (q_stride >= (size_t)D && o_stride >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(n_heads * ratio == 1 || (q_head_stride >= (size_t)D && o_head_stride >= (size_t)D), Q8_EINVAL);
  Q8_REQUIRE(T <= 0x7fffffffu && n_pages <= 0x7fffffffu && (size_t)width * page <= 0x7fffffc0u, Q8_EUNSUPPORTED);
  Q8_REQUIRE(q8_aligned(q_dev, 2) && q8_aligned(out_dev, 2) && q8_aligned(cache_dev, 64) && q8_aligned(table_dev, 4) &&
                 q8_aligned(lengths_dev, 4) && q8_aligned(starts_dev, 4) && q8_aligned(workspace, 16), Q8_EALIGN);
  const size_t tiles = tiles_of(T, n_requests, ratio, starts_dev != nullptr);
  size_t splits = splits_of(tiles, n_heads, (size_t)width * page);
  const size_t part = part_bytes(tiles, n_heads, D);
  if (!workspace || workspace_bytes / part < 2) splits = 1;
  else if (workspace_bytes / part < splits) splits = workspace_bytes / part;
  Q8_REQUIRE(tiles * n_heads * splits <= 0x7fffffffu && T * ratio <= 0x7fffffffu, Q8_EUNSUPPORTED);
  AttendParams p{};
  p.cache = static_cast<const uint8_t*>(cache_dev);
  p.table = table_dev;
  p.lengths = lengths_dev;
  p.starts = starts_dev;
  p.parts = static_cast<float*>(workspace);
  p.q_stride = q_stride, p.q_head = q_head_stride, p.o_stride = o_stride, p.o_head = o_head_stride;
  p.table_stride = table_stride;
  p.n_pages = (long)n_pages;
  p.T = (int)T, p.B = n_requests, p.H = n_heads, p.ratio = ratio, p.width = width;
  p.shift = __builtin_ctz(page) - 4;
  p.tiles = (int)tiles, p.splits = (int)splits, p.window = window;
  p.scale_log2 = scale * 1.4426950408889634f;
  if (type == Q8_F16)
    return launch_any(D / 32, p, static_cast<const _Float16*>(q_dev), static_cast<_Float16*>(out_dev),
                      (hipStream_t)stream);
  return launch_any(D / 32, p, static_cast<const __bf16*>(q_dev), static_cast<__bf16*>(out_dev), (hipStream_t)stream);
}
