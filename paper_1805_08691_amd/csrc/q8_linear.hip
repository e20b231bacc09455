// The 8-bit linear layer on rows of real values, one factor per row of activations (a token, known only when the
// values are) and one per row of weights (an output channel):
//   q_x[m] = max_k |x[m,k]| * fl(1/127),  z_x = Eq. Q(x[m,:], q_x[m])
//   y[m,n] = fp32(sum_k z_x[m,k] z_w[n,k]) * (q_x[m] q_w[n]) + bias[n]          (Eq. x, Eq. D)
// The sum is exact in int32 (128 * 128 * K < 2^31 for K <= 131071); the tail is three fp32 operations and the
// rounding to y's type.
#include "q8_common.h"
#include "q8_linear.h"
#include "q8_quant.h"
#include <math.h>
#pragma clang fp contract(off)

namespace {

using namespace q8;

constexpr int kMaxK = 131071;

inline size_t round_up(size_t a, size_t b) { return (a + b - 1) / b * b; }

// ---------------------------------------------------------------- rows to codes ----------
// A row belongs to WAVES wavefronts of a block of four: the maximum, then the codes.  The first HELD chunks of 8 values
// of a lane stay in registers between the two; what a longer row has beyond them is read again.  Bound by memory where
// rows are many (8192 x 8192 in bf16: 42 us, 4.8 TB/s), by the launch and one trip to memory where they are few (4 us).
template <typename V, bool ALIGNED, int WAVES, int HELD>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const V* __restrict__ x, size_t M, int K, size_t x_stride,
                                                            int8_t* __restrict__ z, size_t z_stride,
                                                            float* __restrict__ q_x) {
  constexpr int THREADS = WAVES * 64, STEP = THREADS * 8;
  const size_t row = WAVES == 4 ? blockIdx.x : (size_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (row >= M) return;
  const V* __restrict__ xr = x + row * x_stride;
  int8_t* __restrict__ zr = z + row * z_stride;
  const int tid = threadIdx.x % THREADS, body = K & ~7;
  V held[HELD][8];
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (tid * 8 + i * STEP < body)
      __builtin_memcpy(held[i], __builtin_assume_aligned(xr + tid * 8 + i * STEP, ALIGNED ? 16 : sizeof(V)), sizeof(held[i]));
  const float tail = tid < K - body ? (float)xr[body + tid] : 0.0f;
  // all of a lane's values one after the other
  auto each = [&](auto use) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (tid * 8 + i * STEP < body) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)held[i][e];
        use(v, tid * 8 + i * STEP);
      }
    for (int k = tid * 8 + HELD * STEP; k < body; k += STEP) {
      float v[8];
      load_values<8, ALIGNED>(xr + k, v);
      use(v, k);
    }
  };
  unsigned all = 0;
  each([&](const float (&v)[8], int) { all = row_bits8(v, all); });
  const bool finite = all < kNotFinite;
  float m = __uint_as_float(all);
  if (!finite) {
    m = 0.0f;
    each([&](const float (&v)[8], int) { m = row_max8(v, m); });
  }
  m = fmaxf(m, finite_abs(tail));
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if constexpr (WAVES == 4) {
    __shared__ float wave_max[4];
    if ((tid & 63) == 0) wave_max[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  }
  float q = __fmul_rn(m, 1.0f / 127.0f);
  q = q > 0.0f ? q : 1.0f;
  if (tid == 0) q_x[row] = q;
  const float inv_q = __fdiv_rn(1.0f, q);
  each([&](const float (&v)[8], int k) { *reinterpret_cast<uint2*>(zr + k) = row_codes(v, q, inv_q, finite); });
  if (tid < K - body) zr[body + tid] = (int8_t)(tail == tail ? quant1(tail, q, -128.0f, 127.0f) : 0);
}

template <typename V, bool ALIGNED>
int launch_quantize_rows(const V* x, size_t M, int K, size_t x_stride, int8_t* z, size_t z_stride, float* q_x,
                         hipStream_t stream) {
  // (a wavefront to a short row, a block to others: 16384 rows of 512 bf16 values 10.1 and 16.9 us, of 1024 15.0 and 20.0)
  const size_t rows = K <= 1024 ? 4 : 1, most = rows * most_blocks(256);       // of a block, of a launch
  for (size_t m = 0; m < M; m += most) {
    const size_t n = M - m < most ? M - m : most;
    const V* const from = x + m * x_stride;
    int8_t* const to = z + m * z_stride;
    if (rows == 4)
      quantize_rows_kernel<V, ALIGNED, 1, 2><<<(unsigned)((n + 3) / 4), 256, 0, stream>>>(from, n, K, x_stride, to, z_stride, q_x + m);
    else
      quantize_rows_kernel<V, ALIGNED, 4, 4><<<(unsigned)n, 256, 0, stream>>>(from, n, K, x_stride, to, z_stride, q_x + m);
  }
  return q8_launch_status();
}

// ---------------------------------------------------------------- weights ----------------
// Packed: blocks of 16 rows x 64 reduction bytes, 1 KB each, [N / 16][K / 64]; inside a block lane l of a wavefront
// holds 16 bytes: row l % 16, bytes 16 (l / 16) .. + 15, the operand of one 16x16x64 product.  Zeros beyond N and K.
__global__ __launch_bounds__(256) void linear_pack_kernel(const int8_t* __restrict__ w, int N, int K, int ksteps,
                                                          size_t chunks, int8_t* __restrict__ packed) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const int lane = (int)(i % 64);
  const size_t block = i / 64;
  const size_t n = block / ksteps * kPackN + lane % 16;
  const int k = (int)(block % ksteps) * kPackK + lane / 16 * 16;
  v4i v = {0, 0, 0, 0};
  int8_t b[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) b[e] = n < (size_t)N && k + e < K ? w[n * K + k + e] : (int8_t)0;
  __builtin_memcpy(&v, b, 16);
  reinterpret_cast<v4i*>(packed)[i] = v;
}

// ---------------------------------------------------------------- product ----------------
// Rows at any distance: one wavefront per 16 channels x 16 rows, operands straight from memory.  For rows more than 4 MB
// apart only, where the offsets of a tile would pass 31 bits; bound by the latency of its loads.
template <typename Y, bool VEC>
__global__ __launch_bounds__(256) void linear_any_kernel(const LinearParams p, Y* __restrict__ y) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nb = blockIdx.x * 4 + wave;
  if (nb * kPackN >= p.N) return;
  const int m0 = blockIdx.y * 16;
  const int row = min(m0 + (lane & 15), p.M - 1), chunk = (lane >> 4) * 16;
  const int8_t* __restrict__ z = p.z + (size_t)row * p.z_stride + chunk;
  const v4i* __restrict__ w = reinterpret_cast<const v4i*>(p.w) + (size_t)nb * p.ksteps * 64 + lane;
  v4i acc = {0, 0, 0, 0};
  for (int s = 0; s < p.ksteps; ++s) {
    v4i b = {0, 0, 0, 0};
    if (s * kPackK + chunk < p.K) b = *reinterpret_cast<const v4i*>(z + s * kPackK);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[(size_t)s * 64], b, acc, 0, 0, 0);
  }
  const int m = m0 + (lane & 15), n = nb * kPackN + 4 * (lane >> 4);
  if (m >= p.M || n >= p.N) return;
  const int v[4] = {acc[0], acc[1], acc[2], acc[3]};
  finish_outputs<4, VEC>(p, y, m, n, p.q_x[m], v);
}

template <typename Y>
int launch_any_rows(const LinearParams& p, Y* y, hipStream_t stream) {
  const dim3 grid((unsigned)((p.N + 63) / 64), (unsigned)((p.M + 15) / 16));
  const bool vec = q8_aligned(y, 4 * sizeof(Y)) && p.y_stride % 4 == 0;
  if (vec)
    linear_any_kernel<Y, true><<<grid, 256, 0, stream>>>(p, y);
  else
    linear_any_kernel<Y, false><<<grid, 256, 0, stream>>>(p, y);
  return q8_launch_status();
}

// The builds of the product, and what the choice between them goes by: a launch of `tiles` tiles takes
//   base + (share * tiles / 256 + (1 - share) * ceil(tiles / 256)) * (round + per_k * K / 1024)
// us (256 compute units; a round costs its steps along K and a constant; `share` of a round that is not full is saved),
// and no less than its operands' way from memory, m = 2.2 us + bytes at 5.4 TB/s; the lesser of the two counts a
// fifth.  The constants are fitted to every build on 128 sizes (1 .. 4096 rows, 512 .. 16384 channels and values a
// row); there the pick is 1.1 % longer than the best build in the mean and 25 % at most.
struct Variant {
  const char* name;
  int bn, bm;                  // channels and rows of a tile
  int columns, squares;        // rows build: packed columns and squares of 16 rows
  int tile;                    // tile build, or -1
  float base, round, per_k, share;
};
constexpr Variant kVariants[] = {
    {"rows_16x16", 16, 16, 1, 1, -1, 1.89f, 0.92f, 0.46f, 0.30f},
    {"rows_32x16", 32, 16, 2, 1, -1, 1.00f, 1.84f, 0.61f, 0.34f},
    {"rows_64x16", 64, 16, 4, 1, -1, 1.00f, 2.40f, 1.00f, 0.00f},
    {"rows_64x32", 64, 32, 4, 2, -1, 1.00f, 1.91f, 1.48f, 0.09f},
    {"tile_64x64", 64, 64, 0, 0, 0, 2.10f, 1.09f, 1.58f, 0.29f},
    {"tile_128x64", 128, 64, 0, 0, 1, 2.01f, 1.53f, 2.49f, 0.21f},
    {"tile_128x128", 128, 128, 0, 0, 2, 1.00f, 3.35f, 3.40f, 0.08f},
    {"tile_128x128_8", 128, 128, 0, 0, 3, 1.00f, 3.30f, 3.63f, 0.00f},
    {"tile_256x256", 256, 256, 0, 0, 4, 1.00f, 7.29f, 9.55f, 0.80f},
    {"rows_any", 16, 16, 0, 0, -1, 0.0f, 0.0f, 0.0f, 0.0f}};      // rows so far apart that a tile passes 2^31 bytes
constexpr int kNumVariants = sizeof(kVariants) / sizeof(kVariants[0]);
constexpr size_t kTileStride = 1 << 22;      // 256 rows of a tile stay below 2^31 bytes
constexpr int kMostRows = 16 * 65535;        // of the builds that are no tiles: a launch's second dimension
// ... and its first one, blocks of eight wavefronts at most.
bool reached(const Variant& v, int M, int N) {
  return v.tile >= 0 || (M <= kMostRows && ((size_t)N + v.bn - 1) / v.bn <= most_blocks(512));
}

int pick(const LinearParams& p) {
  int best = -1;
  float least = 0.0f;
  const float memory = 2.2f + ((float)p.N + (float)p.M) * (float)p.K / 5.4e6f;
  for (int i = 0; i + 1 < kNumVariants; ++i) {
    const Variant& v = kVariants[i];
    if (!reached(v, p.M, p.N)) continue;
    const float tiles = (float)((p.N + v.bn - 1) / v.bn) * (float)((p.M + v.bm - 1) / v.bm), rounds = tiles / 256.0f;
    const float passes = fmaxf(1.0f, v.share * rounds + (1.0f - v.share) * ceilf(rounds));
    const float time = v.base + passes * (v.round + v.per_k * (float)p.K / 1024.0f);
    const float cost = fmaxf(time, memory) + 0.2f * fminf(time, memory);
    if (best < 0 || cost < least) best = i, least = cost;
  }
  return best;
}

// Codes [M][round_up(K, 16)], then the rows' factors.
size_t codes_bytes(size_t M, int K) { return round_up(M * round_up(K, 16), 256); }

bool sizes_ok(size_t M, int N, int K) { return N >= 0 && K >= 1 && K <= kMaxK && M <= 0x7fffffffu; }

}  // namespace

extern "C" int q8_quantize_rows(const void* x_dev, int type, size_t M, int K, size_t x_stride, int8_t* z_dev,
                                size_t z_stride, float* q_x_dev, void* stream) {
  Q8_REQUIRE(type_ok(type) && K >= 1, Q8_EINVAL);
  if (M == 0) return Q8_OK;
  Q8_REQUIRE(M <= 0x7fffffffu, Q8_EUNSUPPORTED);
  Q8_REQUIRE(x_dev && z_dev && q_x_dev && x_stride >= (size_t)K && z_stride >= (size_t)K, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(x_dev, type_bytes(type)) && q8_aligned(q_x_dev, 4), Q8_EALIGN);
  Q8_REQUIRE(q8_aligned(z_dev, 16) && z_stride % 16 == 0, Q8_EALIGN);
  return with_type(type, [&](auto v) {
    using V = decltype(v);
    const V* const x = static_cast<const V*>(x_dev);
    if (q8_aligned(x, 16) && x_stride * sizeof(V) % 16 == 0)
      return launch_quantize_rows<V, true>(x, M, K, x_stride, z_dev, z_stride, q_x_dev, (hipStream_t)stream);
    return launch_quantize_rows<V, false>(x, M, K, x_stride, z_dev, z_stride, q_x_dev, (hipStream_t)stream);
  });
}

extern "C" size_t q8_linear_packed_bytes(int N, int K) {
  if (N < 0 || K < 1 || K > kMaxK) return 0;
  return round_up(N, kPackN) * round_up(K, kPackK);
}

extern "C" int q8_linear_pack(const int8_t* z_w_dev, int N, int K, void* packed_dev, void* stream) {
  Q8_REQUIRE(N >= 0 && K >= 1, Q8_EINVAL);
  Q8_REQUIRE(K <= kMaxK, Q8_EUNSUPPORTED);
  if (N == 0) return Q8_OK;
  Q8_REQUIRE(z_w_dev && packed_dev, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(packed_dev, 16), Q8_EALIGN);
  const size_t chunks = q8_linear_packed_bytes(N, K) / 16, blocks = (chunks + 255) / 256;
  Q8_REQUIRE(blocks <= most_blocks(256), Q8_EUNSUPPORTED);
  linear_pack_kernel<<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>(
      z_w_dev, N, K, (int)(round_up(K, kPackK) / kPackK), chunks, static_cast<int8_t*>(packed_dev));
  return q8_launch_status();
}

extern "C" int q8_linear_num_variants(void) { return kNumVariants; }

extern "C" const char* q8_linear_variant_name(int variant) {
  return variant >= 0 && variant < kNumVariants ? kVariants[variant].name : "unsupported";
}

extern "C" int q8_linear_int8_variant(const int8_t* z_x_dev, size_t z_stride, const float* q_x_dev, size_t M, int N,
                                      int K, const void* packed_dev, const float* q_w_dev, const float* bias_dev,
                                      void* y_dev, int type, size_t y_stride, int variant, void* stream) {
  Q8_REQUIRE(variant < kNumVariants, Q8_EINVAL);
  Q8_REQUIRE(type_ok(type) && N >= 0 && K >= 1, Q8_EINVAL);
  Q8_REQUIRE(sizes_ok(M, N, K), Q8_EUNSUPPORTED);
  if (M == 0 || N == 0) return Q8_OK;
  Q8_REQUIRE(z_x_dev && q_x_dev && packed_dev && q_w_dev && y_dev, Q8_EINVAL);
  Q8_REQUIRE(z_stride >= (size_t)K && y_stride >= (size_t)N, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(z_x_dev, 16) && z_stride % 16 == 0 && q8_aligned(packed_dev, 16), Q8_EALIGN);
  Q8_REQUIRE(q8_aligned(q_x_dev, 4) && q8_aligned(q_w_dev, 4) && q8_aligned(bias_dev, 4) &&
                 q8_aligned(y_dev, type_bytes(type)), Q8_EALIGN);
  const LinearParams p{z_x_dev, q_x_dev, static_cast<const int8_t*>(packed_dev), q_w_dev, bias_dev, z_stride,
                       y_stride, (int)M, N, K, (int)(round_up(K, kPackK) / kPackK)};
  if (variant < 0) variant = z_stride <= kTileStride ? pick(p) : kNumVariants - 1;
  const Variant& v = kVariants[variant];
  Q8_REQUIRE(reached(v, (int)M, N), Q8_EUNSUPPORTED);
  if (v.columns) return linear_rows(p, y_dev, type, v.columns, v.squares, (hipStream_t)stream);
  if (v.tile >= 0 && z_stride > kTileStride) return Q8_EUNSUPPORTED;
  if (v.tile >= 0) return linear_tile(p, y_dev, type, v.tile, (hipStream_t)stream);
  return with_type(type, [&](auto v) { return launch_any_rows(p, static_cast<decltype(v)*>(y_dev), (hipStream_t)stream); });
}

extern "C" int q8_linear_int8(const int8_t* z_x_dev, size_t z_stride, const float* q_x_dev, size_t M, int N, int K,
                              const void* packed_dev, const float* q_w_dev, const float* bias_dev, void* y_dev,
                              int type, size_t y_stride, void* stream) {
  return q8_linear_int8_variant(z_x_dev, z_stride, q_x_dev, M, N, K, packed_dev, q_w_dev, bias_dev, y_dev, type, y_stride,
                                -1, stream);
}

extern "C" size_t q8_linear_workspace_bytes(size_t M, int N, int K) {
  if (!sizes_ok(M, N, K)) return 0;
  return codes_bytes(M, K) + round_up(M * 4, 256);
}

extern "C" int q8_linear(const void* x_dev, int x_type, size_t x_stride, size_t M, int N, int K,
                         const void* packed_dev, const float* q_w_dev, const float* bias_dev, void* y_dev, int y_type,
                         size_t y_stride, void* workspace, size_t workspace_bytes, void* stream) {
  Q8_REQUIRE(type_ok(x_type) && type_ok(y_type) && N >= 0 && K >= 1, Q8_EINVAL);
  Q8_REQUIRE(sizes_ok(M, N, K), Q8_EUNSUPPORTED);
  if (M == 0 || N == 0) return Q8_OK;
  Q8_REQUIRE(x_dev && packed_dev && q_w_dev && y_dev && workspace, Q8_EINVAL);
  Q8_REQUIRE(x_stride >= (size_t)K && y_stride >= (size_t)N, Q8_EINVAL);
  Q8_REQUIRE(q8_aligned(workspace, 256) && q8_aligned(x_dev, type_bytes(x_type)) && q8_aligned(packed_dev, 16) &&
                 q8_aligned(q_w_dev, 4) && q8_aligned(bias_dev, 4) && q8_aligned(y_dev, type_bytes(y_type)), Q8_EALIGN);
  Q8_REQUIRE(workspace_bytes >= q8_linear_workspace_bytes(M, N, K), Q8_EWORKSPACE);
  if (linear_rows_take_real((int)M, N, K)) {
    const LinearParams p{nullptr, nullptr, static_cast<const int8_t*>(packed_dev), q_w_dev, bias_dev, 0, y_stride, (int)M,
                         N, K, (int)(round_up(K, kPackK) / kPackK)};
    return linear_rows_real(p, x_dev, x_type, x_stride, y_dev, y_type, (hipStream_t)stream);
  }
  int8_t* const z = static_cast<int8_t*>(workspace);
  float* const q_x = reinterpret_cast<float*>(z + codes_bytes(M, K));
  const size_t z_stride = round_up(K, 16);
  const int rc = q8_quantize_rows(x_dev, x_type, M, K, x_stride, z, z_stride, q_x, stream);
  if (rc != Q8_OK) return rc;
  return q8_linear_int8(z, z_stride, q_x, M, N, K, packed_dev, q_w_dev, bias_dev, y_dev, y_type, y_stride, stream);
}
