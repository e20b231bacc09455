// The 8-bit linear layer's product where rows are few: bound by the weights' way from memory, each of which is
// multiplied by 16 rows at most before the next is needed.
//
// A workgroup of eight wavefronts owns NB columns of packed blocks (16 channels each) and MT squares of 16 rows; the
// wavefronts take the blocks of K in turn, straight from memory to registers, and multiply them on
// v_mfma_i32_16x16x64_i8: no operand is shared inside a workgroup, so nothing goes through LDS and no wavefront waits
// for another.  Their sums meet in LDS at the end (integers: any order gives the same bits).  With real values as input (REAL) the workgroup makes the rows' codes
// itself, in LDS, while its first weights are on their way: one launch instead of two.  1 x 4096 -> 4096 takes 4.5 us (16.8 MB of
// weights: 3.7 TB/s with the launch), 16 x 4096 -> 16384 15 (4.5 TB/s).
#include "q8_linear.h"
#include "q8_quant.h"
#pragma clang fp contract(off)

namespace {

using namespace q8;

constexpr int kWavesK = 8;                    // wavefronts, which share K
constexpr int kThreads8 = kWavesK * 64;
// Real values, of which a lane holds 4 vectors of 8: one or two rows that the workgroup takes together, or two rows of a
// wavefront (WAVE), SPAN vectors of each.
constexpr int kRealVectors = 4, kSpan = 2, kWaveRows = kWavesK * (kRealVectors / kSpan);

// The largest of a wavefront's values (none is negative or no number), in lane 63.
__device__ __forceinline__ float wave_max(float v) {
  auto step = [&](auto ctrl_c) {
    constexpr int ctrl = decltype(ctrl_c)::value;
    const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, true);
    v = fmaxf(v, __int_as_float(o));
  };
  step(std::integral_constant<int, 0x111>{});        // row_shr 1, 2, 4, 8: lane 15 of each row of 16
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  step(std::integral_constant<int, 0x118>{});
  step(std::integral_constant<int, 0x142>{});        // row_bcast 15 and 31: from each row to the next ones
  step(std::integral_constant<int, 0x143>{});
  return v;
}

template <int NB, int MT, typename X, typename Y, bool VEC, bool REAL, bool WAVE>
__global__ __launch_bounds__(kThreads8) void linear_rows_kernel(const LinearParams p, const X* __restrict__ x,
                                                                size_t x_stride, Y* __restrict__ y) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int kAhead = NB + MT <= 5 ? 4 : 2;                // steps of a wavefront in flight
  extern __shared__ __attribute__((aligned(16))) int8_t lds[];
  __shared__ unsigned row_max[kWaveRows];                     // (bits of a number that is none negative)
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nb = blockIdx.x * NB, nk = p.ksteps;              // first packed column, of NB
  const int chunk = (lane >> 4) * 16;
  const int pitch = nk * kPackK + 16;                         // of a row of codes in LDS
  const int m_grid = blockIdx.y * (16 * MT);

  // ---- real values: vector u of a lane is one of row u / turns, 512 vectors of which are a turn; or of the wavefront's
  // row u / kSpan
  float r[kRealVectors][8];
  const int turns = (p.K + kThreads8 * 8 - 1) / (kThreads8 * 8), vectors = p.M * turns;
  auto row_of = [&](int u) { return WAVE ? wave + u / kSpan * kWavesK : u / turns; };
  auto first_of = [&](int u) { return WAVE ? (lane + u % kSpan * 64) * 8 : (tid + (u - u / turns * turns) * kThreads8) * 8; };
  auto given = [&](int u) { return WAVE ? row_of(u) < p.M && u % kSpan * 512 < p.K : u < vectors; };
  if constexpr (REAL) {
    if (!WAVE && tid < kWaveRows) row_max[tid] = 0;
#pragma unroll
    for (int u = 0; u < kRealVectors; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[u][e] = 0.0f;
      if (given(u)) {
        const int k = first_of(u);
        const X* from = x + row_of(u) * x_stride + k;
        if (k + 8 <= p.K) {
          load_values<8, false>(from, r[u]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (k + e < p.K) r[u][e] = (float)from[e];
        }
      }
    }
  }

  // ---- the first blocks of the wavefront's share: weights (zeros behind the last), and codes that lie in memory
  __amdgpu_buffer_rsrc_t w[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const bool in_n = (nb + c) * kPackN < p.N;
    w[c] = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w + (size_t)(in_n ? nb + c : nb) * nk * 1024), 0,
                                             in_n ? nk * 1024 : 0, 0x00020000);
  }
  auto load_weights = [&](int c, int s) {
    return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(w[c], s * 1024 + lane * 16, 0, 0));
  };
  const int8_t* rows[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = min(m_grid + t * 16 + (lane & 15), p.M - 1);
    if constexpr (REAL) rows[t] = lds + m * pitch;
    else rows[t] = p.z + (size_t)m * p.z_stride;
  }
  // (what is read behind K stands beside zero weights: any bytes will do)
  auto load_row = [&](int t, int s) {
    const int at = s * kPackK + chunk;
    return *reinterpret_cast<const v4i*>(rows[t] + (at < p.K ? at : 0));
  };
  v4i a[kAhead][NB], b[REAL ? 1 : kAhead][MT];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
#pragma unroll
    for (int c = 0; c < NB; ++c) a[u][c] = load_weights(c, wave + u * kWavesK);
    if constexpr (!REAL) {
#pragma unroll
      for (int t = 0; t < MT; ++t) b[u][t] = load_row(t, wave + u * kWavesK);
    }
  }
  auto factor = [&](unsigned most) {
    const float q = __fmul_rn(__uint_as_float(most), 1.0f / 127.0f);
    return q > 0.0f ? q : 1.0f;
  };
  if constexpr (REAL && WAVE) {
#pragma unroll
    for (int i = 0; i < kRealVectors; i += kSpan)
      if (row_of(i) < p.M) {
        unsigned all = 0;
#pragma unroll
        for (int u = i; u < i + kSpan; ++u) all = row_bits8(r[u], all);
        const bool finite = all < kNotFinite;
        float most = __uint_as_float(all);
        if (!finite) {
          most = 0.0f;
#pragma unroll
          for (int u = i; u < i + kSpan; ++u) most = row_max8(r[u], most);
        }
        const unsigned bits = __builtin_amdgcn_readlane(__float_as_uint(wave_max(most)), 63);
        const float q = factor(bits), inv_q = __fdiv_rn(1.0f, q);
        if (lane == 0) row_max[row_of(i)] = bits;
#pragma unroll
        for (int u = i; u < i + kSpan; ++u)
          if (first_of(u) < p.K) *reinterpret_cast<uint2*>(lds + row_of(u) * pitch + first_of(u)) = row_codes(r[u], q, inv_q, finite);
      }
    lds_barrier();
  } else if constexpr (REAL) {
    lds_barrier();                                            // row_max is zero
    bool finite = true;
#pragma unroll
    for (int u = 0; u < kRealVectors; ++u)
      if (given(u)) {
        const unsigned all = row_bits8(r[u], 0);
        finite &= all < kNotFinite;
        const float m = wave_max(all < kNotFinite ? __uint_as_float(all) : row_max8(r[u], 0.0f));
        if (lane == 63) atomicMax(&row_max[row_of(u)], __float_as_uint(m));
      }
    lds_barrier();
#pragma unroll
    for (int u = 0; u < kRealVectors; ++u)
      if (given(u)) {
        const int row = row_of(u), k = first_of(u);
        const float q = factor(row_max[row]);
        if (k < p.K) *reinterpret_cast<uint2*>(lds + row * pitch + k) = row_codes(r[u], q, __fdiv_rn(1.0f, q), finite);
      }
    lds_barrier();
  }

  v4i acc[NB][MT];
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[c][t] = v4i{0, 0, 0, 0};
  auto steps = [&](int s0, auto more_c) __attribute__((always_inline)) {
    constexpr bool more = decltype(more_c)::value;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int s = s0 + u * kWavesK, next = s + kAhead * kWavesK;
      if constexpr (REAL) {
#pragma unroll
        for (int t = 0; t < MT; ++t) b[0][t] = load_row(t, s);
      }
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][c], b[REAL ? 0 : u][t], acc[c][t], 0, 0, 0);
      if constexpr (more) {
#pragma unroll
        for (int c = 0; c < NB; ++c) a[u][c] = load_weights(c, next);
        if constexpr (!REAL) {
#pragma unroll
          for (int t = 0; t < MT; ++t) b[u][t] = load_row(t, next);
        }
      }
    }
  };
  int s0 = wave;
  for (; s0 + kAhead * kWavesK < nk; s0 += kAhead * kWavesK) steps(s0, std::true_type{});
  if (s0 < nk) steps(s0, std::false_type{});

  // ---- the wavefronts' sums, up to four squares of 16 x 16 at a time
  constexpr int PART = NB * MT < 4 ? NB * MT : 4;
  __shared__ v4i sums[kWavesK][PART][64];
#pragma unroll
  for (int part = 0; part < NB * MT; part += PART) {
    if (part) lds_barrier();                                  // the part before has been read
#pragma unroll
    for (int i = 0; i < PART; ++i) sums[wave][i][lane] = acc[(part + i) / MT][(part + i) % MT];
    lds_barrier();
    if (wave < PART) {
      v4i total = sums[0][wave][lane];
#pragma unroll
      for (int u = 1; u < kWavesK; ++u) total += sums[u][wave][lane];
      const int c = (part + wave) / MT, t = (part + wave) % MT;
      const int m = m_grid + t * 16 + (lane & 15), n = (nb + c) * kPackN + 4 * (lane >> 4);
      if (m < p.M && n < p.N) {
        float q;
        if constexpr (REAL) q = factor(row_max[m]);
        else q = p.q_x[m];
        const int v[4] = {total[0], total[1], total[2], total[3]};
        finish_outputs<4, VEC>(p, y, m, n, q, v);
      }
    }
  }
#endif
}

template <int NB, int MT, typename Y>
int launch_codes(const LinearParams& p, Y* y, hipStream_t stream) {
  const dim3 grid((unsigned)((p.N + kPackN * NB - 1) / (kPackN * NB)), (unsigned)((p.M + 16 * MT - 1) / (16 * MT)));
  const bool vec = q8_aligned(y, 4 * sizeof(Y)) && p.y_stride % 4 == 0;
  if (vec)
    linear_rows_kernel<NB, MT, int8_t, Y, true, false, false><<<grid, kThreads8, 0, stream>>>(p, nullptr, 0, y);
  else
    linear_rows_kernel<NB, MT, int8_t, Y, false, false, false><<<grid, kThreads8, 0, stream>>>(p, nullptr, 0, y);
  return q8_launch_status();
}

// Whether real values are taken, a row to a wavefront, or as one or two rows by the workgroup together.  Every workgroup
// makes the rows' codes again; the launch that this saves takes 3 us.  us of the layer in one launch and in two, a row to a
// wavefront: 1024 -> 4096 3 rows 4.7 / 6.5, 8 4.8 / 7.4, 16 7.0 / 8.0; 884 -> 2439 3 rows 5.1 / 6.6, 16 6.9 / 7.7; but
// 512 -> 16384 16 rows 10.8 / 8.4, 2048 -> 2048 16 rows 9.1 / 7.5.  Together, 1.1 us a row: 4096 -> 4096 1 row 5.5 / 8.2,
// 2 6.7 / 8.3, 3 7.8 / 8.4, 4 8.9 / 8.5; 4096 -> 16384 14.2 / 16.9, 16.4 / 17.1, 18.8 / 17.4; 16384 -> 4096 1 row 18.4 / 23.
bool real_rows_of_waves(int M, int N, int K) { return M > 1 && M <= kWaveRows && K <= kSpan * 512 && (M <= kWavesK || N <= 8192); }
bool real_rows_together(int M, int K) { return M <= 2 && M * ((K + kThreads8 * 8 - 1) / (kThreads8 * 8)) <= kRealVectors; }

template <int NB, typename X, typename Y>
int launch_real(const LinearParams& p, const X* x, size_t x_stride, Y* y, hipStream_t stream) {
  const dim3 grid((unsigned)((p.N + kPackN * NB - 1) / (kPackN * NB)));
  const size_t bytes = (size_t)p.M * (p.ksteps * kPackK + 16);
  const bool vec = q8_aligned(y, 4 * sizeof(Y)) && p.y_stride % 4 == 0;
  auto go = [&](auto vec_c, auto wave_c) {
    linear_rows_kernel<NB, 1, X, Y, decltype(vec_c)::value, true, decltype(wave_c)::value>
        <<<grid, kThreads8, bytes, stream>>>(p, x, x_stride, y);
  };
  using T = std::true_type;
  using F = std::false_type;
  const bool wave = real_rows_of_waves(p.M, p.N, p.K);
  if (vec && wave) go(T{}, T{});
  else if (vec) go(T{}, F{});
  else if (wave) go(F{}, T{});
  else go(F{}, F{});
  return q8_launch_status();
}

}  // namespace

namespace q8 {

int linear_rows(const LinearParams& p, void* y, int type, int columns, int squares, hipStream_t stream) {
  return with_type(type, [&](auto one) {
    using Y = decltype(one);
    Y* const to = static_cast<Y*>(y);
    switch (columns * 8 + squares) {
      case 1 * 8 + 1: return launch_codes<1, 1>(p, to, stream);
      case 2 * 8 + 1: return launch_codes<2, 1>(p, to, stream);
      case 4 * 8 + 1: return launch_codes<4, 1>(p, to, stream);
      case 4 * 8 + 2: return launch_codes<4, 2>(p, to, stream);
    }
    return (int)Q8_EUNSUPPORTED;
  });
}

bool linear_rows_take_real(int M, int N, int K) {
  return (size_t)N <= kPackN * most_blocks(kThreads8) && (real_rows_of_waves(M, N, K) || real_rows_together(M, K));
}

int linear_rows_real(const LinearParams& p, const void* x, int x_type, size_t x_stride, void* y, int type,
                     hipStream_t stream) {
  return with_type(x_type, [&](auto xv) {
    return with_type(type, [&](auto yv) {
      return launch_real<1>(p, static_cast<const decltype(xv)*>(x), x_stride, static_cast<decltype(yv)*>(y), stream);
    });
  });
}

}  // namespace q8
