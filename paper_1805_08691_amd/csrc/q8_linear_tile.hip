// The 8-bit linear layer's product where rows are many: y[m][n] = tail(sum_k z_x[m][k] z_w[n][k]).
//
// A workgroup owns a tile of BN channels x BM rows and walks over K in steps of KB times 64 bytes: both operands go from memory
// to LDS without registers in between (a ring of STAGES steps, one bare barrier a step), and a wavefront multiplies its
// TN x TM squares of 32 x 32 on v_mfma_i32_32x32x32_i8.  Packed weights lie in the order in which a wavefront reads
// them; rows of activations are 64 bytes in LDS with their 16-byte chunks swapped (swz) so that neither meets a
// bank twice.  Rows of activations are the matrix instruction's rows: a lane then holds 16 rows of one channel, 32 lanes store
// neighbours (the other way round a store touched 64 lines: 4096 x 4096 x 4096 77 us instead of 65).
// Large products: 8192 x 8192 x 8192 takes 465 us, 2.36 POP/s, with the matrix cores busy 64 % of the cycles and wavefronts
// waiting in 35 % of theirs (two to a SIMD, two steps in flight), at the 1.76 GHz that power leaves; zeros go 1.2 times as fast.
// Small ones are bound by the steps of the one or two tiles that a compute unit has: 0.25 us for 128 bytes of K
// of a 64 x 64 tile, whose 16 KB take half of that out of L2 (777 x 1000 x 2048: 7.7 us).
#include "q8_linear.h"
#include <type_traits>
#pragma clang fp contract(off)

namespace {

using namespace q8;

constexpr int kXcds = 8;

template <int WN_, int WM_, int TN_, int TM_, int STAGES_, int KB_ = 1>
struct Shape {
  static constexpr int WN = WN_, WM = WM_, TN = TN_, TM = TM_, STAGES = STAGES_, KB = KB_;      // KB: 64 bytes of K each, of a step
  static constexpr int NW = WN * WM, BN = WN * TN * 32, BM = WM * TM * 32;
  static constexpr int A_BYTES = BN * kPackK, B_BYTES = BM * kPackK, BLOCK = A_BYTES + B_BYTES, STAGE_BYTES = KB * BLOCK;
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static constexpr int A_LOADS = BN / 16 / NW, B_LOADS = BM / 16 / NW, LOADS = KB * (A_LOADS + B_LOADS);
  static_assert(A_LOADS * NW * 16 == BN && B_LOADS * NW * 16 == BM, "every wavefront issues the same loads");
  static_assert((STAGES - 2) * LOADS < 64, "vmcnt is 6 bits");
};

// Value e of a lane in a square of 32 x 32: its row.
__device__ __forceinline__ constexpr int square_row(int e, int half) { return (e & 3) + 8 * (e >> 2) + 4 * half; }

template <typename Sh, typename Y, bool PAIRS>
__global__ __launch_bounds__(Sh::NW * 64) void linear_tile_kernel(const LinearParams p, Y* __restrict__ y, int tiles_n,
                                                                  int tiles_m) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TN = Sh::TN, TM = Sh::TM, NW = Sh::NW, STAGES = Sh::STAGES, LOADS = Sh::LOADS;
  extern __shared__ __attribute__((aligned(1024))) int8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_n = wave % Sh::WN, wave_m = wave / Sh::WN;

  // ---- the tile: an XCD takes a contiguous run of them, eight rows of tiles at a time
  const int total = tiles_n * tiles_m, per = (total + kXcds - 1) / kXcds;
  const int id = blockIdx.x % kXcds * per + blockIdx.x / kXcds;
  if (blockIdx.x / kXcds >= per || id >= total) return;
  constexpr int GROUP = 8;
  const int group = id / (GROUP * tiles_n), in = id - group * (GROUP * tiles_n);
  const int rows = min(GROUP, tiles_m - group * GROUP);
  const int n0 = in / rows * Sh::BN, m0 = (group * GROUP + in % rows) * Sh::BM;

  // ---- loaders.  Weights: blocks of 16 rows as they lie.  Activations: lane l takes row l / 4, slot l % 4.
  const int nk = p.ksteps;
  const int8_t* a_base = p.w + (size_t)(n0 / kPackN) * nk * 1024;
  const int8_t* b_base = p.z + (size_t)m0 * p.z_stride;
  const size_t a_all = ((size_t)((p.N + kPackN - 1) / kPackN) - n0 / kPackN) * nk * 1024;
  int a_bytes = (int)(a_all < 0x7fffffffu ? a_all : 0x7fffffffu);
  const size_t b_all = (size_t)(p.M - m0 - 1) * p.z_stride + ((p.K + 15) & ~15);
  int b_bytes = (int)(b_all < 0x7fffffffu ? b_all : 0x7fffffffu);
  int a_off[Sh::A_LOADS], b_off[Sh::B_LOADS];
#pragma unroll
  for (int i = 0; i < Sh::A_LOADS; ++i) a_off[i] = (wave + NW * i) * nk * 1024 + lane * 16;
#pragma unroll
  for (int i = 0; i < Sh::B_LOADS; ++i) {
    const int row = (wave + NW * i) * 16 + (lane >> 2);
    b_off[i] = row * (int)p.z_stride + swz<4>(row, lane & 3) * 16;
  }
  // ---- factors and bias of this lane's rows and channels
  float q_x[TM], q_w[TN], bias[TN];
#pragma unroll
  for (int j = 0; j < TM; ++j) q_x[j] = p.q_x[min(m0 + (wave_m * TM + j) * 32 + (lane & 31), p.M - 1)];
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    const int n = min(n0 + (wave_n * TN + i) * 32 + (lane & 31), p.N - 1);
    q_w[i] = p.q_w[n];
    bias[i] = p.bias ? p.bias[n] : 0.0f;
  }

  int issued = 0;
  auto issue = [&](int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < Sh::KB; ++kb) {
      const bool in_k = issued < nk;
      const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)a_base, 0, in_k ? a_bytes : 0, 0x00020000);
      const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)b_base, 0, in_k ? b_bytes : 0, 0x00020000);
      int8_t* to = lds + stage * Sh::STAGE_BYTES + kb * Sh::BLOCK;
#pragma unroll
      for (int i = 0; i < Sh::A_LOADS; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            ra, (__attribute__((address_space(3))) void*)(to + (wave + NW * i) * 1024), 16, a_off[i], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < Sh::B_LOADS; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rb, (__attribute__((address_space(3))) void*)(to + Sh::A_BYTES + (wave + NW * i) * 1024), 16, b_off[i], 0, 0, 0);
      // (a row's last step may end behind its last byte: only as far as the next row, or it reads as zeros)
      ++issued;
      a_base += 1024;
      a_bytes -= 1024;
      b_base += kPackK;
      b_bytes -= kPackK;
    }
  };

  v16i acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

  // ---- operand fragments: half h of a step is the chunks 2 h and 2 h + 1 of its rows
  const int half = lane >> 5, row = lane & 31;
  const int a_frag = wave_n * TN * 2048 + (row >> 4) * 1024 + (row & 15) * 16 + half * 256;
  const int b_frag = Sh::A_BYTES + (wave_m * TM * 32 + row) * kPackK + swz<4>(row, half) * 16;
  v4i af[2][TN], bf[2][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i) af[1][i] = v4i{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < TM; ++j) bf[1][j] = v4i{0, 0, 0, 0};
  auto load_half = [&](const int8_t* stage, auto h_c) __attribute__((always_inline)) {
    constexpr int h = decltype(h_c)::value, kb = h >> 1, half_of = h & 1;
#pragma unroll
    for (int i = 0; i < TN; ++i)
      af[h & 1][i] = *reinterpret_cast<const v4i*>(stage + kb * Sh::BLOCK + a_frag + i * 2048 + half_of * 512);
#pragma unroll
    for (int j = 0; j < TM; ++j)
      bf[h & 1][j] = *reinterpret_cast<const v4i*>(stage + kb * Sh::BLOCK + (b_frag ^ (half_of * 32)) + j * 2048);
  };
  auto multiply = [&](auto h_c) __attribute__((always_inline)) {
    constexpr int h = decltype(h_c)::value & 1;
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[h][j], af[h][i], acc[i][j], 0, 0, 0);
  };
  using std::integral_constant;
  constexpr int HALVES = 2 * Sh::KB;
  constexpr integral_constant<int, HALVES - 1> last{};

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue(s);
  __builtin_amdgcn_s_waitcnt(0xc07f);                // scalar loads are settled before the loop
  int stage = 0;
  const int steps = (nk + Sh::KB - 1) / Sh::KB;
  for (int k = 0; k < steps; ++k) {
    wait_vmcnt<(STAGES - 2) * LOADS>();
    __builtin_amdgcn_s_waitcnt(0xc07f);              // this wavefront's reads of the step before have returned
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int8_t* at = lds + stage * Sh::STAGE_BYTES;
    load_half(at, integral_constant<int, 0>{});
    issue(stage == 0 ? STAGES - 1 : stage - 1);
    multiply(last);                                  // of the step before (zeros at first)
    auto rest = [&](auto self, auto h_c) __attribute__((always_inline)) -> void {
      constexpr int h = decltype(h_c)::value;
      if constexpr (h < HALVES) {
        load_half(at, h_c);
        multiply(integral_constant<int, h - 1>{});
        self(self, integral_constant<int, h + 1>{});
      }
    };
    rest(rest, integral_constant<int, 1>{});
    // reads of the first half; then products with a load to LDS behind each, and the next half's reads between them
    __builtin_amdgcn_sched_group_barrier(0x100, TN + TM, 0);
    int loads = LOADS;
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
      for (int g = 0; g < TN * TM; ++g) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (loads > 0) {
          __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
          --loads;
        }
        if (h + 1 < HALVES) {
          const int reads = (TN + TM) * (g + 1) / (TN * TM) - (TN + TM) * g / (TN * TM);
          for (int i = 0; i < 4; ++i)
            if (i < reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
    __builtin_amdgcn_sched_barrier(0);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  multiply(last);
  wait_vmcnt<0>();                                   // (loads behind the last step write zeros into this LDS)

  // ---- tail: a lane holds 16 rows of one channel, so that 32 lanes store neighbours; 16-bit values change places
  // between two lanes first (PAIRS), which makes them two neighbours of one row each
  const unsigned sel = lane & 1 ? 0x03020706u : 0x05040100u;
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    float q[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) q[e] = __shfl(q_x[j], square_row(e, half), 64);
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      const int m = m0 + (wave_m * TM + j) * 32, n = n0 + (wave_n * TN + i) * 32 + row;
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        v[e] = (float)acc[i][j][e] * (q[e] * q_w[i]);
        if (p.bias) v[e] = v[e] + bias[i];
      }
      if constexpr (PAIRS) {
        Y* const to = y + (size_t)m * p.y_stride + (n & ~1);
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const Y two[2] = {(Y)v[e], (Y)v[e + 1]};
          unsigned own;
          __builtin_memcpy(&own, two, 4);
          const unsigned other = __builtin_amdgcn_update_dpp(0u, own, 0xb1, 0xf, 0xf, true);      // of lane ^ 1
          const unsigned out = __builtin_amdgcn_perm(other, own, sel);
          const int r = square_row(e, half) + (lane & 1);
          if (m + r < p.M && n < p.N) __builtin_memcpy(__builtin_assume_aligned(to + (size_t)r * p.y_stride, 4), &out, 4);
        }
      } else {
        Y* const to = y + (size_t)m * p.y_stride + n;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = square_row(e, half);
          if (m + r < p.M && n < p.N) to[(size_t)r * p.y_stride] = (Y)v[e];
        }
      }
    }
  }
#endif
}

template <typename Sh, typename Y, bool PAIRS>
int launch(const LinearParams& p, Y* y, hipStream_t stream) {
  // as many rows of tiles a launch as its blocks reach
  constexpr size_t kBlocks = most_blocks(Sh::NW * 64) / kXcds * kXcds;
  const size_t tn = ((size_t)p.N + Sh::BN - 1) / Sh::BN, most = kBlocks / tn * Sh::BM;
  Q8_REQUIRE(most > 0, Q8_EUNSUPPORTED);
  if constexpr (Sh::LDS_BYTES > 65536) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&linear_tile_kernel<Sh, Y, PAIRS>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, Sh::LDS_BYTES);
    if (attr != hipSuccess) return Q8_EHIP;
  }
  LinearParams part = p;
  for (size_t m = 0; m < (size_t)p.M; m += most) {
    part.z = p.z + m * p.z_stride;
    part.q_x = p.q_x + m;
    part.M = (int)(p.M - m < most ? p.M - m : most);
    const size_t tm = ((size_t)part.M + Sh::BM - 1) / Sh::BM, blocks = (tn * tm + kXcds - 1) / kXcds * kXcds;
    linear_tile_kernel<Sh, Y, PAIRS><<<(unsigned)blocks, Sh::NW * 64, Sh::LDS_BYTES, stream>>>(part, y + m * p.y_stride, (int)tn, (int)tm);
  }
  return q8_launch_status();
}

template <typename Sh>
int launch_any(const LinearParams& p, void* y, int type, hipStream_t stream) {
  return with_type(type, [&](auto one) {
    using Y = decltype(one);
    if constexpr (sizeof(Y) == 2) {
      if (q8_aligned(y, 4) && p.y_stride % 2 == 0 && p.N % 2 == 0) return launch<Sh, Y, true>(p, static_cast<Y*>(y), stream);
    }
    return launch<Sh, Y, false>(p, static_cast<Y*>(y), stream);
  });
}

}  // namespace

namespace q8 {

int linear_tile(const LinearParams& p, void* y, int type, int variant, hipStream_t stream) {
  switch (variant) {
    case 0: return launch_any<Shape<2, 2, 1, 1, 4, 2>>(p, y, type, stream);      // 64 channels x 64 rows
    case 1: return launch_any<Shape<2, 2, 2, 1, 3, 2>>(p, y, type, stream);      // 128 x 64
    case 2: return launch_any<Shape<2, 2, 2, 2, 4>>(p, y, type, stream);      // 128 x 128
    case 3: return launch_any<Shape<2, 4, 2, 1, 3, 2>>(p, y, type, stream);      // 128 x 128, eight wavefronts
    case 4: return launch_any<Shape<2, 4, 4, 2, 2, 2>>(p, y, type, stream);      // 256 x 256
  }
  return Q8_EUNSUPPORTED;
}

}  // namespace q8
