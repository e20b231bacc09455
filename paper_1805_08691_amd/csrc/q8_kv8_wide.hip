// Attention over the paged 8-bit cache where a request has many columns (prompts, in pieces or whole; a decoder's rows over an
// encoder's states): the mathematics and the layouts of q8_kv8_attend.hip.
//
// A workgroup of four wavefronts owns 128 columns that share a key head, 32 of each wavefront's, and walks over the
// keys they see, 64 at a time.  The codes of the next step go from memory to registers, a quarter to a wavefront, and become
// operands of the matrix instruction in LDS, whole numbers in binary16, in the order in which a wavefront reads them; all
// wavefronts multiply all of them.
#include "q8_kv8_attend.h"

namespace {

using namespace q8;

[[maybe_unused]] constexpr int kTiles = kWideTiles;
[[maybe_unused]] constexpr float kSlack = 8.0f; // powers of two that a maximum may grow by before sums are made relative to it
[[maybe_unused]] constexpr int kLift = 3;       // and that probabilities are scaled by beside their factors: 3 + 4 + 8 < 16

template <int G>
struct Wide {
  static constexpr int OPERANDS = 4096 * G, LDS = 2 * OPERANDS;
};

template <int G, typename V>
__global__ __launch_bounds__(256, G <= 5 ? 2 : 1) void kv8_wide_kernel(const AttendParams p, const V* __restrict__ q,
                                                          V* __restrict__ out) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int D = 32 * G, CT = 2 * G, CHUNKS = (G + 1) / 2, SIXTEEN = kv8_sixteen(D), MINE = (CT + kWaves - 1) / kWaves;
  using W = Wide<G>;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, j = lane >> 4;
  const Codes codes;
  Part a;
  Tile t;
  // (whole tiles: the last of a request see most keys, so they go first)
  const int id = p.parts ? (int)blockIdx.x : (p.tiles - 1 - (int)blockIdx.x / p.H) * p.H + (int)blockIdx.x % p.H;
  if (!find_part<kWideCols, kWideParts>(p, id, shared, &a, &t)) return;
  const int head = a.head, start = t.lo + a.step0 * kStep, steps = a.step1 - a.step0;
  const int last = min(t.lo + t.steps * kStep, t.len);

  // ---- loads: lane l holds where sixteen l % 4 of step l / 4 (of 16) lies, bit l of `held` whether it is there.  One that is
  // not is read as the cache's first.  Wave w takes keys' tile w and the values' tiles w, w + 4, ..
  const int* __restrict__ table = p.table + t.b * p.table_stride;
  long where = 0;
  unsigned long held = 0;
  auto find_sixteens = [&](int s0) {
    const int at = (start >> 4) + s0 * 4 + lane;
    int page = -1;
    if (at * 16 < last) page = table[at >> p.shift];
    const bool in = page >= 0 && page < p.n_pages;
    where = in ? ((((long)page * p.H + head) << p.shift) + (at & ((1 << p.shift) - 1))) * SIXTEEN : 0;
    held = __ballot(in);
  };
  uint4 kc[CHUNKS], vc[MINE];
  float2 factors = {0.0f, 0.0f};
  unsigned next_there = 0;
  auto issue = [&](int s) __attribute__((always_inline)) {
    if ((s & 15) == 0) find_sixteens(s);
    next_there = (unsigned)(held >> ((s & 15) * 4)) & 15u;
    const uint8_t* const keys = p.cache + __shfl(where, (s & 15) * 4 + (r >> 2), 64) + wave * 4 * D;
    const uint8_t* const values = p.cache + __shfl(where, (s & 15) * 4 + j, 64);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      if (c < G / 2) kc[c] = *reinterpret_cast<const uint4*>(keys + c * 256 + (j * 4 + (r & 3)) * 16);
      else __builtin_memcpy(&kc[c], __builtin_assume_aligned(keys + c * 256 + (j * 4 + (r & 3)) * 8, 8), 8);
    }
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int c = wave + i * kWaves;
      if (CT % kWaves == 0 || c < CT) vc[i] = *reinterpret_cast<const uint4*>(values + 16 * D + (16 * c + r) * 16);
    }
    factors = *reinterpret_cast<const float2*>(values + 32 * D);
  };
  if (steps > 0) issue(0);

  // ---- the columns of this lane
  h8 qf[kTiles][G];
  float rest[kTiles], ref[kTiles], limit[kTiles], sum[kTiles];   // scores are products times `rest` and the keys' factor
  int pos[kTiles];
  f4 o[kTiles][CT];
#pragma unroll
  for (int c = 0; c < kTiles; ++c) {
    const int col = t.first + (wave * kTiles + c) * kCols + r, in = min(col, t.cols - 1);
    const int tok = in / p.ratio, qh = in % p.ratio;
    pos[c] = col < t.cols ? row_position(p, t, tok) : -1;
    const V* qr = q + (size_t)(t.row + tok) * p.q_stride + ((size_t)head * p.ratio + qh) * p.q_head;
    float v[G][8], top = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      load_values<8, false>(qr + key_channel<G>(g, j), v[g]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[g][e]));
    }
    top = column_max(top);
    const unsigned e2 = min(max(__float_as_uint(top) >> 23, 1u), 253u);
    const float down = copysignf(__uint_as_float((254u - e2) << 23), p.scale_log2);
    rest[c] = fmaxf(fabsf(p.scale_log2) * __uint_as_float(e2 << 23), 1e-30f);    // (no 0 times infinity)
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[c][g][e] = (_Float16)(v[g][e] * down);
    ref[c] = 0.0f;
    limit[c] = -__builtin_inff();
    sum[c] = 0.0f;
#pragma unroll
    for (int i = 0; i < CT; ++i) o[c][i] = f4{0, 0, 0, 0};
  }
  // steps whose every key is seen by every column of the tile
  const int pos0 = row_position(p, t, t.first / p.ratio), pos1 = row_position(p, t, (min(t.first + kWideCols, t.cols) - 1) / p.ratio);
  const int clear0 = p.window > 0 ? pos1 - p.window : -1, clear1 = pos0;
  Power<4> scaled;

  for (int s = 0; s < steps; ++s) {
    const int key0 = start + s * kStep, base = key0 + 16 * j;
    const unsigned there = next_there;
    lds_barrier();                                    // the operands of the step before have been read
    // ---- a quarter of the keys: tile `wave`, whose row r is token 4 wave + r % 4 of sixteen r / 4; and of the values
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint4& w = kc[g / 2];
      *reinterpret_cast<h8*>(shared + ((wave * G + g) * 64 + lane) * 16) = g & 1 ? codes.eight(w.z, w.w) : codes.eight(w.x, w.y);
    }
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int c = wave + i * kWaves;
      if (CT % kWaves == 0 || c < CT) {
        char* const to = shared + W::OPERANDS + c * 2048 + lane * 16;
        *reinterpret_cast<h8*>(to) = codes.eight(vc[i].x, vc[i].y);
        *reinterpret_cast<h8*>(to + 1024) = codes.eight(vc[i].z, vc[i].w);
      }
    }
    const float fk = factors.x;
    float fv = factors.y;
    if (s + 1 < steps) issue(s + 1);
    lds_barrier();

    // ---- S^T, keys 16 j + 4 tile + i in register i of tile `tile`
    f4 x[kTiles][4];
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c) x[c][tile] = f4{0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const h8 k8 = *reinterpret_cast<const h8*>(shared + ((tile * G + g) * 64 + lane) * 16);
#pragma unroll
        for (int c = 0; c < kTiles; ++c) x[c][tile] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, qf[c][g], x[c][tile], 0, 0, 0);
      }
    }
#pragma unroll
    for (int c = 0; c < kTiles; ++c) {
      const float f = fk * rest[c];
#pragma unroll
      for (int tile = 0; tile < 4; ++tile)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[c][tile][i] = __builtin_fmaf(x[c][tile][i], f, -ref[c]);
    }
    const bool clear = key0 > clear0 && key0 + kStep - 1 <= clear1 && there == 15u;
    if (!clear) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c) {
        const int at = pos[c] + 1 - base;
        unsigned see = token_bits(p.window > 0 ? at - p.window : 0, there >> j & 1u ? at : 0);
        asm volatile("" : "+v"(see));                 // (a branch, not selects in every step)
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[c][tile][i] = see >> (4 * tile + i) & 1u ? x[c][tile][i] : -__builtin_inff();
      }
      // (a sixteen that no row sees: its factor may be anything)
      if (!(there >> j & 1u) || base + 15 < t.seen || base >= last) fv = 0.0f;
    }
    bool grown;
    const float down = scaled.grow(fv, &grown);
    if (grown) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c)
#pragma unroll
        for (int i = 0; i < CT; ++i) o[c][i] *= down;
    }
    const float weight = __builtin_amdgcn_ldexpf(fv, kLift - scaled.power);
    // ---- probabilities
    h8 pr[kTiles][2];
#pragma unroll
    for (int c = 0; c < kTiles; ++c) {
      float m = x[c][0][0];
#pragma unroll
      for (int tile = 0; tile < 4; ++tile)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, x[c][tile][i]);
      m = column_max(m);
      if (__any(m > limit[c])) {                      // (the first keys that a column sees: no limit yet)
        const bool begun = limit[c] > -__builtin_inff(), seen = m > -__builtin_inff();
        const float more = begun ? fmaxf(m, 0.0f) : seen ? m : 0.0f;
        const float shrink = begun ? __builtin_amdgcn_exp2f(-more) : 1.0f;
        ref[c] += more;
        if (seen) limit[c] = kSlack;
        sum[c] *= shrink;
#pragma unroll
        for (int i = 0; i < CT; ++i) o[c][i] *= shrink;
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[c][tile][i] -= more;
      }
#pragma unroll
      for (int tile = 0; tile < 4; ++tile)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(x[c][tile][i]);
          sum[c] += e;
          pr[c][tile >> 1][(tile & 1) * 4 + i] = (_Float16)(e * weight);
        }
    }
    // ---- O^T
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const h8 v8 = *reinterpret_cast<const h8*>(shared + W::OPERANDS + (i * 2 + h) * 1024 + lane * 16);
#pragma unroll
        for (int c = 0; c < kTiles; ++c) o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v8, pr[c][h], o[c][i], 0, 0, 0);
      }
  }
  const float back = two_to(scaled.power - kLift);
  bool seen[kTiles];
#pragma unroll
  for (int c = 0; c < kTiles; ++c) {
    seen[c] = limit[c] > -__builtin_inff();
#pragma unroll
    for (int i = 0; i < CT; ++i) o[c][i] *= back;
  }
  join_wide<D>(p, a, t, shared, out, o, ref, sum, seen);
#endif
}

// (what a cut tile needs of LDS: find_part's and join_wide's)
template <int G, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  constexpr size_t kJoin = (kWideParts + 1) * kWideCols * 4, kFind = 16 * 4 + 3 * kWaves * 4 + (3 * kMaxTiles + 1) * 4;
  constexpr size_t kLds = Wide<G>::LDS > kJoin ? (Wide<G>::LDS > kFind ? Wide<G>::LDS : kFind) : kJoin;
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
