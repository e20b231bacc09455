// Attention over the paged 4-bit cache where a request has many columns (prompts, in pieces or whole): the mathematics
// and the layouts of q8_kv4_attend.hip.
//
// A workgroup of four wavefronts owns 128 columns that share a key head, 32 of each wavefront's, and walks over the
// keys they see, 64 at a time.  The codes go from memory to LDS as they lie; the wavefronts unpack a quarter of them
// each, into operands of the matrix instruction in the order in which a wavefront reads them, and multiply all.
// Bound by vector instructions (unpacking 1.6 a code of a workgroup's keys, the softmax 4.5 a score) beside the matrix
// instructions, of which a third of the cycles is full, so three workgroups share a compute unit and two barriers a step
// are hidden behind each other's.
// bf16 outputs: a key is its code times its factor, and a query has the scale in it, both rounded to binary16 (2^-11 of
// each at most); scores come out of the products relative to the running maximum, which they begin with.  fp16 outputs show
// that: there codes of keys are multiplied, and factors and scale go into the sums.  For both a value is its code times its
// factor, and a probability what the exponential gives, rounded to binary16; the softmax's sum is that of the probabilities so
// rounded, as the values meet them.  A maximum that grows by less than 2^8 is left: probabilities are up to 256, and sums are
// not rescaled.  Outputs are off by, in parts of their norm: fp16 2.4 to 3.4e-4 (their own rounding alone: 2.1e-4); bf16
// 1.7e-3 for scores that spread by 1 or 2, 1.9e-3 by 8, 2.1e-3 by 16, 2.3 to 2.6e-3 by 32 (alone: 1.66e-3).
// Pieces of 2048 tokens of 3 requests over 8192 keys, 32 query heads of 128 channels: 395 us, 910 TFLOP/s; in a window of
// 1024 tokens 110 us; fp16 487 us.
#include "q8_kv4_attend.h"

namespace {

using namespace q8;

constexpr int kTiles = 2;                       // of 16 columns, of a wavefront
constexpr int kWide = kWideCols;                // columns of a workgroup
static_assert(kWide == kWaves * kTiles * kCols, "every wavefront has its own");
[[maybe_unused]] constexpr float kSlack = 8.0f; // powers of two that a maximum may grow by

template <int G>
struct Wide {
  static constexpr int SIXTEEN = 576 * G, CODES = 256 * G, RAW = 4 * SIXTEEN, OPERANDS = 4096 * G;
  static constexpr int K_AT = 2 * RAW, V_AT = K_AT + OPERANDS, POS_AT = V_AT + OPERANDS;
  static constexpr int LDS = POS_AT + kWide * 4;
};

template <int G, typename V>
__global__ __launch_bounds__(256, G <= 4 ? 3 : 1) void kv4_wide_kernel(const AttendParams p, const V* __restrict__ q,
                                                                       V* __restrict__ out) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr bool EXACT = std::is_same<V, _Float16>::value;
  constexpr int CT = 2 * G;
  using W = Wide<G>;
  extern __shared__ __attribute__((aligned(16))) char shared[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, j = lane >> 4;
  const Unpack un;
  Part a;
  Tile t;
  // (whole tiles: the last of a request see most keys, so they go first)
  const int id = p.parts ? (int)blockIdx.x : (p.tiles - 1 - (int)blockIdx.x / p.H) * p.H + (int)blockIdx.x % p.H;
  if (!find_part<kWide, kWideParts>(p, id, shared, &a, &t)) return;
  const int head = a.head, start = t.lo + a.step0 * kStep, steps = a.step1 - a.step0;
  const int last = min(t.lo + t.steps * kStep, t.len);

  // ---- loads: lane l holds where sixteen l % 4 of step l / 4 (of 16) lies, bit l of `held` whether it is there; wave w
  // fetches sixteen w
  const int* __restrict__ table = p.table + t.b * p.table_stride;
  long where = 0;
  unsigned long held = 0;
  auto find_sixteens = [&](int s0) {
    const int at = (start >> 4) + s0 * 4 + lane;
    int page = -1;
    if (at * 16 < last) page = table[at >> p.shift];
    const bool in = page >= 0 && page < p.n_pages;
    where = in ? ((((long)page * p.H + head) << p.shift) + (at & ((1 << p.shift) - 1))) * W::SIXTEEN : 0;
    held = __ballot(in);
  };
  find_sixteens(0);
  unsigned there[2] = {0, 0};
  auto issue = [&](int s) __attribute__((always_inline)) {
    if (s > 0 && (s & 15) == 0) find_sixteens(s);
    const int l = (s & 15) * 4 + wave;
    const unsigned mask = (unsigned)(held >> ((s & 15) * 4)) & 15u;
    there[0] = there[1], there[1] = mask;
    const unsigned lo = __builtin_amdgcn_readlane((int)where, l), hi = __builtin_amdgcn_readlane((int)(where >> 32), l);
    const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(p.cache + ((size_t)hi << 32 | lo)), 0, mask >> wave & 1u ? W::SIXTEEN : 0, 0x00020000);
    char* const to = shared + (s & 1) * W::RAW + wave * W::SIXTEEN;
#pragma unroll
    for (int i = 0; i < (W::SIXTEEN + 1023) / 1024; ++i)
      if (i * 1024 + 1024 <= W::SIXTEEN || lane * 16 < W::SIXTEEN - i * 1024)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + i * 1024), 16,
                                                 lane * 16 + i * 1024, 0, 0, 0);
  };

  // ---- the columns of this lane
  h8 qf[kTiles][G];
  float rest[kTiles], ref[kTiles], limit[kTiles], sum[kTiles];   // scores are products times `rest`
  int* const positions = reinterpret_cast<int*>(shared + W::POS_AT) + wave * kTiles * kCols + r;   // (registers are short)
  f4 o[kTiles][CT];
  if (steps > 0) issue(0);
#pragma unroll
  for (int c = 0; c < kTiles; ++c) {
    const int col = t.first + (wave * kTiles + c) * kCols + r, in = min(col, t.cols - 1);
    const int tok = in / p.ratio, qh = in % p.ratio;
    positions[c * kCols] = col < t.cols ? t.len - t.n + tok : -1;
    const V* qr = q + (size_t)(t.row + tok) * p.q_stride + ((size_t)head * p.ratio + qh) * p.q_head + 8 * j;
    float v[G][8], top = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      load_values<8, false>(qr + 32 * g, v[g]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[g][e]));
    }
    top = column_max(top);
    const unsigned e2 = min(max(__float_as_uint(top) >> 23, 1u), 253u);
    const float down = copysignf(__uint_as_float((254u - e2) << 23), p.scale_log2);
    rest[c] = fmaxf(fabsf(p.scale_log2) * __uint_as_float(e2 << 23), 1e-30f);    // (no 0 times infinity)
    float fold = 1.0f;
    if constexpr (!EXACT) {
      // into the queries, all of it or all but a power of two
      const float power = __uint_as_float(__float_as_uint(rest[c]) & 0x7f800000u);
      const float keep = power >= 0x1p-8f && power <= 0x1p8f ? 1.0f : power;
      fold = rest[c] / keep;
      rest[c] = keep;
    }
    constexpr int kKeyOrder[8] = {0, 4, 2, 6, 1, 5, 3, 7};
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[c][g][e] = (_Float16)(v[g][kKeyOrder[e]] * (down * fold));
    ref[c] = 0.0f;
    limit[c] = -__builtin_inff();
    sum[c] = 0.0f;
#pragma unroll
    for (int i = 0; i < CT; ++i) o[c][i] = f4{0, 0, 0, 0};
  }
  // steps whose every key is seen by every column of the tile
  const int pos0 = t.len - t.n + t.first / p.ratio, pos1 = t.len - t.n + (min(t.first + kWide, t.cols) - 1) / p.ratio;
  const int clear0 = p.window > 0 ? pos1 - p.window : -1, clear1 = pos0;
  constexpr _Float16 kBias = 1032.0f16, kSixteenth = 0.0625f16, kHighBias = -72.0f16;
  auto low = [&](unsigned w) { return un.low(w) - h2{kBias, kBias}; };
  auto high = [&](unsigned w) {
    return __builtin_elementwise_fma(un.high(w), h2{kSixteenth, kSixteenth}, h2{kHighBias, kHighBias});
  };

  bool folded = !EXACT;
#pragma unroll
  for (int c = 0; c < kTiles; ++c) folded &= !__any(rest[c] != 1.0f);
  for (int s = 0; s < steps; ++s) {
    const int key0 = start + s * kStep;
    wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xc07f);               // the operands of the step before have been read
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + 1 < steps) issue(s + 1);
    else there[0] = there[1];
    const char* const raw = shared + (s & 1) * W::RAW;
    // ---- a quarter of the keys: tile `wave`, whose row r is token 4 wave + r % 4 of sixteen r / 4
    {
      const int tk = 4 * wave + (r & 3);
      const char* const at = raw + (r >> 2) * W::SIXTEEN;
      unsigned kc[G];
      _Float16 kf[G];
      __builtin_memcpy(kc, __builtin_assume_aligned(at + tk * 16 * G + j * 4 * G, 4), 4 * G);
      __builtin_memcpy(kf, __builtin_assume_aligned(at + 512 * G + tk * 2 * G, 2), 2 * G);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const unsigned w8 = kc[g] >> 8;
        h2 a[4] = {low(kc[g]), low(w8), high(kc[g]), high(w8)};
        if constexpr (!EXACT) {
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] = a[e] * h2{kf[g], kf[g]};
        }
        *reinterpret_cast<h8*>(shared + W::K_AT + ((wave * G + g) * 64 + lane) * 16) = join4(a[0], a[1], a[2], a[3]);
      }
    }
    // ---- and of the values, a group's 32 of the keys each.  What lies outside the keys that the rows see may be no
    // number: its factors count as zeros.
    const bool edge = key0 < t.seen || key0 + kStep > last;
#pragma unroll
    for (int i0 = 0; i0 < 2 * G; i0 += kWaves) {
      const int i = i0 + wave, g = i >> 1, h = i & 1;
      if (2 * G % kWaves == 0 || i < 2 * G) {
        const char* const at = raw + j * W::SIXTEEN;
        unsigned vc[2];
        h2 vf[4];
        __builtin_memcpy(vc, __builtin_assume_aligned(at + W::CODES + (g * 16 + r) * 16 + 8 * h, 8), 8);
        __builtin_memcpy(vf, __builtin_assume_aligned(at + 544 * G + g * 32 + 16 * h, 16), 16);
        if (edge) {
          unsigned in = token_bits(t.seen - (key0 + 16 * j), last - (key0 + 16 * j)) >> 8 * h;
          asm volatile("" : "+v"(in));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t0 = 4 * (e >> 1) + (e & 1);
            const unsigned keep = (in >> t0 & 1u) * 0xffffu | (in >> (t0 + 2) & 1u) * 0xffff0000u;
            vf[e] = __builtin_bit_cast(h2, __builtin_bit_cast(unsigned, vf[e]) & keep);
          }
        }
        char* const to = shared + W::V_AT + (g * 4 + h) * 1024 + lane * 16;
        *reinterpret_cast<h8*>(to) = join4(low(vc[0]) * vf[0], low(vc[0] >> 8) * vf[1], low(vc[1]) * vf[2], low(vc[1] >> 8) * vf[3]);
        *reinterpret_cast<h8*>(to + 2048) =
            join4(high(vc[0]) * vf[0], high(vc[0] >> 8) * vf[1], high(vc[1]) * vf[2], high(vc[1] >> 8) * vf[3]);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    // (Wavefronts that multiply go before those that unpack: pieces of 2048 tokens 417 -> 395 us, a prompt of 4096 163 -> 170,
    // whose tiles are of all lengths.)
    __builtin_amdgcn_s_setprio(1);
    // ---- S^T, keys 16 j + 4 tile + i in register i of tile `tile`, relative to `ref`: the products begin with it
    f4 x[kTiles][4];
    float from[kTiles];
#pragma unroll
    for (int c = 0; c < kTiles; ++c) from[c] = folded ? -ref[c] : 0.0f;
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c) x[c][tile] = f4{from[c], from[c], from[c], from[c]};
      _Float16 kf[4][G];
      if constexpr (EXACT)
        __builtin_memcpy(kf, __builtin_assume_aligned(raw + j * W::SIXTEEN + 512 * G + tile * 8 * G, 8), 8 * G);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const h8 a = *reinterpret_cast<const h8*>(shared + W::K_AT + ((tile * G + g) * 64 + lane) * 16);
#pragma unroll
        for (int c = 0; c < kTiles; ++c) {
          if constexpr (EXACT) {
            const f4 y = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, qf[c][g], f4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[c][tile][i] = __builtin_fmaf(y[i], (float)kf[i][g], x[c][tile][i]);
          } else {
            x[c][tile] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, qf[c][g], x[c][tile], 0, 0, 0);
          }
        }
      }
    }
    if (EXACT || !folded) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c)
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[c][tile][i] = __builtin_fmaf(x[c][tile][i], rest[c], -ref[c]);
    }
    const bool clear = key0 > clear0 && key0 + kStep - 1 <= clear1 && there[0] == 15u;
    if (!clear) {
#pragma unroll
      for (int c = 0; c < kTiles; ++c) {
        const int pos = positions[c * kCols] + 1 - (key0 + 16 * j);
        unsigned see = token_bits(p.window > 0 ? pos - p.window : 0, there[0] >> j & 1u ? pos : 0);
        asm volatile("" : "+v"(see));                 // (a branch, not selects in every step)
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[c][tile][i] = see >> (4 * tile + i) & 1u ? x[c][tile][i] : -__builtin_inff();
      }
    }
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
      for (int tile = 0; tile < 4; ++tile) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[c][tile][i] = __builtin_amdgcn_exp2f(x[c][tile][i]);
        const h2 ones = {1.0f16, 1.0f16}, even = {(_Float16)x[c][tile][0], (_Float16)x[c][tile][2]};
        const h2 odd = {(_Float16)x[c][tile][1], (_Float16)x[c][tile][3]};
        sum[c] = __builtin_amdgcn_fdot2(even, ones, sum[c], false);             // of what the values are multiplied by
        sum[c] = __builtin_amdgcn_fdot2(odd, ones, sum[c], false);
        h8& to = pr[c][tile >> 1];
        to[4 * (tile & 1)] = even[0], to[4 * (tile & 1) + 1] = even[1];
        to[4 * (tile & 1) + 2] = odd[0], to[4 * (tile & 1) + 3] = odd[1];
      }
    }
    // ---- O^T
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const h8 a = *reinterpret_cast<const h8*>(shared + W::V_AT + (i * 2 + h) * 1024 + lane * 16);
#pragma unroll
        for (int c = 0; c < kTiles; ++c) o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, pr[c][h], o[c][i], 0, 0, 0);
      }
    __builtin_amdgcn_s_setprio(0);
  }
  constexpr int D = 32 * G;
  constexpr size_t kPartWords = (size_t)kWide * (D + 2) / 2;    // of a part: [tile][CT][2][lane], then maxima and sums
  word* const part = reinterpret_cast<word*>(p.parts) + ((size_t)(a.slot + a.part) * p.H + head) * kPartWords;
#pragma unroll
  for (int c = 0; c < kTiles; ++c) {
    sum[c] += __shfl_xor(sum[c], 16, 64);
    sum[c] += __shfl_xor(sum[c], 32, 64);
    const int of = (wave * kTiles + c) * kCols + r, col = t.first + of;
    if (col >= t.cols) continue;
    const float l = sum[c];
    if (a.parts == 1) {
      const float inv = l > 0.0f ? 1.0f / l : l;                // (no key: zeros; no number: none)
      V* const to = out + (size_t)(t.row + col / p.ratio) * p.o_stride + ((size_t)head * p.ratio + col % p.ratio) * p.o_head + 4 * j;
#pragma unroll
      for (int i = 0; i < CT; ++i) {
        const float y[4] = {o[c][i][0] * inv, o[c][i][1] * inv, o[c][i][2] * inv, o[c][i][3] * inv};
        store_values<4, false>(to + 16 * i, y);
      }
    } else {
      word* const to = part + (wave * kTiles + c) * CT * 128 + lane;
#pragma unroll
      for (int i = 0; i < CT; ++i) {
        put(to + 128 * i, o[c][i][0], o[c][i][1]);
        put(to + 128 * i + 64, o[c][i][2], o[c][i][3]);
      }
      if (j == 0) put(part + kWide * D / 2 + of, limit[c] > -__builtin_inff() ? ref[c] : -__builtin_inff(), l);
    }
  }
  if (a.parts == 1) return;

  // ---- the parts of the tile and head: the workgroup that finishes last adds them, whichever it is in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's words have arrived
  __syncthreads();                                      // and the others'; LDS is free
  int* const flag = reinterpret_cast<int*>(shared);
  int* const counter = p.counters + a.rank * p.H + head;
  if (tid == 0) flag[0] = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  __syncthreads();
  if (flag[0] != a.parts - 1) return;
  __syncthreads();
  if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  const word* const parts = reinterpret_cast<const word*>(p.parts) + ((size_t)a.slot * p.H + head) * kPartWords;
  const size_t stride = (size_t)p.H * kPartWords;
  float* const weights = reinterpret_cast<float*>(shared);      // [16][128], then the columns' sums
  float* const totals = weights + kWideParts * kWide;
  if (tid < kWide) {
    f2 rs[kWideParts];
    float most = -__builtin_inff(), l = 0.0f;
#pragma unroll
    for (int u = 0; u < kWideParts; ++u) {
      rs[u] = f2{-__builtin_inff(), 0.0f};
      if (u < a.parts && t.first + tid < t.cols) rs[u] = get(parts + u * stride + kWide * D / 2 + tid);
    }
#pragma unroll
    for (int u = 0; u < kWideParts; ++u) most = fmaxf(most, rs[u][0]);
#pragma unroll
    for (int u = 0; u < kWideParts; ++u) {
      const float weight = rs[u][0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(rs[u][0] - most);
      weights[u * kWide + tid] = weight;
      l += weight * rs[u][1];
    }
    totals[tid] = l;
  }
  __syncthreads();
  // a thread takes four channels of a column, as a lane had them, and several such, so that enough is on its way
  const int valid = t.cols - t.first, groups = min((valid + kCols - 1) / kCols, kWide / kCols) * CT;     // of 64 lanes' quads
  constexpr int kItems = 4, kBatch = 4;
  for (int g0 = wave; g0 < groups; g0 += kWaves * kItems) {
    f4 v[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) v[k] = f4{0, 0, 0, 0};
    for (int s0 = 0; s0 < a.parts; s0 += kBatch) {
      f2 x[kItems][kBatch][2];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
          const word* const from = parts + min(s0 + u, a.parts - 1) * stride + min(g0 + k * kWaves, groups - 1) * 128 + lane;
          x[k][u][0] = get(from), x[k][u][1] = get(from + 64);
        }
#pragma unroll
      for (int k = 0; k < kItems; ++k)
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (s0 + u < a.parts)
            v[k] += weights[(s0 + u) * kWide + min(g0 + k * kWaves, groups - 1) / CT * kCols + r] *
                    f4{x[k][u][0][0], x[k][u][0][1], x[k][u][1][0], x[k][u][1][1]};
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int g = g0 + k * kWaves, of = g / CT * kCols + r, col = t.first + of;
      if (g >= groups || col >= t.cols) continue;
      const float l = totals[of], inv = l > 0.0f ? 1.0f / l : l;
      const float y[4] = {v[k][0] * inv, v[k][1] * inv, v[k][2] * inv, v[k][3] * inv};
      store_values<4, false>(out + (size_t)(t.row + col / p.ratio) * p.o_stride + ((size_t)head * p.ratio + col % p.ratio) * p.o_head +
                                 g % CT * 16 + 4 * j, y);
    }
  }
#endif
}

template <int G, typename V>
int launch(const AttendParams& p, const V* q, V* out, hipStream_t stream) {
  if constexpr (Wide<G>::LDS > 65536) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_wide_kernel<G, V>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, Wide<G>::LDS);
    if (attr != hipSuccess) return Q8_EHIP;
  }
  kv4_wide_kernel<G, V><<<(unsigned)(p.tiles * p.H) + (p.parts ? kTarget : 0), 256, Wide<G>::LDS, stream>>>(p, q, out);
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

int kv4_attend_wide(int G, const AttendParams& p, const void* q, void* out, int type, hipStream_t stream) {
  if (type == Q8_F16)
    return launch_any(G, p, static_cast<const _Float16*>(q), static_cast<_Float16*>(out), stream);
  return launch_any(G, p, static_cast<const __bf16*>(q), static_cast<__bf16*>(out), stream);
}

}  // namespace q8
