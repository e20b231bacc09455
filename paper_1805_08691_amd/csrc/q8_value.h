// The value types of the operators on rows of real values and on the 4-bit cache (Q8_F32, Q8_F16, Q8_BF16): loads
// and stores of runs of them as fp32, in 16-byte accesses where the addresses allow it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "q8_common.h"

namespace q8 {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// Calls f with a value of the C++ type of a Q8_* type code.
template <typename F>
inline int with_type(int type, F f) {
  switch (type) {
    case Q8_F32: return f(float{});
    case Q8_F16: return f(_Float16{});
    case Q8_BF16: return f(__bf16{});
  }
  return Q8_EINVAL;
}
inline size_t type_bytes(int type) { return type == Q8_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == Q8_F32 || type == Q8_F16 || type == Q8_BF16; }

// Blocks of so many threads that one launch takes in a dimension, whose threads are counted in 32 bits.
constexpr size_t most_blocks(size_t threads) { return 0xffffffffu / threads; }

// N consecutive values at p.  ALIGNED: p is 16-byte aligned, or a multiple of the N values' bytes where these are fewer
// (told to the compiler; the accesses are as wide without it, and take longer where they cross a line).
template <int N, bool ALIGNED, typename V>
__device__ __forceinline__ void load_values(const V* p, float (&v)[N]) {
  constexpr size_t A = ALIGNED ? (N * sizeof(V) % 16 == 0 ? 16 : N * sizeof(V)) : sizeof(V);
  V raw[N];
  __builtin_memcpy(raw, __builtin_assume_aligned(p, A), sizeof(raw));
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = (float)raw[e];
}
template <int N, bool ALIGNED, typename V>
__device__ __forceinline__ void store_values(V* p, const float (&v)[N]) {
  constexpr size_t A = ALIGNED ? (N * sizeof(V) % 16 == 0 ? 16 : N * sizeof(V)) : sizeof(V);
  V raw[N];
#pragma unroll
  for (int e = 0; e < N; ++e) raw[e] = (V)v[e];
  __builtin_memcpy(__builtin_assume_aligned(p, A), raw, sizeof(raw));
}

// A barrier that waits for LDS only: loads and stores of memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Sums over the lanes up to this one (16 at a time, then over the rows of 16).
__device__ __forceinline__ unsigned scan64(unsigned v) {
  v += __builtin_amdgcn_update_dpp(0u, v, 0x111, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0u, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0u, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0u, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0u, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0u, v, 0x143, 0xc, 0xf, false);
  return v;
}

// |v| where v is finite, else 0: what enters the maximum behind a factor.
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.0f;
}

}  // namespace q8
