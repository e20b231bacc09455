// Shared by the builds of the 8-bit linear layer's product (q8_linear.hip, q8_linear_tile.hip): its parameters, the
// packed weights' blocks and the tail.
#pragma once
#include "q8_conv_common.h"
#include "q8_rows.h"
#include <type_traits>
#pragma clang fp contract(off)

namespace q8 {

constexpr int kPackK = 64;                    // reduction bytes of a packed block
constexpr int kPackN = 16;                    // and its rows

struct LinearParams {
  const int8_t* __restrict__ z;
  const float* __restrict__ q_x;
  const int8_t* __restrict__ w;
  const float* __restrict__ q_w;
  const float* __restrict__ bias;
  size_t z_stride, y_stride;
  int M, N, K, ksteps;
};

// N consecutive outputs of row m < M, channels n ..: the tail, and whole vectors where the row allows it (VEC: rows
// of y begin at a multiple of N values' bytes, or of 16).
template <int C, bool VEC, typename Y>
__device__ __forceinline__ void finish_outputs(const LinearParams& p, Y* __restrict__ y, int m, int n, float q,
                                               const int (&acc)[C]) {
  float v[C];
  Y* const to = y + (size_t)m * p.y_stride + n;
  if (n + C <= p.N) {
#pragma unroll
    for (int e = 0; e < C; ++e) {
      v[e] = (float)acc[e] * (q * p.q_w[n + e]);
      if (p.bias) v[e] = v[e] + p.bias[n + e];
    }
    store_values<C, VEC>(to, v);
  } else {
#pragma unroll
    for (int e = 0; e < C; ++e)
      if (n + e < p.N) {
        float t = (float)acc[e] * (q * p.q_w[n + e]);
        if (p.bias) t = t + p.bias[n + e];
        to[e] = (Y)t;
      }
  }
}

// The tile builds (q8_linear_tile.hip): whether one takes these sizes, and its launch.
int linear_tile(const LinearParams& p, void* y, int type, int variant, hipStream_t stream);

// The build for few rows (q8_linear_rows.hip), on codes, and on real values where it takes that many.
int linear_rows(const LinearParams& p, void* y, int type, int columns, int squares, hipStream_t stream);
bool linear_rows_take_real(int M, int N, int K);
int linear_rows_real(const LinearParams& p, const void* x, int x_type, size_t x_stride, void* y, int type,
                     hipStream_t stream);

}  // namespace q8
