// What the norms' kernels share: rows of any length and alignment, eight values a thread at a time, and sums over a row's threads.
#ifndef BSP_NORM_H
#define BSP_NORM_H

#include "bsp_f8.h"

template <bool F32>
__device__ __forceinline__ const void* row_of(const void* X, int64_t row, int64_t ld) {
  return F32 ? (const void*)((const float*)X + row * ld) : (const void*)((const uint16_t*)X + row * ld);
}
// eight values of a row of any length, one by one
template <bool F32>
__device__ __forceinline__ void each8(const void* row, int c, int n, float* v) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = 0.f;
    if (c + k < n) v[k] = F32 ? ((const float*)row)[c + k] : bf16_bits_to_f32(((const uint16_t*)row)[c + k]);
  }
}
template <bool F32>
__device__ __forceinline__ void load8(const void* row, int c, int n, float* v) {
  if (n >= 8) f8_unpack8<F32>(f8_raw8<F32>(row, c, n), f8_past(c, n), (n & 7) != 0, v);
  else each8<F32>(row, c, n, v);
}

// sums of N values over the threads of a row (16 lanes, a wave, the workgroup)
template <int ROWT, int N>
__device__ __forceinline__ void row_sum(float* v, float (*sh)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = ROWT == 16 ? f8_row16_sum(v[k]) : f8_wave_sum(v[k]);
  if constexpr (ROWT >= 256) {
    __syncthreads();  // the last use of sh is over
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) sh[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = 0.f;
#pragma unroll
      for (int w = 0; w < ROWT / 64; ++w) v[k] += sh[w][k];
    }
  }
}

// eight results of a row: in X's type, or as codes
// (Args: Y, ldy, D; codes, scale, Dp, srows, e5)
template <bool F32, bool CODES, class Args>
__device__ __forceinline__ void put8(const Args& a, int64_t row, int c, float* y) {
  if constexpr (CODES) {
    if (c >= a.Dp) return;  // (whole groups of sixteen lanes: Dp is a multiple of 128)
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, f8_magnitude(y[k]));
    m = f8_most<16>(m);
    const int b = a.e5 ? f8_scale_byte<true>(m) : f8_scale_byte<false>(m);
    const float s = f8_inverse(b);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] *= s;
    u32x2_t q;
    if (a.e5) q = u32x2_t{f8_encode4<true>(y[0], y[1], y[2], y[3]), f8_encode4<true>(y[4], y[5], y[6], y[7])};
    else q = u32x2_t{f8_encode4<false>(y[0], y[1], y[2], y[3]), f8_encode4<false>(y[4], y[5], y[6], y[7])};
    *(u32x2_t*)(a.codes + row * a.Dp + c) = q;
    if ((threadIdx.x & 15) == 0) a.scale[(int64_t)(c >> 7) * a.srows + row] = (uint8_t)b;
  } else if (c < a.D) {
    f8_store8<F32>((void*)row_of<F32>(a.Y, row, a.ldy), c, a.D - c, y);
  }
}

#endif
