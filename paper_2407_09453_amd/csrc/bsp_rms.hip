// Root-mean-square norm over the last axis with the residual stream's addition, forward and backward, bound by memory.
//
//   h = round(x + residual), q = 1 / sqrt(mean h^2 + eps), y = h q w
//   g = dy w, n = h q, dx = dh + q (g - n mean(g n)), dw = sum over rows of dy n
//
// The sum is rounded to its type before it is squared: the norm is that of what the residual stream holds, and the backward pass, which
// reads h, differentiates the very function that ran.  A row is read once and stays in the registers of the 16 to 1024 threads that
// own it; squares are summed in fp32 in a thread, in 64 bits over a row.  Rows too long for that are read again, and their sums are in 64 bits in a thread, too.  As in the layer norm the gradient's threads own columns and
// add dw over all the rows of their workgroup, and a second launch adds the workgroups' sums in a fixed order.
// Measured: 16384 x 4096 bf16 with a residual to codes 74 to 87 us (470 MB, 5.4 to 6.3 TB/s), its gradient 100 to 113 (537 MB, 4.8 to 5.4 TB/s) and 5 for
// the sums; 777 x 2966 fp32 8.2 and 9.8 (18 and 28 MB, from the last-level cache) and 4.2; one row of 4096 3.9.
#include "bsp_norm.h"

namespace {

struct RmsArgs {
  const void *X, *residual, *dY, *dH;
  const float* weight;
  void *H, *Y, *dX;
  uint8_t *codes, *scale;
  float *rstd, *part, *dweight;  // part: [parts][D]; with one part the sums themselves
  int64_t ldx, ldr, ldh, ldy, ld_dy, ld_dh, ld_dx, srows;
  int32_t T, D, Dp, e5, parts;
  float eps;
  double inv;  // 1 / D
};

// eight values of the residual stream: x + residual as its type holds it
template <bool F32>
__device__ __forceinline__ void add8(float* v, const float* r) {
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    v[k] += r[k];
    v[k + 1] += r[k + 1];
    if constexpr (!F32) {
      const uint32_t h = f8_pack_bf16x2(v[k], v[k + 1]);
      v[k] = __uint_as_float(h << 16);
      v[k + 1] = __uint_as_float(h & 0xFFFF0000u);
    }
  }
}

// The inverse root of a row's mean square, from its threads' sums (fp32, some sixteen terms each, or in 64 bits where a thread has any number of terms: 4096 equal
// ones in fp32, as in a row of 2^20, drift by 500 2^-24 of their sum), and what 32 bits leave of it.  The threads' sums
// meet in 64 bits and h q w is rounded once, for the sake of codes: where a block's largest value lies at the border between two scales the
// wrong side costs 128 codes a step (16384 x 4096 drawn 150 times, 79 million scales: 2 differ from the exact values', with a sum and three roundings in 32 bits
// 6; q is 4.7e-8 of it off at most, with these 1.5e-7).  The time is the same, one row takes 3.9 us instead of 3.7.
struct Root {
  float r, rest;
};
__device__ __forceinline__ double lane_double(double v, uint32_t lo, uint32_t hi) { return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }
template <int CTRL>
__device__ __forceinline__ double add_from_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return lane_double(v, f8_from_lane<CTRL>((uint32_t)u), f8_from_lane<CTRL>((uint32_t)(u >> 32)));
}
template <int ROWT>
__device__ __forceinline__ double row_sum_double(double v, double* sh) {
  v = add_from_lane<kMirror16>(add_from_lane<kMirror8>(add_from_lane<kXor2>(add_from_lane<kXor1>(v))));
  if constexpr (ROWT > 16) {
    const int lane = threadIdx.x & 63;
    uint64_t u = __builtin_bit_cast(uint64_t, v);
    const auto l16 = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false), h16 = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = lane_double(__builtin_bit_cast(double, (uint64_t)h16[0] << 32 | l16[0]), l16[1], h16[1]);
    u = __builtin_bit_cast(uint64_t, v);
    const auto l32 = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false), h32 = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = lane_double(__builtin_bit_cast(double, (uint64_t)h32[0] << 32 | l32[0]), l32[1], h32[1]);
    if constexpr (ROWT >= 256) {
      if (lane == 0) sh[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.;
#pragma unroll
      for (int w = 0; w < ROWT / 64; ++w) v += sh[w];
    }
  }
  return v;
}
template <int ROWT>
__device__ __forceinline__ Root inverse_root(const RmsArgs& a, double s, double* sh) {
  const double x = fma(row_sum_double<ROWT>(s, sh), a.inv, (double)a.eps);
  const float r = 1.f / sqrtf((float)x), more = (float)(0.5 * r * fma(-x * r, (double)r, 1.)), better = r + more;
  return fabsf(more) < 1e-6f * r ? Root{better, more - (better - r)} : Root{r, 0.f};  // (infinities, zeros, NaN)
}
__device__ __forceinline__ float scaled(float h, const Root& q, float w) {
  const float p = h * q.r, y = p * w, rest = fmaf(fmaf(h, q.rest, fmaf(h, q.r, -p)), w, fmaf(p, w, -y));
  return fabsf(y) < INFINITY ? y + rest : y;
}

// NV: groups of eight columns a thread holds; 0: rows of any length, read twice (three times with a residual's sum)
template <bool F32, bool CODES, int ROWT, int NV>
__global__ __launch_bounds__(ROWT > 256 ? ROWT : 256) void rms_forward(RmsArgs a) {
  __shared__ double sh[ROWT > 256 ? ROWT / 64 : 4];
  const int tid = threadIdx.x % ROWT;
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = ROWT >= 256 ? group : group * (256 / ROWT) + threadIdx.x / ROWT;
  if (row >= a.T) return;  // (whole groups of ROWT)
  const void *x = row_of<F32>(a.X, row, a.ldx), *r = row_of<F32>(a.residual, row, a.ldr);
  void* h = (void*)row_of<F32>(a.H, row, a.ldh);
  if constexpr (NV > 0) {  // (D >= 8)
    float s = 0.f;
    const bool ragged = a.D & 7;
    float v[NV][8];
    F8Raw8<F32> raw[NV], more[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = f8_raw8<F32>(x, (tid + j * ROWT) * 8, a.D);
    if (a.residual)
#pragma unroll
      for (int j = 0; j < NV; ++j) more[j] = f8_raw8<F32>(r, (tid + j * ROWT) * 8, a.D);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8, past = f8_past(c, a.D);
      f8_unpack8<F32>(raw[j], past, ragged, v[j]);
      if (a.residual) {
        float w[8];
        f8_unpack8<F32>(more[j], past, ragged, w);
        add8<F32>(v[j], w);
        if (c < a.D) f8_store8<F32>(h, c, a.D - c, v[j]);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[j][k] * v[j][k];  // (zeros past the row)
    }
    const Root root = inverse_root<ROWT>(a, s, sh);
    if (tid == 0) a.rstd[row] = root.r;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
      float w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = 1.f;
      if (a.weight) load8<true>(a.weight, c, a.D, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] = c + k < a.D ? scaled(v[j][k], root, w[k]) : 0.f;
      put8<F32, CODES>(a, row, c, v[j]);
    }
  } else {
    double s = 0.;
    float v[8];
    auto stream = [&](int c) {  // computed anew where it is needed again: H may have been written by other threads' stores
      load8<F32>(x, c, a.D, v);
      if (a.residual) {
        float w[8];
        load8<F32>(r, c, a.D, w);
        add8<F32>(v, w);
      }
    };
    for (int c = tid * 8; c < a.D; c += ROWT * 8) {
      stream(c);
#pragma unroll
      for (int k = 0; k < 8; ++k) s = fma((double)v[k], (double)v[k], s);
    }
    const Root root = inverse_root<ROWT>(a, s, sh);
    if (tid == 0) a.rstd[row] = root.r;
    for (int c = tid * 8; c < a.Dp; c += ROWT * 8) {
      const int left = a.D - c;
      stream(c);
      if (a.residual && left > 0) f8_store8<F32>(h, c, left, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < left ? scaled(v[k], root, a.weight ? a.weight[c + k] : 1.f) : 0.f;
      put8<F32, CODES>(a, row, c, v);
    }
  }
}

template <bool F32, int ROWT, int NV>
__global__ __launch_bounds__(ROWT > 256 ? ROWT : 256) void rms_backward(RmsArgs a) {
  __shared__ float sh[ROWT > 256 ? ROWT / 64 : 4][1];
  const int tid = threadIdx.x % ROWT;
  constexpr int kGroups = ROWT >= 256 ? 1 : 256 / ROWT;  // rows that a workgroup has in work
  const int in_group = threadIdx.x / ROWT;
  const int64_t group = (int64_t)blockIdx.x * kGroups + in_group, step = (int64_t)a.parts * kGroups;
  const float inv = 1.f / (float)a.D;
  const bool ragged = a.D & 7;
  // sixteen waves a workgroup leave each 128 registers: not enough for the weight, nor for a row that is asked for ahead
  constexpr bool kKeep = ROWT < 1024;
  constexpr int kWeights = kKeep ? NV : 1;
  float w[kWeights][8], dw[NV][8] = {};
  auto weights = [&](int j, float (&to)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) to[k] = 1.f;
    if (a.weight) load8<true>(a.weight, (tid + j * ROWT) * 8, a.D, to);
  };
  if constexpr (kKeep)
#pragma unroll
    for (int j = 0; j < NV; ++j) weights(j, w[j]);
  // a row's values are asked for while the row before it is worked on
  F8Raw8<F32> rh[NV], ry[NV], rd[NV];
  float next_rstd = 0.f;
  auto ask = [&](int64_t row) {
    row = row < a.T ? row : a.T - 1;
    next_rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      rh[j] = f8_raw8<F32>(row_of<F32>(a.H, row, a.ldh), (tid + j * ROWT) * 8, a.D);
      ry[j] = f8_raw8<F32>(row_of<F32>(a.dY, row, a.ld_dy), (tid + j * ROWT) * 8, a.D);
      if (a.dH) rd[j] = f8_raw8<F32>(row_of<F32>(a.dH, row, a.ld_dh), (tid + j * ROWT) * 8, a.D);
    }
  };
  if (kKeep && group < a.T) ask(group);
  for (int64_t row = group; row < a.T; row += step) {
    if constexpr (!kKeep) ask(row);
    const float rstd = next_rstd;
    float h[NV][8], g[NV][8], d[NV][8], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int past = f8_past((tid + j * ROWT) * 8, a.D);
      f8_unpack8<F32>(rh[j], past, ragged, h[j]);
      f8_unpack8<F32>(ry[j], past, ragged, g[j]);
      if (a.dH) f8_unpack8<F32>(rd[j], past, ragged, d[j]);
    }
    if constexpr (kKeep) ask(row + step);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (!kKeep) weights(j, w[0]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        h[j][k] *= rstd;
        dw[j][k] += g[j][k] * h[j][k];
        g[j][k] *= w[kKeep ? j : 0][k];
        s[0] += g[j][k] * h[j][k];
      }
    }
    row_sum<ROWT, 1>(s, sh);
    const float mean = s[0] * inv;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) g[j][k] = rstd * (g[j][k] - h[j][k] * mean);
      if (a.dH)
#pragma unroll
        for (int k = 0; k < 8; ++k) g[j][k] += d[j][k];
      if (c < a.D) f8_store8<F32>((void*)row_of<F32>(a.dX, row, a.ld_dx), c, a.D - c, g[j]);
    }
  }
  float* to_w = a.parts == 1 ? a.dweight : a.part + (int64_t)blockIdx.x * a.D;
  if (!to_w) return;
  if constexpr (kGroups == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
      if (c < a.D) f8_store8<true>(to_w, c, a.D - c, dw[j]);
    }
  } else {  // the groups' sums, in their order
    constexpr int kWide = ROWT * NV * 8;
    __shared__ float sums[kGroups][kWide];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) sums[in_group][(tid + j * ROWT) * 8 + k] = dw[j][k];
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += 256) {
      float v = 0.f;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) v += sums[g][c];
      to_w[c] = v;
    }
  }
}

// Rows of any length: dx, reading the row twice, and a second kernel for the columns' sums.
template <bool F32>
__global__ __launch_bounds__(256) void rms_backward_long(RmsArgs a) {
  __shared__ double sh[4];
  const int64_t row = (int64_t)blockIdx.y * kGridX + blockIdx.x;
  if (row >= a.T) return;
  const float rstd = a.rstd[row];
  double s = 0.;
  float h[8], g[8], d[8];
  auto load = [&](int c) {
    load8<F32>(row_of<F32>(a.H, row, a.ldh), c, a.D, h);
    load8<F32>(row_of<F32>(a.dY, row, a.ld_dy), c, a.D, g);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      h[k] *= rstd;
      g[k] *= a.weight && c + k < a.D ? a.weight[c + k] : 1.f;
    }
  };
  for (int c = threadIdx.x * 8; c < a.D; c += 2048) {
    load(c);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fma((double)g[k], (double)h[k], s);
  }
  const float mean = (float)(row_sum_double<256>(s, sh) * a.inv);
  for (int c = threadIdx.x * 8; c < a.D; c += 2048) {
    load(c);
    if (a.dH) load8<F32>(row_of<F32>(a.dH, row, a.ld_dh), c, a.D, d);
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] = rstd * (g[k] - h[k] * mean) + (a.dH ? d[k] : 0.f);
    f8_store8<F32>((void*)row_of<F32>(a.dX, row, a.ld_dx), c, a.D - c, g);
  }
}
template <bool F32>
__global__ __launch_bounds__(256) void rms_columns_long(RmsArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.D) return;
  float dw = 0.f;
  for (int64_t row = blockIdx.y; row < a.T; row += a.parts) {
    const float h = F32 ? ((const float*)a.H)[row * a.ldh + c] : bf16_bits_to_f32(((const uint16_t*)a.H)[row * a.ldh + c]);
    const float g = F32 ? ((const float*)a.dY)[row * a.ld_dy + c] : bf16_bits_to_f32(((const uint16_t*)a.dY)[row * a.ld_dy + c]);
    dw += g * (h * a.rstd[row]);
  }
  (a.parts == 1 ? a.dweight : a.part + (int64_t)blockIdx.y * a.D)[c] = dw;
}

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }

template <bool F32, bool CODES>
int forward(const RmsArgs& a, hipStream_t st) {
  const dim3 block(256), rows = f8_grid(a.T), quads = f8_grid(((int64_t)a.T + 3) / 4), sixteens = f8_grid(((int64_t)a.T + 15) / 16);
  if (a.D < 8 || a.Dp > 16384) hipLaunchKernelGGL((rms_forward<F32, CODES, 256, 0>), rows, block, 0, st, a);
  else if (a.Dp <= 128) hipLaunchKernelGGL((rms_forward<F32, CODES, 16, 1>), sixteens, block, 0, st, a);
  else if (a.Dp <= 256) hipLaunchKernelGGL((rms_forward<F32, CODES, 16, 2>), sixteens, block, 0, st, a);
  else if (a.Dp <= 512) hipLaunchKernelGGL((rms_forward<F32, CODES, 64, 1>), quads, block, 0, st, a);
  else if (a.Dp <= 1024) hipLaunchKernelGGL((rms_forward<F32, CODES, 64, 2>), quads, block, 0, st, a);
  else if (a.Dp <= 2048) hipLaunchKernelGGL((rms_forward<F32, CODES, 256, 1>), rows, block, 0, st, a);
  else if (a.Dp <= 4096) hipLaunchKernelGGL((rms_forward<F32, CODES, 256, 2>), rows, block, 0, st, a);
  else if (a.Dp <= 8192) hipLaunchKernelGGL((rms_forward<F32, CODES, 512, 2>), rows, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((rms_forward<F32, CODES, 1024, 2>), rows, dim3(1024), 0, st, a);
  return launched();
}

// rows that a workgroup of the backward pass has in work at one time
int rows_at_once(int D) { return D < 8 || D > 512 ? 1 : D <= 256 ? 16 : 4; }

template <bool F32>
int backward(const RmsArgs& a, hipStream_t st) {
  const dim3 block(256), parts((unsigned)a.parts);
  if (a.D >= 8 && a.D <= 128) hipLaunchKernelGGL((rms_backward<F32, 16, 1>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 256) hipLaunchKernelGGL((rms_backward<F32, 16, 2>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 512) hipLaunchKernelGGL((rms_backward<F32, 64, 1>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 2048) hipLaunchKernelGGL((rms_backward<F32, 256, 1>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 4096) hipLaunchKernelGGL((rms_backward<F32, 256, 2>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 8192) hipLaunchKernelGGL((rms_backward<F32, 512, 2>), parts, dim3(512), 0, st, a);
  else if (a.D >= 8 && a.D <= 16384) hipLaunchKernelGGL((rms_backward<F32, 1024, 2>), parts, dim3(1024), 0, st, a);
  else {
    if (a.T > 0) hipLaunchKernelGGL((rms_backward_long<F32>), f8_grid(a.T), block, 0, st, a);
    if (launched() != BSP_OK) return BSP_ERR_HIP;
    if (a.dweight) hipLaunchKernelGGL((rms_columns_long<F32>), dim3((unsigned)((a.D + 255) / 256), (unsigned)a.parts), block, 0, st, a);
  }
  return launched();
}

}  // namespace

// Workgroups that share the rows.  Where one is done with all of them in eight turns its sums are the result: a launch less.
int rms_parts(int T, int D) {
  const int64_t turns = ((int64_t)T + rows_at_once(D) - 1) / rows_at_once(D);
  const int most = D > 4096 ? 256 : 512;  // as many as the chip holds at one time (16384 x 4096: 768 and 1024 are slower)
  return turns <= 8 ? 1 : turns < most ? (int)turns : most;
}

int rms_launch_forward(const void* X, int64_t ldx, const void* residual, int64_t ldr, bool f32, int T, int D, const float* weight, float eps, void* H,
                       int64_t ldh, void* Y, int64_t ldy, int code, uint8_t* codes, uint8_t* scale, float* rstd, hipStream_t st) {
  RmsArgs a{};
  a.X = X, a.residual = residual, a.weight = weight, a.H = H, a.Y = Y, a.codes = codes, a.scale = scale, a.rstd = rstd;
  a.ldx = ldx, a.ldr = ldr, a.ldh = ldh, a.ldy = ldy, a.srows = f8_scale_rows(T), a.T = T, a.D = D, a.Dp = f8_blocks(D) * F8_BLOCK, a.e5 = code == BSP_E5M2, a.eps = eps, a.inv = 1. / D;
  if (codes) return f32 ? forward<true, true>(a, st) : forward<false, true>(a, st);
  return f32 ? forward<true, false>(a, st) : forward<false, false>(a, st);
}

int rms_launch_backward(const void* dY, int64_t ld_dy, const void* H, int64_t ldh, const void* dH, int64_t ld_dh, bool f32, const float* rstd,
                        const float* weight, int T, int D, void* dX, int64_t ld_dx, float* dweight, float* part, hipStream_t st) {
  RmsArgs a{};
  a.dY = dY, a.H = (void*)H, a.dH = dH, a.weight = weight, a.dX = dX, a.rstd = (float*)rstd, a.part = part, a.dweight = dweight;
  a.ld_dy = ld_dy, a.ldh = ldh, a.ld_dh = ld_dh, a.ld_dx = ld_dx, a.T = T, a.D = D, a.parts = rms_parts(T, D), a.inv = 1. / D;
  const int rc = f32 ? backward<true>(a, st) : backward<false>(a, st);
  if (rc != BSP_OK || a.parts == 1 || !dweight) return rc;
  return norm_launch_sum(part, a.parts, D, D, dweight, nullptr, st);
}
