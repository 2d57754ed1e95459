// Layer norm over the last axis, forward and backward, bound by memory.
//
//   mu = mean x, v = mean (x - mu)^2, r = 1 / sqrt(v + eps), h = (x - mu) r, y = h w + b
//   g = dy w, dx = r (g - mean g - h mean(g h)), dw = sum over rows of dy h, db = sum over rows of dy
//
// A row is read once and stays in the registers of the 16 to 1024 threads that own it, so the mean is known before the
// deviations are squared (no difference of large sums); everything is summed in fp32.  Rows too long for that are read again.
// The gradient's threads own columns: each adds its columns' dw and db over all the rows that its workgroup takes, and
// a second launch adds the workgroups' sums in a fixed order (no atomics: the same inputs give the same bits).
// The forward pass can leave its result as 8-bit codes, from the fp32 values: sixteen neighbouring lanes hold a block of 128.
// Measured: 16384 x 4096 bf16 forward 45 us (6.0 TB/s, where a copy runs at 6.2), backward 64 (6.3) and 4.6 for the sums; 2019 x 8000 bf16 12.6,
// 16.2 and 4.0; 1021 x 1000 fp32 4.7, 6.6 and 4.0; 2000 x 16001 24, 40 (6 of 128 registers in memory) and 8; 2000 x 17001, read again for each
// pass, 44 forward, 47 for dx, 32 and 9 for the sums.  A wave a row instead of four: 97 us forward
// at 16384 x 4096 against 60 at that time, since a CU then has a quarter of the requests under way.
#include "bsp_f8.h"

namespace {

struct NormArgs {
  const void *X, *dY;
  const float *weight, *bias;
  void *Y, *dX;
  uint8_t *codes, *scale;
  float *mean, *rstd, *part, *dweight, *dbias;  // part: [parts][2][D]; with one part the sums themselves
  int64_t ldx, ldy, ld_dy, ld_dx, srows;
  int32_t T, D, Dp, e5, parts;
  float eps;
};

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
template <bool F32, bool CODES>
__device__ __forceinline__ void put8(const NormArgs& a, int64_t row, int c, float* y) {
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

// NV: groups of eight columns a thread holds; 0: rows of any length, read three times
template <bool F32, bool CODES, int ROWT, int NV>
__global__ __launch_bounds__(ROWT > 256 ? ROWT : 256) void norm_forward(NormArgs a) {
  __shared__ float sh[ROWT > 256 ? ROWT / 64 : 4][1];
  const int tid = threadIdx.x % ROWT;
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = ROWT >= 256 ? group : group * (256 / ROWT) + threadIdx.x / ROWT;
  if (row >= a.T) return;  // (whole groups of ROWT)
  const void* x = row_of<F32>(a.X, row, a.ldx);
  const float inv = 1.f / (float)a.D;
  const bool ragged = a.D & 7;
  if constexpr (NV > 0) {  // (D >= 8)
    float v[NV][8];
    float s[1] = {0.f};
    F8Raw8<F32> raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = f8_raw8<F32>(x, (tid + j * ROWT) * 8, a.D);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      f8_unpack8<F32>(raw[j], f8_past((tid + j * ROWT) * 8, a.D), ragged, v[j]);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[0] += v[j][k];
    }
    row_sum<ROWT, 1>(s, sh);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[j][k] = (tid + j * ROWT) * 8 + k < a.D ? v[j][k] - mean : 0.f;
        s[0] += v[j][k] * v[j][k];
      }
    row_sum<ROWT, 1>(s, sh);
    const float rstd = 1.f / sqrtf(s[0] * inv + a.eps);
    if (tid == 0) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
      float w[8], b[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = 1.f, b[k] = 0.f;
      if (a.weight) load8<true>(a.weight, c, a.D, w);
      if (a.bias) load8<true>(a.bias, c, a.D, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] = c + k < a.D ? v[j][k] * rstd * w[k] + b[k] : 0.f;
      put8<F32, CODES>(a, row, c, v[j]);
    }
  } else {
    float s[1] = {0.f}, v[8];
    for (int c = tid * 8; c < a.D; c += ROWT * 8) {
      load8<F32>(x, c, a.D, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[0] += v[k];
    }
    row_sum<ROWT, 1>(s, sh);
    const float mean = s[0] * inv;
    s[0] = 0.f;
    for (int c = tid * 8; c < a.D; c += ROWT * 8) {
      load8<F32>(x, c, a.D, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[0] += c + k < a.D ? (v[k] - mean) * (v[k] - mean) : 0.f;
    }
    row_sum<ROWT, 1>(s, sh);
    const float rstd = 1.f / sqrtf(s[0] * inv + a.eps);
    if (tid == 0) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
    for (int c = tid * 8; c < a.Dp; c += ROWT * 8) {
      const int left = a.D - c;
      load8<F32>(x, c, a.D, v);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = k < left ? (v[k] - mean) * rstd * (a.weight ? a.weight[c + k] : 1.f) + (a.bias ? a.bias[c + k] : 0.f) : 0.f;
      put8<F32, CODES>(a, row, c, v);
    }
  }
}

template <bool F32, int ROWT, int NV>
__global__ __launch_bounds__(ROWT > 256 ? ROWT : 256) void norm_backward(NormArgs a) {
  __shared__ float sh[ROWT > 256 ? ROWT / 64 : 4][2];
  const int tid = threadIdx.x % ROWT;
  constexpr int kGroups = ROWT >= 256 ? 1 : 256 / ROWT;  // rows that a workgroup has in work
  const int in_group = threadIdx.x / ROWT;
  const int64_t group = (int64_t)blockIdx.x * kGroups + in_group, step = (int64_t)a.parts * kGroups;
  const float inv = 1.f / (float)a.D;
  const bool ragged = a.D & 7;
  // sixteen waves a workgroup leave each 128 registers: not enough for the weight, nor for a row that is asked for ahead
  constexpr bool kKeep = ROWT < 1024;
  constexpr int kWeights = kKeep ? NV : 1;
  float w[kWeights][8], dw[NV][8] = {}, db[NV][8] = {};
  auto weights = [&](int j, float (&to)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) to[k] = 1.f;
    if (a.weight) load8<true>(a.weight, (tid + j * ROWT) * 8, a.D, to);
  };
  if constexpr (kKeep)
#pragma unroll
    for (int j = 0; j < NV; ++j) weights(j, w[j]);
  // a row's values are asked for while the row before it is worked on
  F8Raw8<F32> rx[NV], ry[NV];
  float next_mean = 0.f, next_rstd = 0.f;
  auto ask = [&](int64_t row) {
    row = row < a.T ? row : a.T - 1;
    next_mean = a.mean[row], next_rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      rx[j] = f8_raw8<F32>(row_of<F32>(a.X, row, a.ldx), (tid + j * ROWT) * 8, a.D);
      ry[j] = f8_raw8<F32>(row_of<F32>(a.dY, row, a.ld_dy), (tid + j * ROWT) * 8, a.D);
    }
  };
  if (kKeep && group < a.T) ask(group);
  for (int64_t row = group; row < a.T; row += step) {
    if constexpr (!kKeep) ask(row);
    const float mean = next_mean, rstd = next_rstd;
    float h[NV][8], g[NV][8], s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int past = f8_past((tid + j * ROWT) * 8, a.D);
      f8_unpack8<F32>(rx[j], past, ragged, h[j]);
      f8_unpack8<F32>(ry[j], past, ragged, g[j]);
    }
    if constexpr (kKeep) ask(row + step);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (!kKeep) weights(j, w[0]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        h[j][k] = (tid + j * ROWT) * 8 + k < a.D ? (h[j][k] - mean) * rstd : 0.f;
        dw[j][k] += g[j][k] * h[j][k];
        db[j][k] += g[j][k];
        g[j][k] *= w[kKeep ? j : 0][k];
        s[0] += g[j][k];
        s[1] += g[j][k] * h[j][k];
      }
    }
    row_sum<ROWT, 2>(s, sh);
    const float mg = s[0] * inv, mh = s[1] * inv;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) g[j][k] = rstd * (g[j][k] - mg - h[j][k] * mh);
      if (c < a.D) f8_store8<F32>((void*)row_of<F32>(a.dX, row, a.ld_dx), c, a.D - c, g[j]);
    }
  }
  float *to_w = a.parts == 1 ? a.dweight : a.part + (int64_t)blockIdx.x * 2 * a.D, *to_b = a.parts == 1 ? a.dbias : a.part + ((int64_t)blockIdx.x * 2 + 1) * a.D;
  if constexpr (kGroups == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
      if (c >= a.D) continue;
      if (to_w) f8_store8<true>(to_w, c, a.D - c, dw[j]);
      if (to_b) f8_store8<true>(to_b, c, a.D - c, db[j]);
    }
  } else {  // the groups' sums, in their order
    constexpr int kWide = ROWT * NV * 8;
    __shared__ float sums[2][kGroups][kWide];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sums[0][in_group][(tid + j * ROWT) * 8 + k] = dw[j][k];
        sums[1][in_group][(tid + j * ROWT) * 8 + k] = db[j][k];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += 256) {
      float w = 0.f, b = 0.f;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) w += sums[0][g][c], b += sums[1][g][c];
      if (to_w) to_w[c] = w;
      if (to_b) to_b[c] = b;
    }
  }
}

// Rows of any length: dx, reading the row twice, and a second kernel for the columns' sums.
template <bool F32>
__global__ __launch_bounds__(256) void norm_backward_long(NormArgs a) {
  __shared__ float sh[4][2];
  const int64_t row = (int64_t)blockIdx.y * kGridX + blockIdx.x;
  if (row >= a.T) return;
  const float inv = 1.f / (float)a.D, mean = a.mean[row], rstd = a.rstd[row];
  float s[2] = {0.f, 0.f}, h[8], g[8];
  for (int c = threadIdx.x * 8; c < a.D; c += 2048) {
    load8<F32>(row_of<F32>(a.X, row, a.ldx), c, a.D, h);
    load8<F32>(row_of<F32>(a.dY, row, a.ld_dy), c, a.D, g);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c + k < a.D) {
        const float p = g[k] * (a.weight ? a.weight[c + k] : 1.f);
        s[0] += p;
        s[1] += p * (h[k] - mean) * rstd;
      }
  }
  row_sum<256, 2>(s, sh);
  const float mg = s[0] * inv, mh = s[1] * inv;
  for (int c = threadIdx.x * 8; c < a.D; c += 2048) {
    load8<F32>(row_of<F32>(a.X, row, a.ldx), c, a.D, h);
    load8<F32>(row_of<F32>(a.dY, row, a.ld_dy), c, a.D, g);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      g[k] = c + k < a.D ? rstd * (g[k] * (a.weight ? a.weight[c + k] : 1.f) - mg - (h[k] - mean) * rstd * mh) : 0.f;
    f8_store8<F32>((void*)row_of<F32>(a.dX, row, a.ld_dx), c, a.D - c, g);
  }
}
template <bool F32>
__global__ __launch_bounds__(256) void norm_columns_long(NormArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.D) return;
  float dw = 0.f, db = 0.f;
  for (int64_t row = blockIdx.y; row < a.T; row += a.parts) {
    const float x = F32 ? ((const float*)a.X)[row * a.ldx + c] : bf16_bits_to_f32(((const uint16_t*)a.X)[row * a.ldx + c]);
    const float g = F32 ? ((const float*)a.dY)[row * a.ld_dy + c] : bf16_bits_to_f32(((const uint16_t*)a.dY)[row * a.ld_dy + c]);
    dw += g * (x - a.mean[row]) * a.rstd[row];
    db += g;
  }
  float *to_w = a.parts == 1 ? a.dweight : a.part + (int64_t)blockIdx.y * 2 * a.D, *to_b = a.parts == 1 ? a.dbias : a.part + ((int64_t)blockIdx.y * 2 + 1) * a.D;
  if (to_w) to_w[c] = dw;
  if (to_b) to_b[c] = db;
}

// out[c] = sum of part[p][c] over p: 64 columns a workgroup, sixteen threads a column whose sums are added in their order
__global__ __launch_bounds__(1024) void norm_sum(const float* part, int parts, int64_t width, int64_t split_at, float* out, float* out2) {
  __shared__ float sh[16][64];
  const int l = threadIdx.x & 63, q = threadIdx.x >> 6;
  const int64_t c = ((int64_t)blockIdx.y * kGridX + blockIdx.x) * 64 + l;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int p = q; p < parts; p += 16) s += part[p * width + c];
  }
  sh[q][l] = s;
  __syncthreads();
  if (q == 0 && c < width) {
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += sh[k][l];
    float* to = c < split_at ? out : out2;
    if (to) to[c < split_at ? c : c - split_at] = s;
  }
}

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }

template <bool F32, bool CODES>
int forward(const NormArgs& a, hipStream_t st) {
  const dim3 block(256), rows = f8_grid(a.T), quads = f8_grid(((int64_t)a.T + 3) / 4), sixteens = f8_grid(((int64_t)a.T + 15) / 16);
  if (a.D < 8 || a.Dp > 16384) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 0>), rows, block, 0, st, a);
  else if (a.Dp <= 128) hipLaunchKernelGGL((norm_forward<F32, CODES, 16, 1>), sixteens, block, 0, st, a);
  else if (a.Dp <= 256) hipLaunchKernelGGL((norm_forward<F32, CODES, 16, 2>), sixteens, block, 0, st, a);
  else if (a.Dp <= 512) hipLaunchKernelGGL((norm_forward<F32, CODES, 64, 1>), quads, block, 0, st, a);
  else if (a.Dp <= 1024) hipLaunchKernelGGL((norm_forward<F32, CODES, 64, 2>), quads, block, 0, st, a);
  else if (a.Dp <= 2048) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 1>), rows, block, 0, st, a);
  else if (a.Dp <= 4096) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 2>), rows, block, 0, st, a);
  else if (a.Dp <= 8192) hipLaunchKernelGGL((norm_forward<F32, CODES, 512, 2>), rows, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((norm_forward<F32, CODES, 1024, 2>), rows, dim3(1024), 0, st, a);
  return launched();
}

// rows that a workgroup of the backward pass has in work at one time
int rows_at_once(int D) { return D < 8 || D > 512 ? 1 : D <= 256 ? 16 : 4; }

template <bool F32>
int backward(const NormArgs& a, hipStream_t st) {
  const dim3 block(256), parts((unsigned)a.parts);
  if (a.D >= 8 && a.D <= 128) hipLaunchKernelGGL((norm_backward<F32, 16, 1>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 256) hipLaunchKernelGGL((norm_backward<F32, 16, 2>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 512) hipLaunchKernelGGL((norm_backward<F32, 64, 1>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 2048) hipLaunchKernelGGL((norm_backward<F32, 256, 1>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 4096) hipLaunchKernelGGL((norm_backward<F32, 256, 2>), parts, block, 0, st, a);
  else if (a.D >= 8 && a.D <= 8192) hipLaunchKernelGGL((norm_backward<F32, 512, 2>), parts, dim3(512), 0, st, a);
  else if (a.D >= 8 && a.D <= 16384) hipLaunchKernelGGL((norm_backward<F32, 1024, 2>), parts, dim3(1024), 0, st, a);
  else {
    if (a.T > 0) hipLaunchKernelGGL((norm_backward_long<F32>), f8_grid(a.T), block, 0, st, a);
    if (launched() != BSP_OK) return BSP_ERR_HIP;
    hipLaunchKernelGGL((norm_columns_long<F32>), dim3((unsigned)((a.D + 255) / 256), (unsigned)a.parts), block, 0, st, a);
  }
  return launched();
}

int sum(const float* part, int parts, int64_t width, int64_t split_at, float* out, float* out2, hipStream_t st) {
  hipLaunchKernelGGL(norm_sum, f8_grid((width + 63) / 64), dim3(1024), 0, st, part, parts, width, split_at, out, out2);
  return launched();
}

}  // namespace

// Workgroups that share the rows.  Where one is done with all of them in eight turns its sums are the result: a launch less.
int norm_parts(int T, int D) {
  const int64_t turns = ((int64_t)T + rows_at_once(D) - 1) / rows_at_once(D);
  const int most = D > 4096 ? 256 : 512;  // as many as the chip holds at one time
  return turns <= 8 ? 1 : turns < most ? (int)turns : most;
}

int norm_launch_forward(const void* X, bool f32, int64_t ldx, int T, int D, const float* weight, const float* bias, float eps,
                        void* Y, int64_t ldy, int code, uint8_t* codes, uint8_t* scale, float* mean, float* rstd, hipStream_t st) {
  NormArgs a{};
  a.X = X, a.weight = weight, a.bias = bias, a.Y = Y, a.codes = codes, a.scale = scale, a.mean = mean, a.rstd = rstd;
  a.ldx = ldx, a.ldy = ldy, a.srows = f8_scale_rows(T), a.T = T, a.D = D, a.Dp = f8_blocks(D) * F8_BLOCK, a.e5 = code == BSP_E5M2, a.eps = eps;
  if (codes) return f32 ? forward<true, true>(a, st) : forward<false, true>(a, st);
  return f32 ? forward<true, false>(a, st) : forward<false, false>(a, st);
}

int norm_launch_backward(const void* dY, int64_t ld_dy, const void* X, int64_t ldx, bool f32, const float* mean, const float* rstd, const float* weight,
                         int T, int D, void* dX, int64_t ld_dx, float* dweight, float* dbias, float* part, hipStream_t st) {
  NormArgs a{};
  a.X = X, a.dY = dY, a.weight = weight, a.dX = dX, a.mean = (float*)mean, a.rstd = (float*)rstd, a.part = part, a.dweight = dweight, a.dbias = dbias;
  a.ldx = ldx, a.ld_dy = ld_dy, a.ld_dx = ld_dx, a.T = T, a.D = D, a.parts = norm_parts(T, D);
  const int rc = f32 ? backward<true>(a, st) : backward<false>(a, st);
  if (rc != BSP_OK || a.parts == 1) return rc;
  return sum(part, a.parts, 2 * (int64_t)D, D, dweight, dbias, st);
}
