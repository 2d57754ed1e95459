// Layer norm over the last axis, forward and backward, bound by memory.
//
//   mu = mean x, v = mean (x - mu)^2, r = 1 / sqrt(v + eps), h = (x - mu) r, y = h w + b
//   g = dy w, dx = r (g - mean g - h mean(g h)), dw = sum over rows of dy h, db = sum over rows of dy
//
// A row is read once and stays in the registers of the 64 or 256 threads that own it, so the mean is known before the
// deviations are squared (no difference of large sums); everything is summed in fp32.  Rows too long for that are read again.
// The gradient's threads own columns: each adds its columns' dw and db over all the rows that its workgroup takes, and
// a second launch adds the workgroups' sums in a fixed order (no atomics: the same inputs give the same bits).
// The forward pass can leave its result as 8-bit codes, from the fp32 values: sixteen neighbouring lanes hold a block of 128.
#include "bsp_f8.h"

namespace {

struct NormArgs {
  const void *X, *dY;
  const float *weight, *bias;
  void *Y, *dX;
  uint8_t *codes, *scale;
  float *mean, *rstd, *part;
  int64_t ldx, ldy, ld_dy, ld_dx, srows;
  int32_t T, D, Dp, e5, vec, parts;
  float eps;
};

template <bool F32>
__device__ __forceinline__ void load8(const void* X, int64_t at, int left, bool vec, float* v) {
  if (vec && left >= 8) {
    if constexpr (F32) {
      const f32x4_t a = ((const f32x4_t*)((const float*)X + at))[0], b = ((const f32x4_t*)((const float*)X + at))[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
    } else {
      const u32x4_t w = *(const u32x4_t*)((const uint16_t*)X + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[2 * k] = __uint_as_float(w[k] << 16), v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = 0.f;
    if (k < left) v[k] = F32 ? ((const float*)X)[at + k] : bf16_bits_to_f32(((const uint16_t*)X)[at + k]);
  }
}

template <bool F32>
__device__ __forceinline__ void store8(void* Y, int64_t at, int left, bool vec, const float* v) {
  if constexpr (F32) {
    float* y = (float*)Y + at;
    if (vec && left >= 8) {
      ((f32x4_t*)y)[0] = f32x4_t{v[0], v[1], v[2], v[3]};
      ((f32x4_t*)y)[1] = f32x4_t{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) y[k] = v[k];
  } else {
    uint16_t* y = (uint16_t*)Y + at;
    const u32x4_t w = {f8_pack_bf16x2(v[0], v[1]), f8_pack_bf16x2(v[2], v[3]), f8_pack_bf16x2(v[4], v[5]), f8_pack_bf16x2(v[6], v[7])};
    if (vec && left >= 8) {
      *(u32x4_t*)y = w;
      return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) y[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
  }
}

// sums of N values over the threads of a row (64: a wave, 256: the workgroup)
template <int ROWT, int N>
__device__ __forceinline__ void row_sum(float* v, float (*sh)[N]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], d);
  if constexpr (ROWT == 256) {
    __syncthreads();  // the last use of sh is over
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) sh[threadIdx.x >> 6][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (sh[0][k] + sh[1][k]) + (sh[2][k] + sh[3][k]);
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
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
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
    store8<F32>(a.Y, row * a.ldy + c, a.D - c, a.vec, y);
  }
}

// NV: groups of eight columns a thread holds; 0: rows of any length, read three times
template <bool F32, bool CODES, int ROWT, int NV>
__global__ __launch_bounds__(256) void norm_forward(NormArgs a) {
  __shared__ float sh[4][1];
  const int tid = threadIdx.x % ROWT;
  const int64_t row = ROWT == 256 ? blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.T) return;  // (whole waves)
  const int64_t xr = row * a.ldx;
  const float inv = 1.f / (float)a.D;
  if constexpr (NV > 0) {
    float v[NV][8];
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
      load8<F32>(a.X, c < a.D ? xr + c : 0, c < a.D ? a.D - c : 0, a.vec, v[j]);
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
      if (a.weight) load8<true>(a.weight, c < a.D ? c : 0, c < a.D ? a.D - c : 0, a.vec, w);
      if (a.bias) load8<true>(a.bias, c < a.D ? c : 0, c < a.D ? a.D - c : 0, a.vec, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] = c + k < a.D ? v[j][k] * rstd * w[k] + b[k] : 0.f;
      put8<F32, CODES>(a, row, c, v[j]);
    }
  } else {
    float s[1] = {0.f}, v[8];
    for (int c = tid * 8; c < a.D; c += ROWT * 8) {
      load8<F32>(a.X, xr + c, a.D - c, a.vec, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[0] += v[k];
    }
    row_sum<ROWT, 1>(s, sh);
    const float mean = s[0] * inv;
    s[0] = 0.f;
    for (int c = tid * 8; c < a.D; c += ROWT * 8) {
      load8<F32>(a.X, xr + c, a.D - c, a.vec, v);
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
      load8<F32>(a.X, left > 0 ? xr + c : 0, left, a.vec, v);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = k < left ? (v[k] - mean) * rstd * (a.weight ? a.weight[c + k] : 1.f) + (a.bias ? a.bias[c + k] : 0.f) : 0.f;
      put8<F32, CODES>(a, row, c, v);
    }
  }
}

template <bool F32, int ROWT, int NV>
__global__ __launch_bounds__(256) void norm_backward(NormArgs a) {
  __shared__ float sh[4][2];
  const int tid = threadIdx.x % ROWT;
  const int group = ROWT == 256 ? blockIdx.x : blockIdx.x * 4 + (threadIdx.x >> 6);
  const float inv = 1.f / (float)a.D;
  float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (tid + j * ROWT) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) w[j][k] = 1.f, dw[j][k] = 0.f, db[j][k] = 0.f;
    if (a.weight) load8<true>(a.weight, c < a.D ? c : 0, c < a.D ? a.D - c : 0, a.vec, w[j]);
  }
  for (int64_t row = group; row < a.T; row += a.parts) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    float h[NV][8], g[NV][8], s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
      load8<F32>(a.X, c < a.D ? row * a.ldx + c : 0, c < a.D ? a.D - c : 0, a.vec, h[j]);
      load8<F32>(a.dY, c < a.D ? row * a.ld_dy + c : 0, c < a.D ? a.D - c : 0, a.vec, g[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        h[j][k] = (tid + j * ROWT) * 8 + k < a.D ? (h[j][k] - mean) * rstd : 0.f;
        dw[j][k] += g[j][k] * h[j][k];
        db[j][k] += g[j][k];
        g[j][k] *= w[j][k];
        s[0] += g[j][k];
        s[1] += g[j][k] * h[j][k];
      }
    row_sum<ROWT, 2>(s, sh);
    const float mg = s[0] * inv, mh = s[1] * inv;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (tid + j * ROWT) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) g[j][k] = rstd * (g[j][k] - mg - h[j][k] * mh);
      if (c < a.D) store8<F32>(a.dX, row * a.ld_dx + c, a.D - c, a.vec, g[j]);
    }
  }
  if (group >= a.parts) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (tid + j * ROWT) * 8;
    if (c >= a.D) continue;
    store8<true>(a.part, (int64_t)group * 2 * a.D + c, a.D - c, a.D % 4 == 0, dw[j]);
    store8<true>(a.part, ((int64_t)group * 2 + 1) * a.D + c, a.D - c, a.D % 4 == 0, db[j]);
  }
}

// Rows of any length: dx, reading the row twice, and a second kernel for the columns' sums.
template <bool F32>
__global__ __launch_bounds__(256) void norm_backward_long(NormArgs a) {
  __shared__ float sh[4][2];
  const int64_t row = blockIdx.x;
  const float inv = 1.f / (float)a.D, mean = a.mean[row], rstd = a.rstd[row];
  float s[2] = {0.f, 0.f}, h[8], g[8];
  for (int c = threadIdx.x * 8; c < a.D; c += 2048) {
    load8<F32>(a.X, row * a.ldx + c, a.D - c, a.vec, h);
    load8<F32>(a.dY, row * a.ld_dy + c, a.D - c, a.vec, g);
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
    load8<F32>(a.X, row * a.ldx + c, a.D - c, a.vec, h);
    load8<F32>(a.dY, row * a.ld_dy + c, a.D - c, a.vec, g);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      g[k] = c + k < a.D ? rstd * (g[k] * (a.weight ? a.weight[c + k] : 1.f) - mg - (h[k] - mean) * rstd * mh) : 0.f;
    store8<F32>(a.dX, row * a.ld_dx + c, a.D - c, a.vec, g);
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
  a.part[(int64_t)blockIdx.y * 2 * a.D + c] = dw;
  a.part[((int64_t)blockIdx.y * 2 + 1) * a.D + c] = db;
}

// out[c] = sum of part[p][c] over p, in the order of p within each of four threads: 64 columns a workgroup
__global__ __launch_bounds__(256) void norm_sum(const float* part, int parts, int64_t width, int64_t split_at, float* out, float* out2) {
  __shared__ float sh[4][64];
  const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int q = threadIdx.x >> 6;
  float s = 0.f;
  if (c < width)
    for (int p = q; p < parts; p += 4) s += part[p * width + c];
  sh[q][threadIdx.x & 63] = s;
  __syncthreads();
  if (q == 0 && c < width) {
    s = (sh[0][threadIdx.x] + sh[1][threadIdx.x]) + (sh[2][threadIdx.x] + sh[3][threadIdx.x]);
    float* to = c < split_at ? out + c : out2 + (c - split_at);
    if (c < split_at ? out != nullptr : out2 != nullptr) *to = s;
  }
}

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }
inline bool aligned(const void* p, int64_t stride_bytes) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)stride_bytes) & 15u) == 0; }

template <bool F32, bool CODES>
int forward(const NormArgs& a, hipStream_t st) {
  const dim3 block(256), rows((unsigned)a.T), quads((unsigned)((a.T + 3) / 4));
  if (a.Dp <= 512) hipLaunchKernelGGL((norm_forward<F32, CODES, 64, 1>), quads, block, 0, st, a);
  else if (a.Dp <= 1024) hipLaunchKernelGGL((norm_forward<F32, CODES, 64, 2>), quads, block, 0, st, a);
  else if (a.Dp <= 2048) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 1>), rows, block, 0, st, a);
  else if (a.Dp <= 4096) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 2>), rows, block, 0, st, a);
  else if (a.Dp <= 8192) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 4>), rows, block, 0, st, a);
  else if (a.Dp <= 16384) hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 8>), rows, block, 0, st, a);
  else hipLaunchKernelGGL((norm_forward<F32, CODES, 256, 0>), rows, block, 0, st, a);
  return launched();
}

template <bool F32>
int backward(const NormArgs& a, hipStream_t st) {
  const dim3 block(256), parts((unsigned)a.parts), quads((unsigned)((a.parts + 3) / 4));
  if (a.D <= 512) hipLaunchKernelGGL((norm_backward<F32, 64, 1>), quads, block, 0, st, a);
  else if (a.D <= 2048) hipLaunchKernelGGL((norm_backward<F32, 256, 1>), parts, block, 0, st, a);
  else if (a.D <= 4096) hipLaunchKernelGGL((norm_backward<F32, 256, 2>), parts, block, 0, st, a);
  else if (a.D <= 8192) hipLaunchKernelGGL((norm_backward<F32, 256, 4>), parts, block, 0, st, a);
  else {
    if (a.T > 0) hipLaunchKernelGGL((norm_backward_long<F32>), dim3((unsigned)a.T), block, 0, st, a);
    if (launched() != BSP_OK) return BSP_ERR_HIP;
    hipLaunchKernelGGL((norm_columns_long<F32>), dim3((unsigned)((a.D + 255) / 256), (unsigned)a.parts), block, 0, st, a);
  }
  return launched();
}

int sum(const float* part, int parts, int64_t width, int64_t split_at, float* out, float* out2, hipStream_t st) {
  hipLaunchKernelGGL(norm_sum, dim3((unsigned)((width + 63) / 64)), dim3(256), 0, st, part, parts, width, split_at, out, out2);
  return launched();
}

}  // namespace

int norm_parts(int T) { return T < 1 ? 1 : T < 512 ? T : 512; }

int norm_launch_sum(const float* part, int parts, int O, float* out, hipStream_t st) { return sum(part, parts, O, O, out, nullptr, st); }

int norm_launch_forward(const void* X, bool f32, int64_t ldx, int T, int D, const float* weight, const float* bias, float eps,
                        void* Y, int64_t ldy, int code, uint8_t* codes, uint8_t* scale, float* mean, float* rstd, hipStream_t st) {
  NormArgs a{};
  a.X = X, a.weight = weight, a.bias = bias, a.Y = Y, a.codes = codes, a.scale = scale, a.mean = mean, a.rstd = rstd;
  a.ldx = ldx, a.ldy = ldy, a.srows = f8_scale_rows(T), a.T = T, a.D = D, a.Dp = f8_blocks(D) * F8_BLOCK, a.e5 = code == BSP_E5M2, a.eps = eps;
  const int size = f32 ? 4 : 2;
  a.vec = aligned(X, ldx * size) && aligned(weight, 0) && aligned(bias, 0) && (codes || aligned(Y, ldy * size));
  if (codes) return f32 ? forward<true, true>(a, st) : forward<false, true>(a, st);
  return f32 ? forward<true, false>(a, st) : forward<false, false>(a, st);
}

int norm_launch_backward(const void* dY, int64_t ld_dy, const void* X, int64_t ldx, bool f32, const float* mean, const float* rstd, const float* weight,
                         int T, int D, void* dX, int64_t ld_dx, float* dweight, float* dbias, float* part, hipStream_t st) {
  NormArgs a{};
  a.X = X, a.dY = dY, a.weight = weight, a.dX = dX, a.mean = (float*)mean, a.rstd = (float*)rstd, a.part = part;
  a.ldx = ldx, a.ld_dy = ld_dy, a.ld_dx = ld_dx, a.T = T, a.D = D, a.parts = norm_parts(T);
  const int size = f32 ? 4 : 2;
  a.vec = aligned(X, ldx * size) && aligned(dY, ld_dy * size) && aligned(dX, ld_dx * size) && aligned(weight, 0);
  const int rc = f32 ? backward<true>(a, st) : backward<false>(a, st);
  if (rc != BSP_OK) return rc;
  return sum(part, a.parts, 2 * (int64_t)D, D, dweight, dbias, st);
}
