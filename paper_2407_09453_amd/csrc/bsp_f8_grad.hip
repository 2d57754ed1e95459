// The weights' gradient of an FC layer from the 8-bit checkpoint of its input: dW[o][i] = sum_t dY[t][o] X[t][i] for kept blocks
// only, and the bias's, db[o] = sum_t dY[t][o].
//
// A scale of the checkpoint belongs to a row t and 128 columns, and t is what the product sums over, so no scaled matrix
// instruction fits; code x power of two is exact in bf16, and the product runs on the bf16 matrix cores with fp32 sums.
// Codes become bf16 on their way into LDS (a conversion of two values takes the scale along).  Both operands are
// summed over their rows: LDS holds them as they lie in memory, row after row, and the transposing LDS read hands a lane
// four rows of its column.  It takes four rows of 32 bytes from a group of sixteen lanes, so the 32-byte chunks of a
// row are permuted by the row (bits 0, 1 and 3): four rows' same chunk, and those of two groups, lie in different banks.
#include "bsp_f8.h"

namespace {

constexpr int kStep = 64;  // rows a step

typedef __attribute__((ext_vector_type(4))) short s16x4_t;

__device__ __forceinline__ u32x4_t read_columns(const uint8_t* p) {  // rows +0..3 and +4..7 of this lane's column
  auto* q = (__attribute__((address_space(3))) s16x4_t*)(uintptr_t)p;
  const u32x2_t a = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q));
  const u32x2_t b = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + 4 * 256 / 8));
  return u32x4_t{a.x, a.y, b.x, b.y};
}

__device__ __forceinline__ int chunk_key(int t) { return (t & 3) | (((t >> 3) & 1) << 2); }

template <bool E5, bool VEC>
__global__ __launch_bounds__(256) void f8_grad(F8GradArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t ly[kStep * 256], lx[kStep * 256];
  __shared__ int place;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = blockIdx.x;
  if (tid == 0) {
    int lo = 0, hi = a.nbo;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.row_ptr[mid] <= n) lo = mid; else hi = mid;
    }
    place = lo;
  }
  __syncthreads();
  const int br = place, kb = a.col_idx[n];
  const int Kp = f8_blocks(a.I) * F8_BLOCK;
  const int64_t srows = f8_scale_rows(a.T);
  const int steps = (a.T + kStep - 1) / kStep, per = (steps + a.split - 1) / a.split;
  const int64_t t_begin = (int64_t)blockIdx.y * per * kStep;
  const int64_t t_end = t_begin + (int64_t)per * kStep < a.T ? t_begin + (int64_t)per * kStep : a.T;
  const int wo = wave >> 1, wi = wave & 1;
  const int key = ((lane & 15) >> 2) | ((lane >> 5) << 2);
  const int trow = (lane >> 5) * 8 + ((lane & 15) >> 2);
  int ao[2], ai[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    ao[m] = trow * 256 + (((wo * 4 + m * 2 + ((lane >> 4) & 1)) ^ key) << 5) + (lane & 3) * 8;
    ai[m] = trow * 256 + (((wi * 4 + m * 2 + ((lane >> 4) & 1)) ^ key) << 5) + (lane & 3) * 8;
  }
  f32x16_t acc[2][2] = {};
  for (int64_t t0 = t_begin; t0 < t_end; t0 += kStep) {
    // gradients: a request is four rows of 256 bytes
#pragma unroll
    for (int q = 0; q < kStep / 16; ++q) {
      const int row = (q * 4 + wave) * 4 + (lane >> 4);
      const int slot = lane & 15, piece = (((slot >> 1) ^ chunk_key(row)) << 1) | (slot & 1);
      const int o = br * F8_BLOCK + piece * 8;
      uint8_t* to = ly + (q * 4 + wave) * 1024;
      if constexpr (VEC) {
        if (t0 + row < t_end) {
          const uint16_t* src = a.dY + (t0 + row) * a.ldy + (o < a.O ? o : 0);  // past the last channel: results that go nowhere
          __builtin_amdgcn_global_load_lds((f8_gptr_t)src, (f8_lptr_t)(uintptr_t)to, 16, 0, 0);
        } else {
          *(u32x4_t*)(to + lane * 16) = u32x4_t{0, 0, 0, 0};
        }
      } else {
        uint32_t v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = t0 + row < t_end && o + k < a.O ? a.dY[(t0 + row) * a.ldy + o + k] : 0;
        *(u32x4_t*)(to + lane * 16) = u32x4_t{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
      }
    }
    // the checkpoint: 32 codes a thread
    {
      const int row = tid >> 2, part = tid & 3;
      u32x4_t c[2] = {};
      float s = 0.f;
      if (t0 + row < t_end) {
        const u32x4_t* src = (const u32x4_t*)(a.codes + (t0 + row) * Kp + kb * F8_BLOCK + part * 32);
        c[0] = src[0];
        c[1] = src[1];
        s = __uint_as_float((uint32_t)a.scale[kb * srows + t0 + row] << 23);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4_t* to = (u32x4_t*)(lx + row * 256 + (((part * 2 + h) ^ chunk_key(row)) << 5));
        to[0] = f8_decode_bf16x8<E5>(c[h].x, c[h].y, s);
        to[1] = f8_decode_bf16x8<E5>(c[h].z, c[h].w, s);
      }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep; k += 16) {
      u32x4_t y[2], x[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        y[m] = read_columns(ly + k * 256 + ao[m]);
        x[m] = read_columns(lx + k * 256 + ai[m]);
      }
#pragma unroll
      for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, y[o]), __builtin_bit_cast(bf16x8_t, x[i]), acc[o][i], 0, 0, 0);
    }
    __syncthreads();
  }
  const bool whole = a.split == 1;
  float* out = whole ? a.dW + (int64_t)br * F8_BLOCK * a.I + (int64_t)kb * F8_BLOCK
                     : a.part + ((int64_t)blockIdx.y * a.nnzb + n) * F8_BLOCK_BYTES;
  const int64_t ld = whole ? a.I : F8_BLOCK;
  const int rows = whole ? a.O - br * F8_BLOCK : F8_BLOCK, cols = whole ? a.I - kb * F8_BLOCK : F8_BLOCK;
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = wi * 64 + i * 32 + (lane & 31);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = wo * 64 + o * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
        if (row < rows && c < cols) out[row * ld + c] = acc[o][i][r];
      }
    }
}

// Blocks that are not kept become zeros; those that are get the sum over the ranges of rows, in their order.
__global__ __launch_bounds__(256) void f8_grad_finish(F8GradArgs a) {
  const int kb = blockIdx.x % a.nbi, br = blockIdx.x / a.nbi;
  int n = a.row_ptr[br];
  const int n1 = a.row_ptr[br + 1];
  while (n < n1 && a.col_idx[n] < kb) ++n;
  const bool kept = n < n1 && a.col_idx[n] == kb;
  if (kept && a.split == 1) return;
  const int c = threadIdx.x & 127;
  if (kb * F8_BLOCK + c >= a.I) return;
  for (int r = threadIdx.x >> 7; r < F8_BLOCK; r += 2) {
    const int64_t o = (int64_t)br * F8_BLOCK + r;
    if (o >= a.O) return;
    float v = 0.f;
    if (kept)
      for (int s = 0; s < a.split; ++s) v += a.part[((int64_t)s * a.nnzb + n) * F8_BLOCK_BYTES + r * F8_BLOCK + c];
    a.dW[o * a.I + kb * F8_BLOCK + c] = v;
  }
}

// Column sums of dY over one range of rows a workgroup: a thread owns two columns' sums.
__global__ __launch_bounds__(256) void f8_colsum(const uint16_t* dY, int64_t ldy, int T, int O, int parts, float* part) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= O) return;
  const int64_t per = ((int64_t)T + parts - 1) / parts;
  const int64_t t0 = blockIdx.y * per, t1 = t0 + per < T ? t0 + per : T;
  float s = 0.f;
  for (int64_t t = t0; t < t1; ++t) s += bf16_bits_to_f32(dY[t * ldy + c]);
  part[(int64_t)blockIdx.y * O + c] = s;
}

}  // namespace

int f8_grad_split(int64_t nnzb, int T) {
  const int64_t steps = ((int64_t)T + 2 * kStep - 1) / (2 * kStep);
  int64_t s = nnzb > 0 ? 512 / nnzb : 1;
  if (s > steps) s = steps;
  return s < 1 ? 1 : (int)s;
}

int f8_launch_grad(const F8GradArgs& a, hipStream_t st) {
  const bool vec = ((reinterpret_cast<uintptr_t>(a.dY) | (uintptr_t)(a.ldy * 2)) & 15u) == 0 && a.O % 8 == 0;
  if (a.nnzb > 0) {
    const dim3 grid((unsigned)a.nnzb, (unsigned)a.split), block(256);
    if (a.e5) {
      if (vec) hipLaunchKernelGGL((f8_grad<true, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((f8_grad<true, false>), grid, block, 0, st, a);
    } else {
      if (vec) hipLaunchKernelGGL((f8_grad<false, true>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((f8_grad<false, false>), grid, block, 0, st, a);
    }
    if (hipGetLastError() != hipSuccess) return BSP_ERR_HIP;
  }
  if (a.split > 1 || a.nnzb < (int64_t)a.nbo * a.nbi) {
    hipLaunchKernelGGL(f8_grad_finish, dim3((unsigned)(a.nbo * a.nbi)), dim3(256), 0, st, a);
    if (hipGetLastError() != hipSuccess) return BSP_ERR_HIP;
  }
  return BSP_OK;
}

int f8_launch_colsum(const uint16_t* dY, int64_t ldy, int T, int O, float* part, float* db, hipStream_t st) {
  const int parts = norm_parts(T);
  hipLaunchKernelGGL(f8_colsum, dim3((unsigned)((O + 255) / 256), (unsigned)parts), dim3(256), 0, st, dY, ldy, T, O, parts, part);
  if (hipGetLastError() != hipSuccess) return BSP_ERR_HIP;
  return norm_launch_sum(part, parts, O, db, st);
}
