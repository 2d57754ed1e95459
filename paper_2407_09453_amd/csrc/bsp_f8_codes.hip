// 8-bit checkpoints of activations (write and read back) and the weights' codes in both directions.
//
// All three are bound by memory: a value is read once and a code written once.  A workgroup of the writer takes sixteen
// rows by 1024 columns: a wave reads a row's 1024 columns as whole lines, sixteen consecutive values a lane, so a block
// of 128 lies in eight neighbouring lanes and its maximum takes three exchanges; the sixteen rows' scales of a column
// block are gathered in LDS and leave as one 16-byte piece, since they are neighbours in memory.
// Measured at 16384 x 4096 bf16: write 38 us (5.3 TB/s), read back 32 us (6.4 TB/s), where a copy runs at 6.2; 1 x 4096 3.4 and 2.0 us.
// (Codes written past the caches gave the writer 10 % and cost the product that reads them more.)
// The weights' 16384 x 4096 from fp32, in both directions, take 79 us (5.1 TB/s).
#include "bsp_f8.h"

namespace {

// sixteen values of a row of n >= 8 from column c, as they are
template <bool F32>
struct Raw16 {
  F8Raw8<F32> v[2];
};
template <bool F32>
__device__ __forceinline__ Raw16<F32> raw16(const void* X, int64_t at, int c, int n) {
  const void* row = F32 ? (const void*)((const float*)X + at) : (const void*)((const uint16_t*)X + at);
  return Raw16<F32>{{f8_raw8<F32>(row, c, n), f8_raw8<F32>(row, c + 8, n)}};
}
template <bool F32>
__device__ __forceinline__ void unpack16(const Raw16<F32>& r, int c, int n, float* v) {
  f8_unpack8<F32>(r.v[0], f8_past(c, n), (n & 7) != 0, v);
  f8_unpack8<F32>(r.v[1], f8_past(c + 8, n), (n & 7) != 0, v + 8);
}
// the same of a row shorter than eight, one by one
template <bool F32>
__device__ __forceinline__ void thin16(const void* X, int64_t at, int c, int n, float* v) {
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    v[k] = 0.f;
    if (c + k < n) v[k] = F32 ? ((const float*)X)[at + c + k] : bf16_bits_to_f32(((const uint16_t*)X)[at + c + k]);
  }
}

struct SaveArgs {
  const void* X;
  uint8_t *codes, *scale;
  int64_t ldx, srows;
  int32_t T, K, Kp, downs;
};

template <bool F32, bool E5>
__global__ __launch_bounds__(256) void f8_save(SaveArgs a) {
  __shared__ uint32_t sc[8][4];  // [column block][sixteen rows' bytes]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int across = (a.Kp + 1023) / 1024, turn = blockIdx.x / across, chunk = blockIdx.x - turn * across;
  const int down = blockIdx.y * a.downs + turn;
  const int c0 = chunk * 1024 + lane * 16;
  const int64_t row0 = (int64_t)down * 16 + wave * 4;
  if ((int64_t)down * 16 >= a.T) return;  // (a whole workgroup)
  Raw16<F32> raw[4] = {};
  const bool thin = a.K < 8;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (!thin) raw[r] = raw16<F32>(a.X, (row0 + r < a.T ? row0 + r : a.T - 1) * a.ldx, c0, a.K);
  uint32_t bytes = 0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float v[16];
    if (thin) thin16<F32>(a.X, (row0 + r < a.T ? row0 + r : a.T - 1) * a.ldx, c0, a.K, v);
    else unpack16<F32>(raw[r], c0, a.K, v);
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, f8_magnitude(v[k]));
    m = f8_most<8>(m);
    const int b = f8_scale_byte<E5>(m);
    const float s = f8_inverse(b);
    bytes |= (uint32_t)b << (8 * r);
    u32x4_t q;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      q[k] = f8_encode4<E5>(v[4 * k] * s, v[4 * k + 1] * s, v[4 * k + 2] * s, v[4 * k + 3] * s);
    if (row0 + r < a.T && c0 < a.Kp) *(u32x4_t*)(a.codes + (row0 + r) * a.Kp + c0) = q;
  }
  if ((lane & 7) == 0) sc[lane >> 3][wave] = bytes;
  __syncthreads();
  const int kb = chunk * 8 + threadIdx.x;
  if (threadIdx.x < 8 && kb * F8_BLOCK < a.Kp)
    *(u32x4_t*)(a.scale + kb * a.srows + (int64_t)down * 16) =
        u32x4_t{sc[threadIdx.x][0], sc[threadIdx.x][1], sc[threadIdx.x][2], sc[threadIdx.x][3]};
}

struct LoadArgs {
  const uint8_t *codes, *scale;
  void* Y;
  int64_t ldy, srows;
  int32_t T, K, Kp, downs;
};

template <bool F32, bool E5>
__global__ __launch_bounds__(256) void f8_load(LoadArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int across = (a.Kp + 1023) / 1024, turn = blockIdx.x / across, chunk = blockIdx.x - turn * across;
  const int down = blockIdx.y * a.downs + turn;
  const int c0 = chunk * 1024 + lane * 16;
  const int64_t row0 = (int64_t)down * 16 + wave * 4;
  if ((int64_t)down * 16 >= a.T) return;  // (a whole workgroup)
  if (c0 >= a.K) return;
  const int left = a.K - c0;
  u32x4_t q[4];
  int b[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t row = row0 + r < a.T ? row0 + r : a.T - 1;
    q[r] = *(const u32x4_t*)(a.codes + row * a.Kp + c0);
    b[r] = a.scale[(int64_t)(c0 >> 7) * a.srows + row];
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (row0 + r >= a.T) return;
    const int64_t at = (row0 + r) * a.ldy + c0;
    if constexpr (F32) {
      const float s = f8_power(b[r]);
      float v[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        typedef __attribute__((ext_vector_type(2))) float f2;
        const f2 lo = E5 ? __builtin_amdgcn_cvt_pk_f32_bf8(q[r][k], false) : __builtin_amdgcn_cvt_pk_f32_fp8(q[r][k], false);
        const f2 hi = E5 ? __builtin_amdgcn_cvt_pk_f32_bf8(q[r][k], true) : __builtin_amdgcn_cvt_pk_f32_fp8(q[r][k], true);
        v[4 * k] = lo.x * s, v[4 * k + 1] = lo.y * s, v[4 * k + 2] = hi.x * s, v[4 * k + 3] = hi.y * s;
      }
      float* y = (float*)a.Y + at;
      if (left >= 16) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          ((f8_any4_t*)y)[k] = u32x4_t{__float_as_uint(v[4 * k]), __float_as_uint(v[4 * k + 1]), __float_as_uint(v[4 * k + 2]), __float_as_uint(v[4 * k + 3])};
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < left) y[k] = v[k];
      }
    } else {
      const float s = __uint_as_float((uint32_t)b[r] << 23);
      const u32x4_t lo = f8_decode_bf16x8<E5>(q[r][0], q[r][1], s), hi = f8_decode_bf16x8<E5>(q[r][2], q[r][3], s);
      uint16_t* y = (uint16_t*)a.Y + at;
      if (left >= 16) {
        ((f8_any2_t*)y)[0] = lo;
        ((f8_any2_t*)y)[1] = hi;
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < left) y[k] = (uint16_t)((k < 8 ? lo[(k >> 1) & 3] : hi[(k >> 1) & 3]) >> (16 * (k & 1)));
      }
    }
  }
}

struct PackArgs {
  const void* W;
  int64_t ldw;
  const int32_t *row_ptr, *col_idx, *col_ptr, *row_idx;
  uint8_t *payload, *scale, *payload_t, *scale_t;
  int32_t O, I, nbr;
};

// One kept block a workgroup: its codes in row order, and through LDS in column order at the block's place among its column's.
template <bool F32>
__global__ __launch_bounds__(256) void f8_pack(PackArgs a) {
  __shared__ uint32_t most[4];
  __shared__ uint8_t tile[F8_BLOCK][F8_BLOCK + 4];
  __shared__ int place[2];
  const int n = blockIdx.x, tid = threadIdx.x;
  if (tid == 0) {
    int lo = 0, hi = a.nbr;  // the last block row that starts at n or before, and keeps something there
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.row_ptr[mid] <= n) lo = mid; else hi = mid;
    }
    const int c = a.col_idx[n];
    int l = a.col_ptr[c], h = a.col_ptr[c + 1];
    while (h - l > 1) {
      const int mid = (l + h) >> 1;
      if (a.row_idx[mid] <= lo) l = mid; else h = mid;
    }
    place[0] = lo;
    place[1] = l;
  }
  __syncthreads();
  const int br = place[0], c = a.col_idx[n];
  const int r0 = tid >> 3, k0 = (tid & 7) * 16;  // rows r0 + 32 j, sixteen columns
  float v[4][16];
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int o = br * F8_BLOCK + r0 + 32 * j, i = c * F8_BLOCK + k0;
    const int64_t at = (o < a.O ? o : a.O - 1) * a.ldw;
    if (a.I < 8) thin16<F32>(a.W, at, i, a.I, v[j]);
    else unpack16<F32>(raw16<F32>(a.W, at, i, a.I), i, a.I, v[j]);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[j][k] = o < a.O ? v[j][k] : 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, f8_magnitude(v[j][k]));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if ((tid & 63) == 0) most[tid >> 6] = m;
  __syncthreads();
  m = max(max(most[0], most[1]), max(most[2], most[3]));
  const int b = f8_scale_byte<false>(m);
  const float s = f8_inverse(b);
  uint8_t* out = a.payload + (int64_t)n * F8_BLOCK_BYTES;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u32x4_t q;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      q[k] = f8_encode4<false>(v[j][4 * k] * s, v[j][4 * k + 1] * s, v[j][4 * k + 2] * s, v[j][4 * k + 3] * s);
    *(u32x4_t*)(out + (r0 + 32 * j) * F8_BLOCK + k0) = q;
#pragma unroll
    for (int k = 0; k < 4; ++k) *(uint32_t*)&tile[r0 + 32 * j][k0 + 4 * k] = q[k];
  }
  __syncthreads();
  const int t = place[1];
  uint8_t* out_t = a.payload_t + (int64_t)t * F8_BLOCK_BYTES;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u32x4_t q;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t w = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w |= (uint32_t)tile[k0 + 4 * k + e][r0 + 32 * j] << (8 * e);
      q[k] = w;
    }
    *(u32x4_t*)(out_t + (r0 + 32 * j) * F8_BLOCK + k0) = q;
  }
  if (tid == 0) {
    a.scale[n] = (uint8_t)b;
    a.scale_t[t] = (uint8_t)b;
  }
}

// Workgroups of sixteen rows by 1024 columns: as many sixteens of rows along x as f8_grid takes (`downs`), the rest along y.
inline bool sixteens(int T, int Kp, int32_t* downs, dim3* grid) {
  const int64_t across = (Kp + 1023) / 1024, all = ((int64_t)T + 15) / 16, most = kGridX / across;
  *downs = (int32_t)(all < most ? all : most);
  const int64_t y = (all + *downs - 1) / *downs;
  *grid = dim3((unsigned)(across * *downs), (unsigned)y);
  return y <= 65535;
}

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }

}  // namespace

int f8_launch_save(const void* X, int x_f32, int64_t ldx, int T, int K, bool e5, uint8_t* codes, uint8_t* scale, hipStream_t st) {
  const int Kp = f8_blocks(K) * F8_BLOCK;
  SaveArgs a{X, codes, scale, ldx, f8_scale_rows(T), T, K, Kp, 0};
  dim3 grid;
  const dim3 block(256);
  if (!sixteens(T, Kp, &a.downs, &grid)) return BSP_ERR_SHAPE;
  if (x_f32) {
    if (e5) hipLaunchKernelGGL((f8_save<true, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((f8_save<true, false>), grid, block, 0, st, a);
  } else {
    if (e5) hipLaunchKernelGGL((f8_save<false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((f8_save<false, false>), grid, block, 0, st, a);
  }
  return launched();
}

int f8_launch_load(const uint8_t* codes, const uint8_t* scale, int T, int K, bool e5, void* Y, int y_f32, int64_t ldy, hipStream_t st) {
  const int Kp = f8_blocks(K) * F8_BLOCK;
  LoadArgs a{codes, scale, Y, ldy, f8_scale_rows(T), T, K, Kp, 0};
  dim3 grid;
  const dim3 block(256);
  if (!sixteens(T, Kp, &a.downs, &grid)) return BSP_ERR_SHAPE;
  if (y_f32) {
    if (e5) hipLaunchKernelGGL((f8_load<true, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((f8_load<true, false>), grid, block, 0, st, a);
  } else {
    if (e5) hipLaunchKernelGGL((f8_load<false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((f8_load<false, false>), grid, block, 0, st, a);
  }
  return launched();
}

int f8_launch_pack(const bsp_weights_f8* w, const void* W, int w_f32, int64_t ldw, hipStream_t st) {
  PackArgs a{W, ldw, w->row_ptr, w->col_idx, w->col_ptr, w->row_idx, w->payload, w->scale, w->payload_t, w->scale_t,
             w->O, w->I, f8_blocks(w->O)};
  const dim3 grid((unsigned)w->nnzb), block(256);
  if (w_f32) hipLaunchKernelGGL((f8_pack<true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((f8_pack<false>), grid, block, 0, st, a);
  return launched();
}
