// FC layers on many rows, weights and activations in 8-bit codes: Y = act(X W^t + b + residual), bound by the matrix cores.
//
// A workgroup owns BT rows by R block rows of 128 channels and walks the block columns that its block rows keep; a step is 128
// columns, both operands staged in LDS with 16-byte asynchronous copies (two buffers: a step is multiplied while the
// next one arrives).  The weights are the matrix core's rows and the activations its columns, so a lane's four
// neighbouring results are neighbouring channels of one row of Y, and an activation's scale is one byte a lane.
// A staged row of 128 bytes is eight pieces of 16; piece p of row r lies at place p ^ (r / 2 mod 8), so sixteen rows' same
// piece, which sixteen lanes read together, lie in sixteen different bank groups.
#include "bsp_f8.h"

namespace {

struct TileArgs {
  F8Rows w;
  const uint8_t *X, *scale;
  F8Epilogue q;
  int64_t ld, srows;
  int32_t T, tiles_t, tiles_o;
};

__device__ __forceinline__ i32x8_t read_fragment(const uint8_t* p, int at0, int at1) {
  const u32x4_t a = *(const u32x4_t*)(p + at0), b = *(const u32x4_t*)(p + at1);
  return i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

__device__ __forceinline__ f32x16_t mfma_bf16_32x32x16(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// MO x MT tiles of 32 x 32 a wave, WO x WT waves; R block rows
template <int MO, int MT, int WO, int WT, bool E5, bool F32>
__global__ __launch_bounds__(64 * WO * WT) void f8_tile(TileArgs a) {
  constexpr int NO = 32 * MO * WO, NT = 32 * MT * WT, WAVES = WO * WT, R = NO / F8_BLOCK;
  constexpr int STAGE = (NO + NT) * F8_BLOCK;
  static_assert(NO % F8_BLOCK == 0 && (NO + NT) % (8 * WAVES) == 0);
  extern __shared__ uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave / WT, wt = wave % WT;
  const int tile_o = blockIdx.x % a.tiles_o, tile_t = blockIdx.x / a.tiles_o;
  const int br = tile_o * R;
  const int64_t t0 = (int64_t)tile_t * NT;
  const int n0 = a.w.ptr[br], n1 = a.w.ptr[br + 1];

  // this lane's part of a request of eight staged rows: row lane / 8 at place lane % 8
  const int srow = lane >> 3;
  // pieces that this lane reads of its row of a fragment, for the two halves of a step
  const int f = (lane >> 1) & 7, g2 = (lane >> 5) * 2;
  int at[2][2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int q = 0; q < 2; ++q) at[h][q] = (lane & 31) * F8_BLOCK + (((4 * h + g2 + q) ^ f) << 4);

  int64_t trow[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t t = t0 + (wt * MT + m) * 32 + (lane & 31);
    trow[m] = t < a.T ? t : a.T - 1;
  }

  auto stage = [&](int n, int buf) {
    uint8_t* base = lds + buf * STAGE;
    const int kb = a.w.idx[n];
#pragma unroll
    for (int q = wave; q < (NO + NT) / 8; q += WAVES) {
      const int row = q * 8 + srow;
      const int piece = (lane & 7) ^ ((row >> 1) & 7);
      const uint8_t* src;
      if (row < NO) {
        const int64_t blk = R == 1 ? n : n + (int64_t)(row >> 7) * (n1 - n0);
        src = a.w.payload + blk * F8_BLOCK_BYTES + (row & 127) * F8_BLOCK + piece * 16;
      } else {
        int64_t t = t0 + row - NO;
        t = t < a.T ? t : a.T - 1;  // rows past the last: the last one's bytes, their results go nowhere
        src = a.X + t * a.ld + (int64_t)kb * F8_BLOCK + piece * 16;
      }
      __builtin_amdgcn_global_load_lds((f8_gptr_t)src, (f8_lptr_t)(base + q * 1024), 16, 0, 0);
    }
  };

  f32x16_t acc[MO][MT] = {};
  if (n0 < n1) stage(n0, 0);
  for (int n = n0; n < n1; ++n) {
    const int buf = (n - n0) & 1;
    int sx[MT];
    const int kb = a.w.idx[n];
#pragma unroll
    for (int m = 0; m < MT; ++m) sx[m] = a.scale[kb * a.srows + trow[m]];
    const int sw = a.w.scale[R == 1 ? n : n + (int64_t)((wo * MO * 32) >> 7) * (n1 - n0)];
    __builtin_amdgcn_s_waitcnt(0);  // this wave's requests have landed,
    __builtin_amdgcn_s_barrier();   // and every wave's; the other buffer has been read
    asm volatile("" ::: "memory");
    if (n + 1 < n1) stage(n + 1, buf ^ 1);
    const uint8_t* W = lds + buf * STAGE + wo * MO * 32 * F8_BLOCK;
    const uint8_t* X = lds + buf * STAGE + (NO + wt * MT * 32) * F8_BLOCK;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i32x8_t x[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) x[m] = read_fragment(X + m * 32 * F8_BLOCK, at[h][0], at[h][1]);
#pragma unroll
      for (int o = 0; o < MO; ++o) {
        const i32x8_t w = read_fragment(W + o * 32 * F8_BLOCK, at[h][0], at[h][1]);
        if constexpr (F32) {  // as bf16, so that nothing is lost in the sum (see f8_few)
          const float fw = __uint_as_float((uint32_t)sw << 23);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x4_t wj = f8_decode_bf16x8<false>(w[2 * j], w[2 * j + 1], fw);
#pragma unroll
            for (int m = 0; m < MT; ++m)
              acc[o][m] = mfma_bf16_32x32x16(wj, f8_decode_bf16x8<E5>(x[m][2 * j], x[m][2 * j + 1], __uint_as_float((uint32_t)sx[m] << 23)), acc[o][m]);
          }
        } else {
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[o][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x[m], acc[o][m], 0, E5 ? 1 : 0, 0, sw, 0, sx[m]);
        }
      }
    }
  }

  const int ob = tile_o * NO + wo * MO * 32 + (lane >> 5) * 4;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t t = t0 + (wt * MT + m) * 32 + (lane & 31);
    if (t >= a.T) continue;
#pragma unroll
    for (int o = 0; o < MO; ++o)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = ob + o * 32 + q * 8;
        if (c < a.w.out) f8_store4<F32>(a.q, t, c, a.w.out, acc[o][m][4 * q], acc[o][m][4 * q + 1], acc[o][m][4 * q + 2], acc[o][m][4 * q + 3]);
      }
  }
}

template <int MO, int MT, int WO, int WT, bool E5, bool F32>
int launch(TileArgs a, hipStream_t st) {
  constexpr int NO = 32 * MO * WO, NT = 32 * MT * WT;
  constexpr int lds = 2 * (NO + NT) * F8_BLOCK;
  static const bool raised = hipFuncSetAttribute((const void*)&f8_tile<MO, MT, WO, WT, E5, F32>, hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
  if (!raised) return BSP_ERR_HIP;
  a.tiles_o = (a.w.out + NO - 1) / NO;
  a.tiles_t = (a.T + NT - 1) / NT;
  if ((int64_t)a.tiles_o * a.tiles_t > INT32_MAX) return BSP_ERR_SHAPE;
  hipLaunchKernelGGL((f8_tile<MO, MT, WO, WT, E5, F32>), dim3((unsigned)(a.tiles_o * a.tiles_t)), dim3(64 * WO * WT), lds, st, a);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}

}  // namespace

int f8_launch_tile(const F8Rows& w, const F8Input& x, int T, const F8Epilogue& q, bool f32, hipStream_t st) {
  TileArgs a{w, (const uint8_t*)x.X, x.scale, q, x.ld, f8_scale_rows(T), T, 0, 0};
  const bool e5 = x.e5;
  if (f32) return e5 ? launch<2, 2, 2, 2, true, true>(a, st) : launch<2, 2, 2, 2, false, true>(a, st);
  return e5 ? launch<2, 2, 2, 2, true, false>(a, st) : launch<2, 2, 2, 2, false, false>(a, st);
}
