// FC layers on few rows, weights in 8-bit codes: Y = X W^t, bound by the bytes of the weights (serving), or by latency.
//
// A workgroup owns 16 output channels and 16 MT rows; its waves share out the kept blocks of the channels' block row, each
// adding its blocks' products in its own accumulators, and the waves' sums meet in LDS: the long axis is split inside the
// workgroup, with no second launch and no memory for partial sums.  Operands go from memory to registers: a lane's 32 bytes of
// a weight row are two loads, sixteen rows are 2 KB in one piece, and a block's lines are each asked for once in the chip.
// Rows given as bf16 or fp32 are brought to codes in registers (MT = 1): a lane reads the 32 columns that it feeds to
// the matrix core, the four lanes of a row exchange their largest magnitudes, and the codes are where they are wanted.
#include "bsp_f8.h"

namespace {

struct FewArgs {
  F8Rows w;
  F8Input x;
  F8Epilogue q;
  int64_t srows;   // rows of x.scale
  int32_t T, xvec;
};

// 128 products per lane row: scaled codes, or (F32) both sides as bf16 so that nothing is lost in the sum.  The instruction on
// codes adds eight products at a time and cuts each off 13 bits below the largest of the eight (256 x 256 + 7 is 256 x 256): 1.4e-5
// of a sum's spread on ordinary data, far below a bf16 result's rounding, but not below an fp32 one's.
template <bool F32, bool E5>
__device__ __forceinline__ f32x4_t few_mfma(i32x8_t a, int sa, i32x8_t b, int sb, f32x4_t c) {
  if constexpr (F32) {
    const float fa = __uint_as_float((uint32_t)sa << 23), fb = __uint_as_float((uint32_t)sb << 23);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = mfma_bf16_16x16x32(f8_decode_bf16x8<false>(a[2 * j], a[2 * j + 1], fa), f8_decode_bf16x8<E5>(b[2 * j], b[2 * j + 1], fb), c);
    return c;
  } else {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, E5 ? 1 : 0, 0, sa, 0, sb);
  }
}

enum { kCodes, kBf16, kF32 };  // what the rows are given as
template <int SRC, bool E5>
__device__ __forceinline__ i32x8_t few_input(const FewArgs& a, int64_t t, int kb, int g, int* scale) {
  if constexpr (SRC == kCodes) {
    *scale = a.x.scale[kb * a.srows + t];
    const i32x8_t* p = (const i32x8_t*)((const uint8_t*)a.x.X + t * a.x.ld + kb * F8_BLOCK + g * 32);
    return *p;
  } else {
    float v[32];
    const int k0 = kb * F8_BLOCK + g * 32, left = a.w.in - k0;
    if (a.xvec && left >= 32) {
      if constexpr (SRC == kBf16) {
        const u32x4_t* p = (const u32x4_t*)((const uint16_t*)a.x.X + t * a.x.ld + k0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const u32x4_t w = p[k];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[8 * k + 2 * j] = __uint_as_float(w[j] << 16);
            v[8 * k + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
          }
        }
      } else {
        const f32x4_t* p = (const f32x4_t*)((const float*)a.x.X + t * a.x.ld + k0);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const f32x4_t w = p[k];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * k + j] = w[j];
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        v[k] = 0.f;
        if (k < left) v[k] = SRC == kF32 ? ((const float*)a.x.X)[t * a.x.ld + k0 + k] : bf16_bits_to_f32(((const uint16_t*)a.x.X)[t * a.x.ld + k0 + k]);
      }
    }
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) m = max(m, f8_magnitude(v[k]));
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    const int b = f8_scale_byte<E5>(m);
    const float s = f8_inverse(b);
    i32x8_t q;
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k] = (int)f8_encode4<E5>(v[4 * k] * s, v[4 * k + 1] * s, v[4 * k + 2] * s, v[4 * k + 3] * s);
    *scale = b;
    return q;
  }
}

template <int MT, int SRC, bool E5, bool F32>
__global__ __launch_bounds__(1024) void f8_few(FewArgs a) {
  extern __shared__ float sums[];  // [waves][MT][64][4]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int br = blockIdx.x >> 3;
  const int n1 = a.w.ptr[br + 1];
  const uint8_t* wp = a.w.payload + ((blockIdx.x & 7) * 16 + r) * F8_BLOCK + g * 32;
  int64_t t[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t row = (int64_t)blockIdx.y * (16 * MT) + m * 16 + r;
    t[m] = row < a.T ? row : a.T - 1;  // rows past the last read the last one's bytes; their results go nowhere
  }
  f32x4_t acc[MT] = {};
  for (int n = a.w.ptr[br] + wave; n < n1; n += waves) {
    const int kb = a.w.idx[n], sw = a.w.scale[n];
    const i32x8_t w = *(const i32x8_t*)(wp + (int64_t)n * F8_BLOCK_BYTES);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      int sx;
      const i32x8_t x = few_input<SRC, E5>(a, t[m], kb, g, &sx);
      acc[m] = few_mfma<F32, E5>(w, sw, x, sx, acc[m]);
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) *(f32x4_t*)(sums + ((wave * MT + m) * 64 + lane) * 4) = acc[m];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 64; i += blockDim.x) {
    f32x4_t s = *(const f32x4_t*)(sums + i * 4);
    for (int w = 1; w < waves; ++w) s += *(const f32x4_t*)(sums + (w * MT * 64 + i) * 4);
    const int64_t row = (int64_t)blockIdx.y * (16 * MT) + (i >> 6) * 16 + (i & 15);
    const int o = blockIdx.x * 16 + ((i >> 4) & 3) * 4;
    if (row < a.T && o < a.w.out) f8_store4<F32>(a.q, row, o, a.w.out, s[0], s[1], s[2], s[3]);
  }
}

template <int MT, int SRC, bool E5>
int launch(const FewArgs& a, bool f32, hipStream_t st) {
  const int strips = (a.w.out + 15) / 16;
  const int per_row = (int)(a.w.nnzb / f8_blocks(a.w.out)) + 1;
  int waves = 1;
  while (waves < 16 && waves < per_row) waves *= 2;
  const dim3 grid((unsigned)strips, (unsigned)((a.T + 16 * MT - 1) / (16 * MT))), block((unsigned)(64 * waves));
  const size_t lds = (size_t)waves * MT * 1024;
  if (f32) hipLaunchKernelGGL((f8_few<MT, SRC, E5, true>), grid, block, lds, st, a);
  else hipLaunchKernelGGL((f8_few<MT, SRC, E5, false>), grid, block, lds, st, a);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}

template <bool E5>
int launch_rows(const FewArgs& a, bool f32, hipStream_t st) {
  if (a.x.dtype == BSP_BF16) return launch<1, kBf16, E5>(a, f32, st);
  if (a.x.dtype == BSP_F32) return launch<1, kF32, E5>(a, f32, st);
  if (a.T <= 16) return launch<1, kCodes, E5>(a, f32, st);
  if (a.T <= 32) return launch<2, kCodes, E5>(a, f32, st);
  return launch<4, kCodes, E5>(a, f32, st);
}

}  // namespace

int f8_launch_few(const F8Rows& w, const F8Input& x, int T, const F8Epilogue& q, bool f32, hipStream_t st) {
  FewArgs a{w, x, q, f8_scale_rows(T), T, 0};
  a.xvec = ((reinterpret_cast<uintptr_t>(x.X) | (uintptr_t)(x.ld * (x.dtype == BSP_F32 ? 4 : 2))) & 15u) == 0;
  return x.e5 ? launch_rows<true>(a, f32, st) : launch_rows<false>(a, f32, st);
}
