// FC layers on few rows, weights in 8-bit codes: Y = X W^t, bound by the bytes of the weights (serving), or by latency.
//
// A workgroup owns 16 output channels and 16 MT rows; its waves share out the kept blocks of the channels' block row, each
// adding its blocks' products in its own accumulators, and the waves' sums meet in LDS: the long axis is split inside the
// workgroup.  Only where that leaves many CUs without one (few channels, a long contraction: f8_few_split) are there shares of the block
// columns too, whose sums a second launch joins.  Operands go from memory to registers, up to kAhead blocks at a time: a lane's 32
// bytes of a weight row are pieces g and 4 + g of sixteen, so that a request covers whole
// 64-byte halves of sixteen lines that follow one another, and a block's lines are each asked for once in the chip.
// The loop asks kAhead blocks ahead where a wave has 2 kAhead of them or more.  With fewer, as on 16 x 25088 -> 4096 half kept (six or seven a
// wave, 16.6 us, 3.2 TB/s), latency is paid several times: the rows of each block are asked for behind a wait for the number of its column, with
// the weights of the block before already waited for, and the tail waits for each block that it asks for at once.
// Up to 16 rows given as bf16 or fp32, in whole aligned pieces of 16 bytes, become codes in LDS first, in every workgroup for itself, while the
// first weights are on their way: less than a launch of its own takes
// (us, 1 x 4096 -> 4096: 5.8 to 6.2, with rows that are codes 5.4; 1 x 25088 -> 4096, half of the blocks kept, 13.4; 1 x 4096 -> 16384 14.6 to 15.1, 4.5 TB/s).
#include "bsp_f8.h"

namespace {

struct FewArgs {
  F8Rows w;
  F8Input x;
  F8Epilogue q;
  int64_t srows;   // rows of x.scale
  int32_t T, rows;  // rows: how many become codes in LDS
  int32_t full;    // blocks in a block row, where all are kept; else 0
  int32_t split;
  float* part;     // split > 1: sums of each share of the block columns, as f8_join reads them
  F8Low low;
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

// A workgroup's rows as codes in LDS: [row][Kp + 16] (sixteen rows' same piece then lies in different banks), behind them the scales [row][blocks].
// Eight lanes take a block of a row, sixteen values each; a row ends between two pieces of 16 bytes, those past it are zeros.
template <int SRC, bool E5>
__device__ __forceinline__ void few_stage(const FewArgs& a, uint8_t* codes, uint8_t* scale, int64_t t0, int rows) {
  constexpr int kBytes = SRC == kBf16 ? 2 : 4, kPieces = kBytes;
  const int nb = f8_blocks(a.w.in), per_row = nb * 8;
  for (int i = threadIdx.x; i < rows * per_row; i += blockDim.x) {  // (whole groups of eight lanes)
    const int row = i / per_row, k0 = (i - row * per_row) * 16;
    const uint8_t* p = (const uint8_t*)a.x.X + ((t0 + row) * a.x.ld + k0) * kBytes;
    float v[16];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const bool in = k0 + k * (16 / kBytes) < a.w.in;
      u32x4_t w = *(const u32x4_t*)(in ? p + k * 16 : (const uint8_t*)a.x.X);
      w = in ? w : u32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 16 / kBytes; ++e)
        v[k * (16 / kBytes) + e] = __uint_as_float(SRC == kF32 ? w[e & 3] : e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, f8_magnitude(v[k]));
    m = f8_most<8>(m);
    const int b = f8_scale_byte<E5>(m);
    const float s = f8_inverse(b);
    u32x4_t q;
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = f8_encode4<E5>(v[4 * k] * s, v[4 * k + 1] * s, v[4 * k + 2] * s, v[4 * k + 3] * s);
    *(u32x4_t*)(codes + row * (nb * F8_BLOCK + 16) + k0) = q;
    if ((k0 & 127) == 0) scale[row * nb + (k0 >> 7)] = (uint8_t)b;
  }
}

// Waves a workgroup may have: sixteen leave each 128 registers, eight 256.
template <int MT>
constexpr int kMostWaves = MT == 1 ? 16 : 8;

// four channels' share of a row's adapter: fp32 products of u with bf16 weights, while the wave's first blocks are on their way (1 x 4096 -> 4096 of rank 16
// 6.3 us without, 7.7 with)
__device__ __forceinline__ f32x4_t few_low(const F8Low& low, int64_t row, int o) {
  f32x4_t s = {};
  const int of = low.which[row];
  if (of < 0) return s;
  // (channels are padded to whole blocks; 32 channels, sixteen ranks, 64 lanes of eight)
  const uint16_t* b = low.up + of * low.step + (int64_t)(o & ~31) * low.rank + (o & 31) * 8;
  const float* u = low.u + row * low.rank;
#pragma unroll 1
  for (int r = 0; r < low.rank; r += 8) {
    f32x4_t u0 = *(const f32x4_t*)(u + r), u1 = *(const f32x4_t*)(u + r + 4);
#pragma unroll 3
    for (int k = 1; k < low.slices; ++k) {
      u0 += *(const f32x4_t*)(u + k * low.u_step + r);
      u1 += *(const f32x4_t*)(u + k * low.u_step + r + 4);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const u32x4_t w = *(const u32x4_t*)(b + ((r >> 4) * 64 + ((r >> 3) & 1) * 32 + c) * 8);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[c] += __uint_as_float(w[e] << 16) * (e < 2 ? u0 : u1)[2 * (e & 1)] + __uint_as_float(w[e] & 0xFFFF0000u) * (e < 2 ? u0 : u1)[2 * (e & 1) + 1];
    }
  }
  return s;
}

// LOW: with adapters beside the layer.
template <int MT, int SRC, bool E5, bool F32, bool LOW>
__device__ __forceinline__ void few(const FewArgs& a, float* sums) {  // sums: [waves][MT][64][4], behind them the rows' codes
  constexpr int kAhead = MT == 1 && F32 ? 3 : 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int br = blockIdx.x >> 3;
  // (where all blocks are kept their places need not be read)
  const auto* ptr = (const __attribute__((address_space(4))) int32_t*)a.w.ptr;
  const int row0 = a.full ? br * a.full : ptr[br];
  const int row_cnt = a.full ? a.full : ptr[br + 1] - row0;
  const int first = (int)((int64_t)row_cnt * blockIdx.z / a.split), n0 = row0 + first;
  const int cnt = (int)((int64_t)row_cnt * (blockIdx.z + 1) / a.split) - first;
  const int mine = cnt > wave ? (cnt - wave + waves - 1) / waves : 0;
  const uint8_t* wp = a.w.payload + (int64_t)n0 * F8_BLOCK_BYTES + ((blockIdx.x & 7) * 16 + r) * F8_BLOCK + g * 16;
  const int64_t t0 = (int64_t)blockIdx.y * (16 * MT);
  // rows past the last: the last one's bytes, their results go nowhere
  const uint8_t *xp[MT], *xs[MT];
  const int nb = f8_blocks(a.w.in);
  uint8_t *staged = (uint8_t*)(sums + waves * MT * 256), *staged_scale = staged + a.rows * (nb * F8_BLOCK + 16);
  int64_t scale_step;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t row = t0 + m * 16 + r < a.T ? t0 + m * 16 + r : a.T - 1;
    if constexpr (SRC == kCodes) {
      xp[m] = (const uint8_t*)a.x.X + row * a.x.ld + g * 16;
      xs[m] = a.x.scale + row;
      scale_step = a.srows;
    } else {
      xp[m] = staged + (int)(row - t0) * (nb * F8_BLOCK + 16) + g * 16;
      xs[m] = staged_scale + (int)(row - t0) * nb;
      scale_step = 1;
    }
  }
  u32x4_t w[kAhead][2], x[kAhead][MT][2];
  int ws[kAhead], col[kAhead], sx[kAhead][MT];
  f32x4_t acc[MT] = {};
  f32x4_t low[LOW ? MT : 1];  // the first wave's, for the results that it puts out below
  for (int c = 0; c < mine || c == 0; c += 64) {  // the wave's block columns, 64 at a time, one a lane
    const int of = wave + (c + lane) * waves < cnt ? wave + (c + lane) * waves : cnt - 1;
    const int cols = a.full ? first + of : cnt > 0 ? a.w.idx[n0 + of] : 0;
    const int end = mine - c < 64 ? mine - c : 64;
    auto rows = [&](int j) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        x[j][m][0] = *(const u32x4_t*)(xp[m] + (int64_t)col[j] * F8_BLOCK);
        x[j][m][1] = *(const u32x4_t*)(xp[m] + (int64_t)col[j] * F8_BLOCK + 64);
        sx[j][m] = xs[m][col[j] * scale_step];
      }
    };
    auto load = [&](int s, int j) {
      const int n = wave + (c + s) * waves;
      const u32x4_t* p = (const u32x4_t*)(wp + (int64_t)n * F8_BLOCK_BYTES);
      w[j][0] = p[0];
      w[j][1] = p[4];
      ws[j] = a.w.scale[n0 + n];
      col[j] = __builtin_amdgcn_readlane(cols, s);
      if constexpr (SRC == kCodes) rows(j);
    };
    auto multiply = [&](int j) {
      if constexpr (SRC != kCodes) rows(j);
      const i32x8_t wv = {(int)w[j][0].x, (int)w[j][0].y, (int)w[j][0].z, (int)w[j][0].w, (int)w[j][1].x, (int)w[j][1].y, (int)w[j][1].z, (int)w[j][1].w};
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const i32x8_t xv = {(int)x[j][m][0].x, (int)x[j][m][0].y, (int)x[j][m][0].z, (int)x[j][m][0].w, (int)x[j][m][1].x, (int)x[j][m][1].y, (int)x[j][m][1].z, (int)x[j][m][1].w};
        acc[m] = few_mfma<F32, E5>(wv, ws[j], xv, sx[j][m], acc[m]);
      }
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (j < end) load(j, j);
    if constexpr (SRC != kCodes) {
      if (c == 0) {  // the first weights are on their way
        few_stage<SRC, E5>(a, staged, staged_scale, t0, a.rows);
        __syncthreads();
      }
    }
    if constexpr (LOW) {
      if (c == 0 && wave == 0 && blockIdx.z == 0) {  // (likewise)
#pragma unroll
        for (int m = 0; m < MT; ++m) low[m] = few_low(a.low, t0 + m * 16 + r < a.T ? t0 + m * 16 + r : a.T - 1, blockIdx.x * 16 + g * 4);
      }
    }
    int s = 0;
    for (; s + 2 * kAhead <= end; s += kAhead)
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        multiply(j);
        load(s + kAhead + j, j);
      }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (s + j < end) {
        multiply(j);
        if (s + kAhead + j < end) load(s + kAhead + j, j);
      }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (s + kAhead + j < end) multiply(j);
  }
  if constexpr (LOW) {
    if (wave == 0 && blockIdx.z == 0)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m] += low[m];
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) *(f32x4_t*)(sums + ((wave * MT + m) * 64 + lane) * 4) = acc[m];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 64; i += blockDim.x) {
    f32x4_t s = *(const f32x4_t*)(sums + i * 4);
    for (int w = 1; w < waves; ++w) s += *(const f32x4_t*)(sums + (w * MT * 64 + i) * 4);
    const int64_t row = t0 + (i >> 6) * 16 + (i & 15);
    const int o = blockIdx.x * 16 + ((i >> 4) & 3) * 4;
    if (row >= a.T || o >= a.w.out) continue;
    if (a.split > 1) *(f32x4_t*)(a.part + (((int64_t)blockIdx.z * a.T + row) * ((a.w.out + 3) >> 2) + (o >> 2)) * 4) = s;
    else f8_store4<F32>(a.q, row, o, a.w.out, s[0], s[1], s[2], s[3]);
  }
}

template <int MT, int SRC, bool E5, bool F32>
__global__ __launch_bounds__((64 * kMostWaves<MT>)) void f8_few(FewArgs a) {
  extern __shared__ float sums[];
  kernarg_touch<FewArgs>();
  few<MT, SRC, E5, F32, false>(a, sums);
}
template <int MT, int SRC, bool E5, bool F32>
__global__ __launch_bounds__((64 * kMostWaves<MT>)) void f8_few_low(FewArgs a) {
  extern __shared__ float sums[];
  kernarg_touch<FewArgs>();
  few<MT, SRC, E5, F32, true>(a, sums);
}

template <int MT, int SRC, bool E5, bool F32, bool LOW>
int launch(FewArgs a, hipStream_t st) {
  constexpr auto kernel = LOW ? &f8_few_low<MT, SRC, E5, F32> : &f8_few<MT, SRC, E5, F32>;
  const int strips = (a.w.out + 15) / 16, tiles = (a.T + 16 * MT - 1) / (16 * MT);
  const int64_t per_row = (a.w.nnzb + (int64_t)f8_blocks(a.w.out) * a.split - 1) / ((int64_t)f8_blocks(a.w.out) * a.split);
  // as many waves as a CU holds, on every CU; a wave for every block is enough
  constexpr int most = kMostWaves<MT>;
  int waves = 1;
  while (waves < most && waves < per_row && (waves < 2 || (int64_t)strips * tiles * a.split * waves < 256 * most)) waves *= 2;
  int lds = waves * MT * 1024;
  if constexpr (SRC != kCodes) {
    a.rows = a.T;
    lds += (f8_few_staged(a.T, a.w.in) + 15) & ~15;
    static const bool raised = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kFewStaged + 16 * 1024 + 16) == hipSuccess;
    if (!raised) return BSP_ERR_HIP;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)strips, (unsigned)tiles, (unsigned)a.split), dim3((unsigned)(64 * waves)), (size_t)lds, st, a);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}

template <bool E5, bool F32, bool LOW>
int launch_rows(const FewArgs& a, hipStream_t st) {
  if (a.x.dtype == BSP_BF16) return launch<1, kBf16, E5, F32, LOW>(a, st);
  if (a.x.dtype == BSP_F32) return launch<1, kF32, E5, F32, LOW>(a, st);
  if (a.T <= 16) return launch<1, kCodes, E5, F32, LOW>(a, st);
  return launch<2, kCodes, E5, F32, LOW>(a, st);
}
template <bool LOW>
int launch_any(const FewArgs& a, bool f32, hipStream_t st) {
  if (f32) return a.x.e5 ? launch_rows<true, true, LOW>(a, st) : launch_rows<false, true, LOW>(a, st);
  return a.x.e5 ? launch_rows<true, false, LOW>(a, st) : launch_rows<false, false, LOW>(a, st);
}

}  // namespace

// Where a workgroup's sixteen waves would each have six blocks or more and many CUs have none, shares of two blocks a wave whose sums a second launch joins.
int f8_few_split(const F8Rows& w, int T) {
  const int64_t groups = (int64_t)((w.out + 15) / 16) * ((T + 31) / 32), row = w.nnzb / f8_blocks(w.out);
  int split = 1;
  if (row >= 6 * 16)
    while (groups * split * 2 <= 256 && row >= 2 * 16 * split * 2) split *= 2;
  return split;
}

int f8_launch_few(const F8Rows& w, const F8Input& x, int T, const F8Low& low, const F8Epilogue& q, bool f32, float* part, hipStream_t st) {
  FewArgs a{w, x, q, f8_scale_rows(T), T, 0, 0, f8_few_split(w, T), part, low};
  if (w.nnzb == (int64_t)f8_blocks(w.out) * f8_blocks(w.in)) a.full = f8_blocks(w.in);
  return low.rank ? launch_any<true>(a, f32, st) : launch_any<false>(a, f32, st);
}
