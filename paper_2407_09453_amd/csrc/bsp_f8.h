// 8-bit floating-point codes with power-of-two scales: the rule, and what the kernels on them share.
//
// A block is 128 columns of a row (activations) or 128 x 128 entries (weights).  With a = m 2^E (1 <= m < 2) the largest
// finite magnitude in it, its exponent is e = E - 8 (e4m3, whose largest value is 1.75 2^8) or E - 15 (e5m2: 1.75 2^15),
// one more where m > 1.75, and its codes are x 2^-e rounded to nearest, ties to even: the smallest power of two under
// which nothing saturates.  e is held in a byte as e + 127, the form in which the matrix cores take a scale, so a scale
// costs the product nothing, and code x 2^e is exact in bf16.
#ifndef BSP_F8_H
#define BSP_F8_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bsp.h"
#include "bsp_device.h"

typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef const __attribute__((address_space(1))) void* f8_gptr_t;
typedef __attribute__((address_space(3))) void* f8_lptr_t;

enum { F8_BLOCK = 128, F8_BLOCK_BYTES = F8_BLOCK * F8_BLOCK };

__host__ __device__ inline int f8_blocks(int n) { return (n + F8_BLOCK - 1) / F8_BLOCK; }
// rows of a scale array: one byte for each row of a column block, whole sixteens of them
__host__ __device__ inline int64_t f8_scale_rows(int T) { return ((int64_t)T + 15) & ~(int64_t)15; }

// A launch has fewer than 2^32 threads along x: workgroups past kGridX go along y, where workgroup x of row y is number y kGridX + x.
enum { kGridX = 1 << 21 };
inline dim3 f8_grid(int64_t groups) {
  return groups <= kGridX ? dim3((unsigned)groups) : dim3(kGridX, (unsigned)((groups + kGridX - 1) / kGridX));
}
// whether so many workgroups along x can be launched
inline bool f8_fits_x(int64_t groups, int threads) { return groups * threads <= (int64_t)UINT32_MAX; }

// Exchanges between neighbouring lanes without LDS: the lane whose number differs in bit 0, in bit 1; the mirrored lane of eight, of
// sixteen; the lane 16 away in a pair of rows, 32 away.
enum { kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140 };
template <int CTRL>
__device__ __forceinline__ uint32_t f8_from_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
// the largest of eight or sixteen lanes, in each of them
template <int LANES>
__device__ __forceinline__ uint32_t f8_most(uint32_t m) {
  m = max(m, f8_from_lane<kXor1>(m));
  m = max(m, f8_from_lane<kXor2>(m));
  m = max(m, f8_from_lane<kMirror8>(m));
  if constexpr (LANES == 16) m = max(m, f8_from_lane<kMirror16>(m));
  return m;
}
// the sum of a row of sixteen lanes, of a wave, in every lane of it
__device__ __forceinline__ float f8_row16_sum(float v) {
  v += __uint_as_float(f8_from_lane<kXor1>(__float_as_uint(v)));
  v += __uint_as_float(f8_from_lane<kXor2>(__float_as_uint(v)));
  v += __uint_as_float(f8_from_lane<kMirror8>(__float_as_uint(v)));
  return v + __uint_as_float(f8_from_lane<kMirror16>(__float_as_uint(v)));
}
__device__ __forceinline__ float f8_wave_sum(float v) {
  v = f8_row16_sum(v);
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// |x| as an ordered integer, 0 for infinities and NaN (they do not take part in a block's scale)
__device__ __forceinline__ uint32_t f8_magnitude(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}

// the scale byte e + 127 of a block whose largest magnitude has the bits `a`; E5: e5m2
template <bool E5>
__device__ __forceinline__ int f8_scale_byte(uint32_t a) {
  if (a == 0) return 127;
  const int e = (int)(a >> 23) - (E5 ? 15 : 8) + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0 : e;  // (a subnormal's field is 0, so it too ends at 2^-127)
}
// 2^-e as a float, for scale byte b <= 247
__device__ __forceinline__ float f8_inverse(int b) { return __uint_as_float((uint32_t)(254 - b) << 23); }
// 2^e as a float
__device__ __forceinline__ float f8_power(int b) { return __uint_as_float(b ? (uint32_t)b << 23 : 0x00400000u); }

// four values to four codes
template <bool E5>
__device__ __forceinline__ uint32_t f8_encode4(float a, float b, float c, float d) {
  int v = 0;
  if constexpr (E5) {
    v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
  } else {
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  }
  return (uint32_t)v;
}

// two codes (low or high half of v) times 2^e as a bf16 pair; scale = byte << 23 (the instruction reads the exponent alone)
template <bool E5, bool HIGH>
__device__ __forceinline__ uint32_t f8_decode_bf16x2(uint32_t v, float scale) {
  if constexpr (E5) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v, scale, HIGH));
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, HIGH));
}
// eight codes (two words) times 2^e as eight bf16
template <bool E5>
__device__ __forceinline__ u32x4_t f8_decode_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  return u32x4_t{f8_decode_bf16x2<E5, false>(lo, scale), f8_decode_bf16x2<E5, true>(lo, scale),
                 f8_decode_bf16x2<E5, false>(hi, scale), f8_decode_bf16x2<E5, true>(hi, scale)};
}

__device__ __forceinline__ uint32_t f8_pack_bf16x2(float a, float b) {
  const bf16x2_t v = {(__bf16)a, (__bf16)b};  // v_cvt_pk_bf16_f32: to nearest, ties to even
  return __builtin_bit_cast(uint32_t, v);
}

// Eight values of a row of n >= 8, from column c, at any address that suits their type: one or two loads with no branch.  At the row's end
// they are its last eight; f8_unpack8 moves them down by the `past` of them that lie before c, and fills up with zeros.
template <bool F32>
struct F8Raw8 {
  u32x4_t v[F32 ? 2 : 1];
};
typedef u32x4_t __attribute__((aligned(2))) f8_any2_t;
typedef u32x4_t __attribute__((aligned(4))) f8_any4_t;
template <bool F32>
__device__ __forceinline__ F8Raw8<F32> f8_raw8(const void* row, int c, int n) {
  const int at = c + 8 <= n ? c : n - 8;
  F8Raw8<F32> r;
  if constexpr (F32) {
    const f8_any4_t* p = (const f8_any4_t*)((const float*)row + at);
    r.v[0] = p[0];
    r.v[1] = p[1];
  } else {
    r.v[0] = *(const f8_any2_t*)((const uint16_t*)row + at);
  }
  return r;
}
__device__ __forceinline__ int f8_past(int c, int n) { return c + 8 <= n ? 0 : c < n ? c + 8 - n : 8; }
// `ragged`: n is no multiple of eight (the same in all lanes)
template <bool F32>
__device__ __forceinline__ void f8_unpack8(const F8Raw8<F32>& r, int past, bool ragged, float* v) {
  if constexpr (F32) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(r.v[k >> 2][k & 3]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(r.v[0][k] << 16);
      v[2 * k + 1] = __uint_as_float(r.v[0][k] & 0xFFFF0000u);
    }
  }
  if (ragged) {
#pragma unroll
    for (int d = 1; d < 8; d *= 2)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float up = k + d < 8 ? v[k + d < 8 ? k + d : 7] : 0.f;
        v[k] = past & d ? up : v[k];
      }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = past == 8 ? 0.f : v[k];
}
// the first `left` of eight values to a row, at any address that suits their type
template <bool F32>
__device__ __forceinline__ void f8_store8(void* row, int c, int left, const float* v) {
  if constexpr (F32) {
    float* y = (float*)row + c;
    if (left >= 8) {
      ((f8_any4_t*)y)[0] = u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      ((f8_any4_t*)y)[1] = u32x4_t{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
      return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) y[k] = v[k];
  } else {
    uint16_t* y = (uint16_t*)row + c;
    const u32x4_t w = {f8_pack_bf16x2(v[0], v[1]), f8_pack_bf16x2(v[2], v[3]), f8_pack_bf16x2(v[4], v[5]), f8_pack_bf16x2(v[6], v[7])};
    if (left >= 8) {
      __builtin_nontemporal_store(w, (f8_any2_t*)y);
      return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) y[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
  }
}

// whether a code stands for a value above zero
__device__ __forceinline__ bool f8_positive(uint32_t code, int e5) { return code - 1u < (e5 ? 0x7Cu : 0x7Eu); }

// what follows a product: Y = act(sum + bias + residual) times the gate, one rounding to Y's type
struct F8Epilogue {
  void* Y;               // [T][O], rows contiguous
  const float* bias;     // [O] or null
  const void* residual;  // [T][O] of Y's type, or null
  const uint8_t* gate;   // codes [T][128 ceil(O / 128)], or null: a result is kept where its code stands for a value > 0
  int32_t relu, gate_e5;
};

// several elements at once at any element's address
typedef f32x4_t __attribute__((aligned(4))) f32x4_any;
typedef u32x2_t __attribute__((aligned(2))) u32x2_any;
typedef u32x4_t __attribute__((aligned(2))) u32x4_any;

// channels o .. o+3 (those below O) of row t
template <bool F32>
__device__ __forceinline__ void f8_store4(const F8Epilogue& q, int64_t t, int o, int O, float v0, float v1, float v2, float v3) {
  float v[4] = {v0, v1, v2, v3};
  const int n = O - o < 4 ? O - o : 4;
  const bool whole = n == 4;
  if (q.bias) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) v[k] += q.bias[o + k];
  }
  const int64_t at = t * O + o;
  if (q.residual) {
    if constexpr (F32) {
      const float* r = (const float*)q.residual + at;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) v[k] += r[k];
    } else {
      const uint16_t* r = (const uint16_t*)q.residual + at;
      if (whole) {
        const u32x2_t w = *(const u32x2_any*)r;
        v[0] += __uint_as_float(w.x << 16);
        v[1] += __uint_as_float(w.x & 0xFFFF0000u);
        v[2] += __uint_as_float(w.y << 16);
        v[3] += __uint_as_float(w.y & 0xFFFF0000u);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < n) v[k] += bf16_bits_to_f32(r[k]);
      }
    }
  }
  if (q.relu) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] < 0.f ? 0.f : v[k];  // (a NaN stays one)
  }
  if (q.gate) {  // o is a multiple of four and a gate row one of 128, so the word is there and aligned
    const uint32_t c = *(const uint32_t*)(q.gate + t * (int64_t)f8_blocks(O) * F8_BLOCK + o);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = f8_positive((c >> (8 * k)) & 0xFFu, q.gate_e5) ? v[k] : 0.f;
  }
  if constexpr (F32) {
    float* y = (float*)q.Y + at;
    if (whole) {
      *(f32x4_any*)y = f32x4_t{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) y[k] = v[k];
    }
  } else {
    uint16_t* y = (uint16_t*)q.Y + at;
    const u32x2_t w = {f8_pack_bf16x2(v[0], v[1]), f8_pack_bf16x2(v[2], v[3])};
    if (whole) {
      *(u32x2_any*)y = w;
    } else {
      const uint32_t h[2] = {w.x, w.y};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) y[k] = (uint16_t)(h[k >> 1] >> (16 * (k & 1)));
    }
  }
}

// ---------------------------------------------------------------- launchers (each returns a bsp_status)
struct F8Rows {       // one direction of a layer's weights: compressed block rows of 128 x 128 codes
  const int32_t *ptr, *idx;
  const uint8_t *payload, *scale;
  int32_t out, in;    // channels
  int64_t nnzb;
};
struct F8Input {      // rows to multiply: codes with their scales, or values brought to e4m3 codes on the way
  const void* X;
  const uint8_t* scale;  // null: X holds values
  int32_t dtype;      // of the rows as given: BSP_E4M3, BSP_E5M2, BSP_BF16, BSP_F32
  int32_t e5;         // the codes are e5m2
  int64_t ld;         // elements from row to row
};
// The rows of a batch by their adapters, as adapt_plan leaves them: adapter a has rows order[start[a]] .. order[start[a + 1] - 1], those behind
// have none.
struct F8Requests {
  int32_t *start, *which, *order;  // [N + 1], [T] (-1: none), [T]
  int32_t* tiles;                  // how many tiles have an adapter, how many there are, whether the adapters' rows are mixed, a word; then the tiles' records
};
struct F8Adapters {  // bf16, ranks padded to Rp with zeros, columns to whole blocks
  uint16_t *a, *a_t, *b, *b_t;  // [N][Rp Ip] by rank and by column, [N][Op Rp] by column and by rank, as adapt_set lays them out
  float* scale;
  int32_t N, R, I, O, Rp, Ip, Op;
};
// What is added to a product: B_a u_t for the adapter of row t.
struct F8Low {
  const int32_t* which;
  const float* u;        // [slices][T][rank]: u_t is the sum of the slices'
  const uint16_t* up;    // [N][128 ceil(out / 128) rank], by column
  int64_t step, u_step;  // elements of an adapter, of a slice
  int32_t rank;          // 0: nothing is added
  int32_t slices;
  // Where the adapters' rows are mixed many rows are multiplied in the order of their adapters: row i of these codes is row order[i], or null
  const int32_t *mixed, *order;
  const uint8_t *codes, *scale;
};
// Few rows: the contraction split over a workgroup's waves.  Rows given as values become codes in each workgroup's LDS, T <= 16 of them and
// no more than kFewStaged bytes.
enum { kFewStaged = 72 * 1024 };
inline int64_t f8_few_staged(int T, int K) { return (int64_t)T * (f8_blocks(K) * (F8_BLOCK + 1) + 16); }
// `part`, here and below: [split][T][4 ceil(out / 4)] floats where *_split says more than one, to be joined
int f8_few_split(const F8Rows& w, int T);
int f8_launch_few(const F8Rows& w, const F8Input& x, int T, const F8Low& low, const F8Epilogue& q, bool f32, float* part, hipStream_t st);
// many rows, codes only
int f8_tile_split(const F8Rows& w, int T, bool f32);
int f8_launch_tile(const F8Rows& w, const F8Input& x, int T, const F8Low& low, const F8Epilogue& q, bool f32, float* part, hipStream_t st);
int f8_launch_join(const float* part, int split, int T, int O, const F8Epilogue& q, bool f32, hipStream_t st);
int f8_launch_save(const void* X, int x_f32, int64_t ldx, int T, int K, bool e5, uint8_t* codes, uint8_t* scale, hipStream_t st);
int f8_launch_load(const uint8_t* codes, const uint8_t* scale, int T, int K, bool e5, void* Y, int y_f32, int64_t ldy, hipStream_t st);
int f8_launch_pack(const bsp_weights_f8* w, const void* W, int w_f32, int64_t ldw, hipStream_t st);
// weights' and bias's gradient: dW float [O][I], a kept block's entries or zeros; db float [O]; either may be null
struct F8GradArgs {
  const uint16_t* dY;   // bf16 [T][O]
  int64_t ldy;
  const uint8_t *codes, *scale;
  const int32_t *row_ptr, *col_idx;
  float *dW, *db;
  float *part, *part_db;  // split > 1: [split][nnzb][128][128] and [split][O]
  int32_t T, O, I, nbo, nbi, groups, e5, split;
  int64_t nnzb;
};
int f8_grad_split(int64_t nnzb, int T);              // into how many ranges of rows the sums are cut
int f8_launch_grad(const F8GradArgs& a, hipStream_t st);
// adapters: which rows are whose, an adapter's weights, u = s A x ([slices][T][Rp] fp32, rows without an adapter left as they were), gradients
int64_t f8_request_tiles(int T, int N);  // at most so many
int64_t f8_requests_bytes(int T, int N);
F8Requests f8_requests_of(const bsp_f8_requests* r);
F8Adapters f8_adapters_of(const bsp_f8_adapters* d);
int f8_launch_plan(const bsp_f8_requests* r, const void* which, bool wide, hipStream_t st);
int f8_launch_set(const F8Adapters& d, int slot, int rank, const void* A, int64_t lda, const void* B, int64_t ldb, bool f32, float scale, hipStream_t st);
int f8_down_slices(int T, int N, int K, bool grad);  // of u: up to eight for a product, two for the gradients
// codes, scale: where values are to become codes (of x.e5) on the way, too, or where codes go, mixed and `sorts`; or null.  sorts: mixed rows leave in
// the order of their adapters
int f8_launch_down(const F8Adapters& d, bool transposed, const F8Input& x, int T, const F8Requests& q, float* u, uint8_t* codes, uint8_t* scale, bool sorts, hipStream_t st);
// u of the layer's input and v of its result's gradient (bf16)
int f8_launch_down_both(const F8Adapters& d, const F8Input& x, const F8Input& dY, int T, const F8Requests& q, float* u, float* v, hipStream_t st);
int64_t f8_adapt_part_bytes(const F8Adapters& d, int T);
int f8_launch_adapt_grad(const F8Adapters& d, const uint16_t* dY, int64_t ldy, const F8Input& x, int T, const F8Requests& q, const float* u, const float* v,
                         float* part, float* dA, float* dB, hipStream_t st);
int norm_parts(int T, int D);                        // workgroups that share the rows of a column sum
int norm_launch_forward(const void* X, bool f32, int64_t ldx, int T, int D, const float* weight, const float* bias, float eps,
                        void* Y, int64_t ldy, int code, uint8_t* codes, uint8_t* scale, float* mean, float* rstd, hipStream_t st);
int norm_launch_backward(const void* dY, int64_t ld_dy, const void* X, int64_t ldx, bool f32, const float* mean, const float* rstd, const float* weight,
                         int T, int D, void* dX, int64_t ld_dx, float* dweight, float* dbias, float* part, hipStream_t st);
// out[c] = sum over p of part[p][c], in their order; columns from split_at on to out2; either may be null
int norm_launch_sum(const float* part, int parts, int64_t width, int64_t split_at, float* out, float* out2, hipStream_t st);
// root-mean-square norm: h = x + residual in their type, y = h rstd weight
int rms_launch_forward(const void* X, int64_t ldx, const void* residual, int64_t ldr, bool f32, int T, int D, const float* weight, float eps, void* H,
                       int64_t ldh, void* Y, int64_t ldy, int code, uint8_t* codes, uint8_t* scale, float* rstd, hipStream_t st);
int rms_parts(int T, int D);
int rms_launch_backward(const void* dY, int64_t ld_dy, const void* H, int64_t ldh, const void* dH, int64_t ld_dh, bool f32, const float* rstd,
                        const float* weight, int T, int D, void* dX, int64_t ld_dx, float* dweight, float* part, hipStream_t st);
// log probabilities, entropy and the k likeliest of rows of logits, and the logits' gradient; workspace: logp_workspace bytes
int64_t logp_workspace(int T, int V, int k);
int logp_launch(const void* X, bool f32, int64_t ld, int T, int V, const void* tokens, bool wide_tokens, float scale, int k, float* logp, float* lse,
                float* entropy, float* top, int32_t* ids, void* workspace, hipStream_t st);
int logp_launch_grad(const void* X, bool f32, int64_t ld, int T, int V, const void* tokens, bool wide_tokens, float scale, const float* lse, const float* entropy,
                     const float* dlogp, const float* dentropy, void* dX, int64_t ld_dx, hipStream_t st);

#endif
