// Log probabilities of given tokens, the entropy and the likeliest tokens from logits, and the gradient of the logits, bound by memory.
//
//   z = scale x, m = max z, n = how many reach it, s = sum of the others' e^(z-m), S = n + s, q = sum (z-m) e^(z-m)
//   lse = m + log S, log p = z - lse, entropy = log S - q / S
//   dx = scale (dlogp ([token] - p) - dentropy p (log p + entropy))
//
// A row is read once and stays in the registers of the 64 to 1024 threads that own it, so its maximum is known before the first
// exponential.  What does not reach the maximum is summed by itself: for a sure token S is 1 + s with s far below a unit in the last place of 1,
// and log S = log1p(s), its log probability and the entropy keep all their bits.  Long rows, and rows of a few tokens' batch, are cut
// into chunks whose (m, n, s, q) and likeliest a second launch joins, in their order.
//
// The k likeliest of a row: the k-th largest of 64 groups' maxima is at most the k-th largest value, so what lies below it is out; what is left,
// little more than k on logits in any order that is not made for it, goes to LDS and is ranked by counting.  Keys are the value's bits,
// ordered, and the complement of the index: all differ, and the lowest index wins a tie.  Where more is left than LDS holds (a row of
// equal values) the k-th key is found bit by bit.
#include "bsp_norm.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kKeys = 512;     // keys kept for ranking
constexpr int kChunksMost = 64, kTopMost = 64;

struct LogpArgs {
  const void* X;
  const void* tokens;  // int32 or int64
  int64_t ld;
  float *logp, *lse, *entropy, *top;
  int32_t* ids;
  float* part;         // [T][chunks][4]
  uint64_t* keys;      // [T][chunks][k]
  int32_t T, V, k, chunk, chunks, wide_tokens;
  float scale;
};

__device__ __forceinline__ float from_lane_max(float v, uint32_t other) { return fmaxf(v, __uint_as_float(other)); }
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {  // of 1, 4, 8, 16 or 64 neighbouring lanes, in each of them
  if constexpr (LANES >= 4) {
    v = from_lane_max(v, f8_from_lane<kXor1>(__float_as_uint(v)));
    v = from_lane_max(v, f8_from_lane<kXor2>(__float_as_uint(v)));
  }
  if constexpr (LANES >= 8) v = from_lane_max(v, f8_from_lane<kMirror8>(__float_as_uint(v)));
  if constexpr (LANES >= 16) v = from_lane_max(v, f8_from_lane<kMirror16>(__float_as_uint(v)));
  if constexpr (LANES == 64) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  }
  return v;
}

// A value and its place as one number: larger values first, the lower index where values are equal (0 and -0 are), NaN before all.
// 0 is no key of a value.
__device__ __forceinline__ uint64_t key_of(float x, int i) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 becomes 0)
  const uint32_t k = x != x ? 0xFFFFFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)k << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t k = (uint32_t)(key >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

struct Sums {  // of a chunk or a row
  float m, n, s, q;
};
// log of the sum, minus the largest
__device__ __forceinline__ float log_of(const Sums& v) { return v.n == 1.f ? log1pf(v.s) : logf(v.n + v.s); }

__device__ __forceinline__ float logit(const LogpArgs& a, int64_t row, int64_t i, bool f32) {
  return f32 ? ((const float*)a.X)[row * a.ld + i] : bf16_bits_to_f32(((const uint16_t*)a.X)[row * a.ld + i]);
}

// a row's three results: one thread
__device__ __forceinline__ void put_row(const LogpArgs& a, int64_t row, const Sums& v, bool f32) {
  const int64_t token = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int32_t*)a.tokens)[row];
  const bool none = v.n == 0.f && v.s == 0.f;  // no token is left: every probability is zero
  const float log = log_of(v);
  float p = 0.f;
  if (token >= a.V) p = __builtin_nanf("");
  else if (token >= 0) p = none ? -INFINITY : (logit(a, row, token, f32) - v.m) * a.scale - log;
  a.logp[row] = p;
  a.lse[row] = none ? -INFINITY : v.m * a.scale + log;
  a.entropy[row] = none ? 0.f : log - v.q / (v.n + v.s);
}
__device__ __forceinline__ void put_top(const LogpArgs& a, int64_t row, int r, uint64_t key, const Sums& v) {
  const bool none = v.n == 0.f && v.s == 0.f;
  a.top[row * a.k + r] = none ? -INFINITY : (value_of(key) - v.m) * a.scale - log_of(v);
  a.ids[row * a.k + r] = (int32_t)~(uint32_t)key;
}

// The place of the k-th largest of 64 lanes' values among them (equal ones by their lane): the lane whose rank is k - 1 has it.
template <class V>
__device__ __forceinline__ int lane_rank(V v, int lane) {
  int rank = 0;
  for (int j = 0; j < 64; ++j) {
    V o;
    if constexpr (sizeof(V) == 8) {
      o = (V)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, j);
    } else {
      o = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), j));
    }
    rank += o > v || (o == v && j < lane);
  }
  return rank;
}

// eight logits of a row from column c, minus infinity where none is
template <bool F32>
struct Eight {
  F8Raw8<F32> raw;
  __device__ __forceinline__ void ask(const void* row, int c, int n) {
    if (n >= 8) {
      raw = f8_raw8<F32>(row, c, n);
    } else {
      float v[8];
      each8<F32>(row, c, n, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (F32) raw.v[k >> 2][k & 3] = __float_as_uint(v[k]);
        else raw.v[0][k >> 1] = (k & 1 ? raw.v[0][k >> 1] & 0xFFFFu : 0u) | (k & 1 ? __float_as_uint(v[k]) & 0xFFFF0000u : __float_as_uint(v[k]) >> 16);
      }
    }
  }
  // end: the chunk's (a multiple of eight, or n)
  __device__ __forceinline__ void get(int c, int n, int end, float* v) const {
    const int past = c >= end ? 8 : n >= 8 ? f8_past(c, n) : 0;
    f8_unpack8<F32>(raw, past, (n & 7) != 0 && n >= 8, v);
    if (c + 8 > end) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c + k < end ? v[k] : -INFINITY;
    }
  }
};

// ROWT threads hold a chunk of up to ROWT x NV x 8 logits.
template <bool F32, bool TOP, int ROWT, int NV>
__global__ __launch_bounds__(ROWT) void logp_rows(LogpArgs a) {
  constexpr int WAVES = ROWT / 64, LANES = ROWT / 64;  // waves; lanes of one of the 64 groups
  __shared__ float sh_max[WAVES], sh_sum[WAVES][3];
  __shared__ float sh_group[TOP ? 64 : 1], sh_least;
  __shared__ uint32_t sh_count[2];
  __shared__ uint64_t sh_key[TOP ? kKeys : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = a.chunks == 1 ? group : group / a.chunks;
  if (row >= a.T) return;
  const int chunk = (int)(group - row * a.chunks), begin = chunk * a.chunk, end = begin + a.chunk < a.V ? begin + a.chunk : a.V;
  const void* x = row_of<F32>(a.X, row, a.ld);
  Eight<F32> in[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) in[j].ask(x, begin + (tid + j * ROWT) * 8, a.V);
  float m = -INFINITY, v[8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    in[j].get(begin + (tid + j * ROWT) * 8, a.V, end, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, v[k]);
  }
  if constexpr (TOP) {
    const float g = lanes_max<LANES>(m);
    if (tid % LANES == 0) sh_group[tid / LANES] = g;
    if (tid < 2) sh_count[tid] = 0;
  }
  m = lanes_max<64>(m);
  if constexpr (WAVES > 1) {
    if (lane == 0) sh_max[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh_max[w]);
  } else if constexpr (TOP) {
    __syncthreads();
  }
  if constexpr (TOP) {
    if (wave == 0) {
      const float g = sh_group[lane];
      if (lane_rank(g, lane) == a.k - 1) sh_least = g;
    }
  }
  // exponentials
  const float from = m == -INFINITY ? 0.f : m, c2 = a.scale * kLog2e;
  float s = 0.f, q = 0.f;
  uint32_t n = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    in[j].get(begin + (tid + j * ROWT) * 8, a.V, end, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float t = (v[k] - from) * c2;
      t = t < -200.f ? -200.f : t;  // 2^-200 is 0, and 0 times it too; a NaN stays one
      const bool most = t == 0.f;
      n += __popcll(__ballot(most));
      const float e = most ? 0.f : __builtin_amdgcn_exp2f(t);
      s += e;
      q += t * e;
    }
  }
  s = f8_wave_sum(s);
  q = f8_wave_sum(q);
  Sums sum{from, (float)n, s, q};
  if constexpr (WAVES > 1) {
    if (lane == 0) sh_sum[wave][0] = sum.n, sh_sum[wave][1] = s, sh_sum[wave][2] = q;
    __syncthreads();
    sum = Sums{from, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum.n += sh_sum[w][0], sum.s += sh_sum[w][1], sum.q += sh_sum[w][2];
  } else if constexpr (TOP) {
    __syncthreads();
  }
  sum.q *= kLn2;
  if (m == -INFINITY && sum.s == 0.f) sum = Sums{-INFINITY, 0.f, 0.f, 0.f};
  if (tid == 0) {
    if (a.chunks == 1) put_row(a, row, sum, F32);
    else *(f32x4_t*)(a.part + (row * a.chunks + chunk) * 4) = f32x4_t{sum.m, sum.n, sum.s, sum.q};
  }
  if constexpr (TOP) {
    const float least = sh_least;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = begin + (tid + j * ROWT) * 8;
      in[j].get(c, a.V, end, v);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (!(v[k] < least) && c + k < end) {
          const uint32_t at = atomicAdd(&sh_count[0], 1u);
          if (at < kKeys) sh_key[at] = key_of(v[k], c + k);
        }
    }
    __syncthreads();
    uint32_t have = sh_count[0];
    if (have > kKeys) {  // the k-th largest key, from its highest bit down
      uint64_t kth = 0;
      for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = kth | 1ull << bit;
        uint32_t above = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = begin + (tid + j * ROWT) * 8;
          in[j].get(c, a.V, end, v);
#pragma unroll
          for (int k = 0; k < 8; ++k) above += __popcll(__ballot(c + k < end && key_of(v[k], c + k) >= trial));
        }
        __syncthreads();  // the last count has been read
        if (tid == 0) sh_count[1] = 0;
        __syncthreads();
        if (lane == 0) atomicAdd(&sh_count[1], above);
        __syncthreads();
        if (sh_count[1] >= (uint32_t)a.k) kth = trial;
      }
      if (tid == 0) sh_count[0] = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = begin + (tid + j * ROWT) * 8;
        in[j].get(c, a.V, end, v);
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < end && key_of(v[k], c + k) >= kth) {
            const uint32_t at = atomicAdd(&sh_count[0], 1u);
            if (at < kKeys) sh_key[at] = key_of(v[k], c + k);
          }
      }
      __syncthreads();
      have = sh_count[0];
    }
    for (uint32_t i = tid; i < have; i += ROWT) {
      const uint64_t mine = sh_key[i];
      int rank = 0;
      for (uint32_t j = 0; j < have; ++j) rank += sh_key[j] > mine;
      if (rank >= a.k) continue;
      if (a.chunks == 1) put_top(a, row, rank, mine, sum);
      else a.keys[(row * a.chunks + chunk) * a.k + rank] = mine;
    }
    if (a.chunks > 1)  // a chunk of fewer than k
      for (int r = have + tid; r < a.k; r += ROWT) a.keys[(row * a.chunks + chunk) * a.k + r] = 0;
  }
}

// A row's chunks joined: one wave a row for the sums; for the likeliest a workgroup of four.
template <bool F32, bool TOP>
__global__ __launch_bounds__(256) void logp_join(LogpArgs a) {
  __shared__ float sh[5];
  __shared__ uint64_t sh_group[TOP ? 64 : 1], sh_least, sh_key[TOP ? kChunksMost * kTopMost : 1];
  __shared__ uint32_t sh_count;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = TOP ? group : group * 4 + (tid >> 6);
  if (row >= a.T) return;  // (whole waves, and with TOP the whole workgroup)
  Sums sum{};
  if (!TOP || tid < 64) {
    f32x4_t v = {-INFINITY, 0.f, 0.f, 0.f};
    if (lane < a.chunks) v = *(const f32x4_t*)(a.part + (row * a.chunks + lane) * 4);
    const float m = lanes_max<64>(v[0]), from = m == -INFINITY ? 0.f : m;
    const float d = v[0] == from ? 0.f : (v[0] - from) * a.scale, e = v[0] == -INFINITY ? 0.f : expf(d);
    // what reached a lower chunk's maximum is one of the others here
    const float all = v[1] + v[2], n = d == 0.f ? v[1] : 0.f, s = d == 0.f ? v[2] : e * all, q = d == 0.f ? v[3] : e == 0.f ? e * all : e * (v[3] + d * all);
    sum = Sums{m, f8_wave_sum(n), f8_wave_sum(s), f8_wave_sum(q)};
    if (lane == 0) put_row(a, row, sum, F32);
    if constexpr (TOP) {
      if (lane == 0) sh[0] = sum.m, sh[1] = sum.n, sh[2] = sum.s, sh[3] = sum.q, sh_count = 0;
    }
  }
  if constexpr (TOP) {
    // keys in 64 groups of every 64th
    const uint64_t* keys = a.keys + row * a.chunks * a.k;
    const int total = a.chunks * a.k;
    uint64_t most = 0;
    if (tid < 64)
      for (int i = tid; i < total; i += 64) most = most > keys[i] ? most : keys[i];
    if (tid < 64 && lane_rank(most, lane) == a.k - 1) sh_least = most;
    __syncthreads();
    sum = Sums{sh[0], sh[1], sh[2], sh[3]};
    const uint64_t least = sh_least;
    for (int i = tid; i < total; i += 256) {
      const uint64_t key = keys[i];
      if (key && key >= least) sh_key[atomicAdd(&sh_count, 1u)] = key;
    }
    __syncthreads();
    const uint32_t have = sh_count;
    for (uint32_t i = tid; i < have; i += 256) {
      const uint64_t mine = sh_key[i];
      int rank = 0;
      for (uint32_t j = 0; j < have; ++j) rank += sh_key[j] > mine;
      if (rank < a.k) put_top(a, row, rank, mine, sum);
    }
  }
}

struct LogpGradArgs {
  const void *X, *tokens;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dX;
  int64_t ld, ld_dx;
  int32_t T, V, chunks, wide_tokens;
  float scale;
};

// A thread takes NV groups of eight columns, and reads them before it writes any: the gradient may replace the logits.
template <bool F32, int NV>
__global__ __launch_bounds__(256) void logp_grad(LogpGradArgs a) {
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = group / a.chunks;
  if (row >= a.T) return;
  const int begin = (int)(group - row * a.chunks) * (256 * 8 * NV);
  const int64_t token = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int32_t*)a.tokens)[row];
  const float lse = a.lse[row], h = a.entropy[row];
  const float dl = token >= 0 && a.dlogp ? a.dlogp[row] * a.scale : 0.f, dh = a.dentropy ? a.dentropy[row] * a.scale : 0.f;
  const float bad = token >= a.V ? __builtin_nanf("") : 0.f;  // (as the log probability)
  const void* x = row_of<F32>(a.X, row, a.ld);
  void* y = (void*)row_of<F32>(a.dX, row, a.ld_dx);
  F8Raw8<F32> raw[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = begin + (threadIdx.x + j * 256) * 8;
    if (c + 8 <= a.V) raw[j] = f8_raw8<F32>(x, c, a.V);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = begin + (threadIdx.x + j * 256) * 8;
    if (c >= a.V) continue;
    float v[8];
    if (c + 8 <= a.V) f8_unpack8<F32>(raw[j], 0, false, v);
    else each8<F32>(x, c, a.V, v);  // a row's end by itself: its last eight would be another thread's too
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float lp = v[k] * a.scale - lse;
      lp = lp < -200.f ? -200.f : lp;  // no probability, and nothing times minus infinity
      const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
      float g = -p * (dl + dh * (lp + h)) + bad;
      if (c + k == token) g += dl;
      v[k] = lse == -INFINITY ? 0.f : g;
    }
    f8_store8<F32>(y, c, a.V - c, v);
  }
}

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }

// Chunks of a row and their length.
struct Cut {
  int chunk, chunks;
};
Cut cut_of(int T, int V) {
  int most = 32768;
  while (most > 2048 && (int64_t)T * ((V + most - 1) / most) < 512) most /= 2;
  while ((V + most - 1) / most > kChunksMost) most *= 2;
  const int chunks = (V + most - 1) / most;
  const int chunk = chunks == 1 ? (V + 7) / 8 * 8 : ((V + chunks - 1) / chunks + 7) / 8 * 8;
  return Cut{chunk, (V + chunk - 1) / chunk};
}

template <bool F32, bool TOP>
int rows(const LogpArgs& a, hipStream_t st) {
  const dim3 grid = f8_grid((int64_t)a.T * a.chunks);
  if (a.chunk <= 512) hipLaunchKernelGGL((logp_rows<F32, TOP, 64, 1>), grid, dim3(64), 0, st, a);
  else if (a.chunk <= 1024) hipLaunchKernelGGL((logp_rows<F32, TOP, 64, 2>), grid, dim3(64), 0, st, a);
  else if (a.chunk <= 2048) hipLaunchKernelGGL((logp_rows<F32, TOP, 256, 1>), grid, dim3(256), 0, st, a);
  else if (a.chunk <= 4096) hipLaunchKernelGGL((logp_rows<F32, TOP, 256, 2>), grid, dim3(256), 0, st, a);
  else if (a.chunk <= 8192) hipLaunchKernelGGL((logp_rows<F32, TOP, 256, 4>), grid, dim3(256), 0, st, a);
  else if (a.chunk <= 16384) hipLaunchKernelGGL((logp_rows<F32, TOP, 512, 4>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((logp_rows<F32, TOP, 1024, 4>), grid, dim3(1024), 0, st, a);
  if (launched() != BSP_OK) return BSP_ERR_HIP;
  if (a.chunks == 1) return BSP_OK;
  hipLaunchKernelGGL((logp_join<F32, TOP>), f8_grid(TOP ? (int64_t)a.T : ((int64_t)a.T + 3) / 4), dim3(256), 0, st, a);
  return launched();
}

}  // namespace

int64_t logp_workspace(int T, int V, int k) {
  const Cut c = cut_of(T, V);
  return c.chunks == 1 ? 0 : (int64_t)T * c.chunks * (16 + 8 * (int64_t)k);
}

int logp_launch(const void* X, bool f32, int64_t ld, int T, int V, const void* tokens, bool wide_tokens, float scale, int k, float* logp, float* lse,
                float* entropy, float* top, int32_t* ids, void* workspace, hipStream_t st) {
  const Cut c = cut_of(T, V);
  LogpArgs a{};
  a.X = X, a.tokens = tokens, a.ld = ld, a.logp = logp, a.lse = lse, a.entropy = entropy, a.top = top, a.ids = ids;
  a.part = (float*)workspace, a.keys = (uint64_t*)((uint8_t*)workspace + (int64_t)T * c.chunks * 16);
  a.T = T, a.V = V, a.k = k, a.chunk = c.chunk, a.chunks = c.chunks, a.wide_tokens = wide_tokens, a.scale = scale;
  if (k) return f32 ? rows<true, true>(a, st) : rows<false, true>(a, st);
  return f32 ? rows<true, false>(a, st) : rows<false, false>(a, st);
}

int logp_launch_grad(const void* X, bool f32, int64_t ld, int T, int V, const void* tokens, bool wide_tokens, float scale, const float* lse, const float* entropy,
                     const float* dlogp, const float* dentropy, void* dX, int64_t ld_dx, hipStream_t st) {
  LogpGradArgs a{X, tokens, lse, entropy, dlogp, dentropy, dX, ld, ld_dx, T, V, 0, wide_tokens, scale};
  auto run = [&](auto kernel, int nv) {
    a.chunks = (V + 256 * 8 * nv - 1) / (256 * 8 * nv);
    hipLaunchKernelGGL(kernel, f8_grid((int64_t)T * a.chunks), dim3(256), 0, st, a);
    return launched();
  };
  if (V <= 2048) return f32 ? run(logp_grad<true, 1>, 1) : run(logp_grad<false, 1>, 1);
  return f32 ? run(logp_grad<true, 2>, 2) : run(logp_grad<false, 4>, 4);
}
