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
// The k likeliest of a row: the k-th largest of 64 groups' maxima is at most the k-th largest value, so what lies below it is out (below its
// upper 16 bits, which is what is searched for); what is left, little more than k on logits in any order that is not made for it, goes to LDS,
// each wave's to a list of its own, and is ranked by counting.  Keys are the value's bits, ordered, and the complement of the
// index: all differ, and the lowest index wins a tie.  Where more is left than a list holds (a row of equal values) the k-th key is
// found bit by bit.
// Measured: 8192 x 32768 bf16 90 to 140 us after kernels that left 500 MB to be written back, 102 by itself (537 MB, 5.3 TB/s), 7 to join, the gradient
// 192, in the logits' place 186 (1.07 GB, 5.6 to 5.8 TB/s), of rows that it adds up anew 223 and 244; with the 1, 8, 20 and 50 likeliest 117, 127, 136, 190; 1021 x 50001
// with none 28, with 8 33.5 (102 MB, 3 TB/s: seven chunks a row are three and a half rounds of what the chip holds); vector instructions take nine tenths of
// the time, too; 1 x 131072 with 20 5.1 and 7.9 to join; 253 x 1000 fp32 with 5 5.3, gradient 3.7.
#include "bsp_norm.h"

#include <type_traits>

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
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
__device__ __forceinline__ void put_row(const LogpArgs& a, int64_t row, const Sums& v, float log, bool f32) {
  const int64_t token = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int32_t*)a.tokens)[row];
  const bool none = v.n == 0.f && v.s == 0.f;  // no token is left: every probability is zero
  float p = 0.f;
  if (token >= a.V) p = __builtin_nanf("");
  else if (token >= 0) p = none ? -INFINITY : (logit(a, row, token, f32) - v.m) * a.scale - log;
  a.logp[row] = p;
  a.lse[row] = none ? -INFINITY : v.m * a.scale + log;
  a.entropy[row] = none ? 0.f : log - v.q / (v.n + v.s);
}
__device__ __forceinline__ void put_top(const LogpArgs& a, int64_t row, int r, uint64_t key, const Sums& v, float log) {
  const bool none = v.n == 0.f && v.s == 0.f;
  a.top[row * a.k + r] = none ? -INFINITY : (value_of(key) - v.m) * a.scale - log;
  a.ids[row * a.k + r] = (int32_t)~(uint32_t)key;
}

// The k-th largest of 64 lanes' 16-bit numbers, bit by bit.
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t v, int k) {
  uint32_t kth = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t trial = kth | 1u << bit;
    if (__popcll(__ballot(v >= trial)) >= k) kth = trial;
  }
  return kth;
}
// lanes before this one in a mask
__device__ __forceinline__ int before(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// Eight logits of a row, as they lie in memory.
template <bool F32, bool SHORT>  // SHORT: the row may have fewer than eight
struct Eight {
  F8Raw8<F32> raw;
  __device__ __forceinline__ void ask(const void* row, int c, int n) {
    if (!SHORT || n >= 8) {
      raw = f8_raw8<F32>(row, c, n);
    } else {
      float v[8];
      each8<F32>(row, c, n, v);
      put(v);
    }
  }
  __device__ __forceinline__ void put(const float* v) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t u = __float_as_uint(v[k]);
      if constexpr (F32) raw.v[k >> 2][k & 3] = u;
      else raw.v[0][k >> 1] = k & 1 ? (raw.v[0][k >> 1] & 0xFFFFu) | (u & 0xFFFF0000u) : u >> 16;
    }
  }
  // at a row's end, once: into their places, minus infinity from `end` on (the chunk's: a multiple of eight, or n)
  __device__ __forceinline__ void place(int c, int n, int end) {
    const int past = c >= end ? 8 : !SHORT || n >= 8 ? f8_past(c, n) : 0;
    float v[8];
    f8_unpack8<F32>(raw, past, (n & 7) != 0 && (!SHORT || n >= 8), v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < end ? v[k] : -INFINITY;
    put(v);
  }
  __device__ __forceinline__ void get(float* v) {
    // (hidden from the optimiser, which would keep the unpacked values of one pass for the next)
#pragma unroll
    for (int k = 0; k < (F32 ? 2 : 1); ++k) asm volatile("" : "+v"(raw.v[k]));
    f8_unpack8<F32>(raw, 0, false, v);
  }
};
// (the builtin first makes every operand that it has not seen computed a canonical one, an instruction each)
__device__ __forceinline__ float most3(float a, float b, float c) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}
__device__ __forceinline__ float most8(const float* v) { return most3(most3(most3(v[0], v[1], v[2]), v[3], v[4]), most3(v[5], v[6], v[7]), v[0]); }

// ROWT threads hold a chunk of up to ROWT x NV x 8 logits.
// An exponent is one fused multiply-add, t = x c - r with r = m c rounded: the sums are then those relative to r, and the exact difference
// d = m c - r (one fused multiply-add again) brings them to m.  Nothing is done for single elements that a row in a thousand needs: where the
// sum is near 1, as a sure token makes it, or r is too large to be near m c, the workgroup adds once more what does not reach the maximum, relative to m itself.  (Minus infinities are not so rare: with
// a second pass where the sum of t e^t was no number 1021 masked rows of 50001 took 40 us instead of 33.5, and 8192 x 32768 without any
// 3 of 125 less.)
template <bool F32, bool TOP, int ROWT, int NV>
__global__ __launch_bounds__(ROWT, (F32 || TOP) && NV == 4 ? 4 : 8) void logp_rows(LogpArgs a) {
  constexpr int WAVES = ROWT / 64, LANES = ROWT / 64;  // waves; lanes of one of the 64 groups
  constexpr int kList = WAVES == 1 ? 256 : WAVES <= 8 ? 128 : kTopMost, kEights = WAVES == 1 ? 96 : kList / 2;  // keys of a wave; eights that may hold some
  __shared__ float sh_max[WAVES], sh_sum[2][WAVES][3];
  __shared__ float sh_group[TOP ? 64 : 1], sh_least, sh_log;
  __shared__ uint32_t sh_count[WAVES], sh_above;
  __shared__ uint64_t sh_key[TOP ? WAVES : 1][kList];
  __shared__ F8Raw8<F32> sh_eight[TOP ? WAVES : 1][kEights];
  __shared__ int sh_column[TOP ? WAVES : 1][kEights];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = a.chunks == 1 ? group : group / a.chunks;
  if (row >= a.T) return;
  const int chunk = (int)(group - row * a.chunks), begin = chunk * a.chunk, end = begin + a.chunk < a.V ? begin + a.chunk : a.V;
  const void* x = row_of<F32>(a.X, row, a.ld);
  Eight<F32, ROWT == 64 && NV == 1> in[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) in[j].ask(x, begin + (tid + j * ROWT) * 8, a.V);
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (begin + (wave * 64 + 63 + j * ROWT) * 8 + 8 > end) in[j].place(begin + (tid + j * ROWT) * 8, a.V, end);
  // f(the eight values of group j, their first column), group by group: registers are what lets two workgroups share a CU
  auto each = [&](int j, auto f) {
    float v[8];
    in[j].get(v);
    int c = tid * 8;
    asm volatile("" : "+v"(c));  // (a place of its own for every column it would keep, too)
    f(v, c + begin + j * ROWT * 8);
    __builtin_amdgcn_sched_barrier(0);
  };
  float m = -INFINITY, most[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    each(j, [&](const float* v, int) { most[j] = most8(v); });
    m = fmaxf(m, most[j]);
  }
  if constexpr (TOP) {
    const float g = lanes_max<LANES>(m);
    if (tid % LANES == 0) sh_group[tid / LANES] = g;
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
      const uint32_t kth = kth_of_lanes((uint32_t)(key_of(sh_group[lane], 0) >> 48), a.k);
      if (lane == 0) sh_least = kth <= 0x7Fu ? -INFINITY : value_of((uint64_t)kth << 48);
    }
  }
  const float from = m == -INFINITY ? 0.f : m, c2 = a.scale * kLog2e, r = from * c2, d = fmaf(from, c2, -r);
  float s = 0.f, q = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    each(j, [&](const float* v, int) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float t = fmaf(v[k], c2, -r), e = __builtin_amdgcn_exp2f(t);
        s += e;
        q = fmaf(fmaxf(t, -200.f), e, q);  // (of -200 and less e is 0; 0 times minus infinity would be no number)
      }
    });
  // the workgroup's sums, in the order of its waves
  auto total = [&](float (*sh)[3], float n, float s, float q) {
    s = f8_wave_sum(s);
    q = f8_wave_sum(q);
    if constexpr (WAVES == 1) return Sums{from, n, s, q};
    if (lane == 0) sh[wave][0] = n, sh[wave][1] = s, sh[wave][2] = q;
    __syncthreads();
    Sums v{from, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v.n += sh[w][0], v.s += sh[w][1], v.q += sh[w][2];
    return v;
  };
  Sums sum = total(sh_sum[0], 0.f, s, q);
  // r is up to half its last place off, of 2^22 a quarter; of 2^31 it is 128, and neither the sums nor what brings them to m are numbers
  if (sum.s < 1.5f || !(fabsf(r) < 0x1p22f)) {
    uint32_t n = 0;
    s = q = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      each(j, [&](const float* v, int) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float t = (v[k] - from) * c2;
          t = t < -200.f ? -200.f : t;
          n += __popcll(__ballot(t == 0.f));
          const float e = t == 0.f ? 0.f : __builtin_amdgcn_exp2f(t);
          s += e;
          q = fmaf(t, e, q);
        }
      });
    sum = total(sh_sum[1], (float)n, s, q);
  } else {
    const float f = __builtin_amdgcn_exp2f(-d);
    sum.q = (sum.q - d * sum.s) * f;
    sum.s *= f;
  }
  sum.q *= kLn2;
  if (m == -INFINITY && sum.s == 0.f) sum = Sums{-INFINITY, 0.f, 0.f, 0.f};
  if (tid == 0) {
    if (a.chunks == 1) {
      const float log = log_of(sum);
      if constexpr (TOP) sh_log = log;
      put_row(a, row, sum, log, F32);
    } else {
      *(f32x4_t*)(a.part + (row * a.chunks + chunk) * 4) = f32x4_t{sum.m, sum.n, sum.s, sum.q};
    }
  }
  if constexpr (TOP) {
    if constexpr (WAVES == 1) __syncthreads();
    const float least = sh_least;
    uint32_t mine = 0;  // keys of this wave, which its list may have no room for
    // A maximum passes over NaN, and minus infinity is what stands past the row: then every group is looked into.  Where fewer than k groups
    // hold more than minus infinity, its lowest places that can be wanted are among the first k.
    const bool careful = sum.s != sum.s || least == -INFINITY;
    auto keep = [&](auto wanted) {
      mine = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        each(j, [&](const float* v, int c) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const bool is = !(v[k] < least) && wanted(v[k], c + k);
            const uint64_t those = __ballot(is);
            if (!those) continue;
            const uint32_t at = mine + before(those);
            if (is && at < kList) sh_key[wave][at] = key_of(v[k], c + k);
            mine += __popcll(those);
          }
        });
      }
      if (lane == 0) sh_count[wave] = mine;
      __syncthreads();
    };
    int eights = 0;
    if (!careful) {
      // Eights with a key among them go to LDS whole, a few of a hundred, and are looked through there, one value a lane: looked
      // through in their registers, for all lanes' sake, they take four times the instructions.
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bool is = !(most[j] < least);
        const uint64_t those = __ballot(is);
        if (!those) continue;
        const int at = eights + before(those);
        if (is && at < kEights) sh_eight[wave][at] = in[j].raw, sh_column[wave][at] = begin + (tid + j * ROWT) * 8;
        eights += __popcll(those);
      }
      __builtin_amdgcn_wave_barrier();  // (a wave's own; its accesses to LDS are in order)
      for (int i0 = 0; i0 < (eights < kEights ? eights : kEights) * 8; i0 += 64) {
        const int i = i0 + lane, at = i >> 3 < eights ? i >> 3 : 0;
        const uint32_t* words = (const uint32_t*)&sh_eight[wave][at];
        const float v = __uint_as_float(F32 ? words[i & 7] : i & 1 ? words[(i & 7) >> 1] & 0xFFFF0000u : words[(i & 7) >> 1] << 16);
        const bool is = i >> 3 < eights && !(v < least);
        const uint64_t those = __ballot(is);
        const uint32_t to = mine + before(those);
        if (is && to < kList) sh_key[wave][to] = key_of(v, sh_column[wave][at] + (i & 7));
        mine += __popcll(those);
      }
      if (lane == 0) sh_count[wave] = eights > kEights ? kList + 1 : mine;
      __syncthreads();
    } else {
      keep([&](float v, int c) { return c < end && (v != -INFINITY || c < begin + a.k); });
    }
    bool over = false;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) over |= sh_count[w] > kList;
    if (over) {  // the k-th largest key, from its highest bit down
      uint64_t kth = 0;
      for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = kth | 1ull << bit;
        uint32_t above = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
          each(j, [&](const float* v, int c) {
#pragma unroll
            for (int k = 0; k < 8; ++k) above += __popcll(__ballot(c + k < end && key_of(v[k], c + k) >= trial));
          });
        __syncthreads();  // the last counts have been read
        if (tid == 0) sh_above = 0;
        __syncthreads();
        if (lane == 0) atomicAdd(&sh_above, above);
        __syncthreads();
        if (sh_above >= (uint32_t)a.k) kth = trial;
      }
      keep([&](float v, int c) { return c < end && key_of(v, c) >= kth; });
    }
    const float log = sh_log;
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += sh_count[w];
    auto put = [&](int rank, uint64_t key) {
      if (rank >= a.k) return;
      if (a.chunks == 1) put_top(a, row, rank, key, sum, log);
      else a.keys[(row * a.chunks + chunk) * a.k + rank] = key;
    };
    if (total <= 64) {  // as good as always: one wave, a key a lane
      if (wave == 0) {
        uint32_t w = 0, i = lane;
        for (; w + 1 < WAVES && i >= sh_count[w]; ++w) i -= sh_count[w];
        const uint64_t key = lane < (int)total ? sh_key[w][i] : 0;
        int rank = 0;
        for (uint32_t j = 0; j < total; ++j)
          rank += ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)key, j)) > key;
        if (lane < (int)total) put(rank, key);
      }
      mine = 0;
    }
    for (uint32_t i = lane; i < mine; i += 64) {
      const uint64_t key = sh_key[wave][i];
      int rank = 0;
      for (int w = 0; w < WAVES; ++w) {
        const uint32_t n = sh_count[w];
#pragma unroll 4
        for (uint32_t j = 0; j < n; ++j) rank += sh_key[w][j] > key;
      }
      put(rank, key);
    }
    if (a.chunks > 1)  // a chunk of fewer than k
      for (int r = end - begin + tid; r < a.k; r += ROWT) a.keys[(row * a.chunks + chunk) * a.k + r] = 0;
  }
}

// A row's chunks joined: one wave a row, four rows a workgroup; with TOP one, and LDS for all of the chunks' keys.
template <bool F32, bool TOP>
__global__ __launch_bounds__(TOP ? 64 : 256) void logp_join(LogpArgs a) {
  extern __shared__ uint64_t sh_key[];
  const int lane = threadIdx.x & 63;
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = TOP ? group : group * 4 + (threadIdx.x >> 6);
  if (row >= a.T) return;  // (whole waves)
  f32x4_t v = {-INFINITY, 0.f, 0.f, 0.f};
  if (lane < a.chunks) v = *(const f32x4_t*)(a.part + (row * a.chunks + lane) * 4);
  const float m = lanes_max<64>(v[0]), from = m == -INFINITY ? 0.f : m;
  const float d = v[0] == from ? 0.f : (v[0] - from) * a.scale, e = v[0] == -INFINITY ? 0.f : expf(d);
  // what reached a lower chunk's maximum is one of the others here
  const float all = v[1] + v[2], n = d == 0.f ? v[1] : 0.f, s = d == 0.f ? v[2] : e * all, q = d == 0.f ? v[3] : e == 0.f ? e * all : e * (v[3] + d * all);
  const Sums sum{m, f8_wave_sum(n), f8_wave_sum(s), f8_wave_sum(q)};
  const float log = log_of(sum);
  if (lane == 0) put_row(a, row, sum, log, F32);
  if constexpr (TOP) {
    const uint64_t* keys = a.keys + row * a.chunks * a.k;
    const int total = a.chunks * a.k;
    // 64 keys' turn after turn, four turns' keys asked for together: a loop of ballots is not unrolled, and each would wait for its own
    auto turns = [&](auto at_once, auto f) {
      constexpr int kAtOnce = decltype(at_once)::value;
      for (int i0 = 0; i0 < total; i0 += 64 * kAtOnce) {
        uint64_t key[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
          const int i = i0 + e * 64 + lane;
          key[e] = keys[i < total ? i : total - 1];
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) f(i0 + e * 64 + lane < total ? key[e] : 0);
      }
    };
    auto all = [&](auto f) {
      if (total <= 64) turns(std::integral_constant<int, 1>{}, f);
      else turns(std::integral_constant<int, 4>{}, f);
    };
    uint64_t most = 0;
    all([&](uint64_t key) { most = most > key ? most : key; });
    const uint64_t least = (uint64_t)kth_of_lanes((uint32_t)(most >> 48), a.k) << 48;
    int have = 0;
    all([&](uint64_t key) {
      const bool is = key && key >= least;
      const uint64_t those = __ballot(is);
      if (is) sh_key[have + before(those)] = key;
      have += __popcll(those);
    });
    __syncthreads();
    for (int i = lane; i < have; i += 64) {
      const uint64_t mine = sh_key[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < have; ++j) rank += sh_key[j] > mine;
      if (rank < a.k) put_top(a, row, rank, mine, sum, log);
    }
  }
}

struct LogpGradArgs {
  const void *X, *tokens;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dX;
  int64_t ld, ld_dx;
  int32_t T, V, shares, alone, wide_tokens;  // workgroups of a long row; whether one of them does all of a row that is added up anew
  float scale;
};

// Whether lse, in its 32 bits, still holds the log of the sum for a gradient in bf16: a probability from it is up to U |lse| of itself off (U = 2^-24),
// at most 2^-18, and what the likeliest leaves, 1 - p >= entropy / 25, up to 25 U |lse| / entropy, at most 2^-11: a quarter of what the result's
// rounding takes.  (At a scale of 10^4 a probability would be 10^-2 of itself off, at 10^6 anything.)
__device__ __forceinline__ bool lse_holds(float lse, float entropy) { return fabsf(lse) <= fminf(64.f, 256.f * entropy); }

// p = e^(z-m) / S.  A row's workgroup forms m, n and s anew, as above but with a running maximum for each wave, and takes 1 - p of the likeliest from what does not
// reach the maximum; only where lse holds enough for results in bf16 it is e^(z-lse).  A row of up to ROWT NV 8 logits stays in registers; a longer one
// is shared out among workgroups, each of which adds up all of it where it has to be, or the first does all (many rows, or the gradient takes
// the logits' place), reading the row twice, the second time from the last-level cache.  What is added up is read before any gradient is written,
// and a thread that writes has itself read what stood there.
template <bool F32, int ROWT, int NV, bool LONG>
__global__ __launch_bounds__(ROWT, F32 && NV >= 4 ? 4 : LONG ? 6 : 8) void logp_grad(LogpGradArgs a) {
  constexpr int WAVES = ROWT / 64, kTurn = ROWT * NV * 8;
  __shared__ float sh[WAVES][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t group = (int64_t)blockIdx.y * kGridX + blockIdx.x, row = LONG ? group / a.shares : group;
  if (row >= a.T) return;
  const int share = LONG ? (int)(group - row * a.shares) : 0;
  const void* x = row_of<F32>(a.X, row, a.ld);
  const int64_t token = a.wide_tokens ? ((const int64_t*)a.tokens)[row] : (int64_t)((const int32_t*)a.tokens)[row];
  const float lse = a.lse[row], entropy = a.entropy[row], dh = a.dentropy ? a.dentropy[row] * a.scale : 0.f;
  const float dl = a.dlogp && token >= 0 ? a.dlogp[row] * a.scale : 0.f;
  const bool anew = F32 || !lse_holds(lse, entropy);
  if (LONG && anew && a.alone && share != (int)((row + row / 8) % a.shares)) return;  // (which goes by the row, for the XCDs' sake)
  Eight<F32, ROWT == 64 && NV == 1> in[NV];
  auto ask = [&](int begin) {
#pragma unroll
    for (int j = 0; j < NV; ++j) in[j].ask(x, begin + (tid + j * ROWT) * 8, a.V);
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (begin + (wave * 64 + 63 + j * ROWT) * 8 + 8 > a.V) in[j].place(begin + (tid + j * ROWT) * 8, a.V, a.V);
  };
  if (!LONG) ask(0);
  // log2 of p S: (factor z - minus) by_log2
  float factor = a.scale, minus = lse, by_log2 = kLog2e, top = __builtin_nanf(""), inv = 1.f, log = 0.f, rest = 0.f;
  bool none = false;
  if (anew) {
    const float c2 = a.scale * kLog2e;
    float m = -INFINITY, n = 0.f, s = 0.f;  // the wave's maximum, a lane's sums
    for (int begin = 0; begin < (LONG ? a.V : 1); begin += kTurn) {
      if (LONG) ask(begin);
      float most[NV], now = -INFINITY;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float v[8];
        in[j].get(v);
        most[j] = most8(v);
        now = fmaxf(now, most[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
      now = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(lanes_max<64>(now))));
      if (now > m) {
        if (LONG) s = (s + n) * __builtin_amdgcn_exp2f((m - now) * c2), n = 0.f;
        m = now;
      }
      const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float v[8];
        in[j].get(v);
        if (__any(most[j] == from)) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float e = __builtin_amdgcn_exp2f((v[k] - from) * c2);
            n += v[k] == from ? 1.f : 0.f;
            s += v[k] == from ? 0.f : e;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) s += __builtin_amdgcn_exp2f((v[k] - from) * c2);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    n = f8_wave_sum(n);
    s = f8_wave_sum(s);
    if constexpr (WAVES > 1) {
      if (lane == 0) sh[wave][0] = m, sh[wave][1] = n, sh[wave][2] = s;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh[w][0]);
      n = s = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {  // (what reached a lower maximum is one of the others)
        const bool same = sh[w][0] == m;
        n += same ? sh[w][1] : 0.f;
        s += same ? sh[w][2] : __builtin_amdgcn_exp2f((sh[w][0] - m) * c2) * (sh[w][1] + sh[w][2]);
      }
    }
    none = n == 0.f && s == 0.f;
    factor = 1.f, minus = top = m == -INFINITY ? 0.f : m, by_log2 = c2, inv = 1.f / (n + s), rest = n - 1.f + s, log = log_of(Sums{m, n, s, 0.f});
  }
  // -(log p + entropy) dentropy / S = t h1 + h0
  float h1 = 0.f - dh * kLn2 * inv, h0 = 0.f - dh * (entropy - log) * inv, l0 = h0 - dl * inv;
  if (token >= a.V) l0 = __builtin_nanf("");  // (as the log probability)
  if (none) h0 = h1 = l0 = 0.f;
  const int at = token >= 0 && token < a.V && !none ? (int)token : -8;
  void* y = (void*)row_of<F32>(a.dX, row, a.ld_dx);
  const bool all = LONG && anew && a.alone;
  for (int begin = all ? 0 : share * kTurn; begin < a.V; begin += kTurn) {
    if constexpr (LONG) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = begin + (tid + j * ROWT) * 8;
        if (c + 8 <= a.V) in[j].raw = f8_raw8<F32>(x, c, a.V);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = begin + (tid + j * ROWT) * 8;
      if (c >= a.V) continue;
      float v[8], g[8];
      if (!LONG || c + 8 <= a.V) in[j].get(v);
      else each8<F32>(x, c, a.V, v);  // a row's end by itself: its last eight would be another thread's too
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float t = fmaxf(fmaf(v[k], factor, -minus) * by_log2, -200.f);  // (of -200 and less e is 0; 0 times minus infinity would be no number)
        g[k] = __builtin_amdgcn_exp2f(t) * fmaf(t, h1, l0);
      }
      if (at >= c && at < c + 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float t = fmaxf(fmaf(v[k], factor, -minus) * by_log2, -200.f), e = __builtin_amdgcn_exp2f(t);
          if (c + k == at) g[k] = fmaf(dl, v[k] == top ? rest * inv : 1.f - e * inv, e * fmaf(t, h1, h0));
        }
      }
      f8_store8<F32>(y, c, a.V - c, g);
    }
    if (!all) break;
  }
}

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }

// Chunks of a row and their length.  Four waves and 8192 logits a chunk leave a CU several workgroups that wait for memory and add up in turn (us, chunks of
// 8192, 16384 and 32768: 8192 x 32768 bf16 106, 115, 127, with the 20 likeliest 157, 171, 274; 2048 x 131072 with them 142, 158, 268);
// shorter ones where rows are too few for the chip.
struct Cut {
  int chunk, chunks;
};
Cut cut_of(int T, int V) {
  int most = 8192;
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
  if (TOP) hipLaunchKernelGGL((logp_join<F32, TOP>), f8_grid(a.T), dim3(64), (size_t)a.chunks * a.k * 8, st, a);
  else hipLaunchKernelGGL((logp_join<F32, TOP>), f8_grid(((int64_t)a.T + 3) / 4), dim3(256), 0, st, a);
  return launched();
}

template <bool F32>
int grad(LogpGradArgs& a, hipStream_t st) {
  // Long rows of bf16 come in shares of 256 threads, which is what those want that lse holds: 2048 x 131072 190, in shares of 1024
  // threads 306, 8192 x 32768 192 and 186 in the logits' place, held in 1024 threads' registers 213 and 202 (added up 223 and 244, held 210 and 200).  fp32,
  // always added up, is held longer and comes in shares of 1024: 2048 x 32768 108, 1024 x 131072 283, in shares of 256 364.  One workgroup does all
  // of a row as soon as there are about 1024 (us): 16 x 131072 bf16 43, shared out 20, 64 x 131072 45 and 45.
  constexpr int kHeld = F32 ? 32768 : 16384, kThreads = F32 ? 1024 : 256, kShare = kThreads * 8 * 4;
  if (a.V > kHeld) {
    a.shares = (a.V + kShare - 1) / kShare;
    a.alone = a.X == a.dX || (int64_t)a.T * a.shares >= 1024;
  }
  const dim3 grid = f8_grid((int64_t)a.T * a.shares);
  if (a.V <= 512) hipLaunchKernelGGL((logp_grad<F32, 64, 1, false>), grid, dim3(64), 0, st, a);
  else if (a.V <= 1024) hipLaunchKernelGGL((logp_grad<F32, 64, 2, false>), grid, dim3(64), 0, st, a);
  else if (a.V <= 2048) hipLaunchKernelGGL((logp_grad<F32, 256, 1, false>), grid, dim3(256), 0, st, a);
  else if (a.V <= 4096) hipLaunchKernelGGL((logp_grad<F32, 256, 2, false>), grid, dim3(256), 0, st, a);
  else if (a.V <= 8192) hipLaunchKernelGGL((logp_grad<F32, 256, 4, false>), grid, dim3(256), 0, st, a);
  else if (a.V <= 16384) hipLaunchKernelGGL((logp_grad<F32, 512, 4, false>), grid, dim3(512), 0, st, a);
  else if (F32 && a.V <= kHeld) hipLaunchKernelGGL((logp_grad<true, 512, 8, false>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((logp_grad<F32, kThreads, 4, true>), grid, dim3(kThreads), 0, st, a);
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
  LogpGradArgs a{X, tokens, lse, entropy, dlogp, dentropy, dX, ld, ld_dx, T, V, 1, 0, wide_tokens, scale};
  return f32 ? grad<true>(a, st) : grad<false>(a, st);
}
