// Low-rank adapters of many requests beside an 8-bit layer: y_t += s_a B_a (A_a x_t) for the adapter a of row t, and their gradients.
//
//   down:  u_t = s_a A_a x_t                     here, on rows sorted by adapter, up to 64 of one adapter to a workgroup
//   up:    y_t += B_a u_t                        in the products' own kernels, before their epilogue: one rounding for the whole result
//   grad:  dB_a = sum_t dy_t u_t^t, dA_a = sum_t v_t x_t^t with v_t = s_a B_a^t dy_t (down, transposed)
//
// A and B are held as bf16, in both directions, ranks padded to 16, 32, 64 or 128 with zeros; products are summed in fp32.  u and v are fp32, and
// where they enter a matrix instruction again they do so as bf16 parts: as two, which keep 16 bits, for results in bf16, as three, which keep all,
// for gradients and fp32 results.  Rows enter as they were given: bf16 values and codes are exact in bf16, fp32 values go as three parts.
// `down` is bound by the bytes of the rows on many rows, by latency on few.  `grad` reads each block of 128 columns of the rows of an adapter
// once: both operands are summed over rows, so they lie in LDS as in memory and the transposing read hands a lane a column's
// rows.  An adapter with many rows is cut into chunks whose sums a second launch joins, in order: no atomics.
// Measured: A x of 16384 x 4096 codes, rank 16 18 to 20 us (3.5 TB/s), rank 32 22.6, of 8192 x 16384 bf16, rank 32 52 to 62 (4.3 to 5.1 TB/s), with the rows' codes on
// the way 101 to 118 (403 MB, 3.4 to 4.0 TB/s; of rank 16 87, of rank 64 117: a workgroup's rows read the adapters' columns again), of one row of 4096 4.4; grad of 8192 rows, 4096 codes and 16384 bf16, rank 32 80 to 91 (302 MB, 3.3 to 3.8 TB/s)
// and 4 to 9 to join; 37 rows of 1000 and 520 columns 5.4 for u and v, 6.4 for the gradients.  The plan of 64 rows 5 to 9 us, of 8192 28, of 16384 50.
#include "bsp_norm.h"

#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
constexpr int kTileRows = 64, kTileWords = 4 + kTileRows;  // a tile's record: adapter (-1: none), rows, place of the first in the order, a word, the rows' numbers (past the last: its)

inline int launched() { return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP; }

// ------------------------------------------------------------------ which rows are whose
// Rows sorted by adapter, in their order within each, those of none last (counted, not compared: one workgroup of sixteen waves, each with a range
// of the rows).  Ids that are no adapter's become -1.  Tiles of up to 64 rows of one adapter hold their rows' numbers themselves, so
// that a kernel that works on one finds all it needs with one load.  Rows are mixed where more than a row
// in eight has another adapter than the row before: then the products of many rows go through them in this order (us, A x and the product, as
// they come and so, the codes' copy included: 16384 x 4096 -> 4096 of rank 16, twelve adapters mixed 322 and 282, 32 364 and 283; 2048 rows of 32
// 73 and 51; 4877 x 5816 -> 4224 of rank 19, 39 337 and 187; in runs, which stay as they are, 280).
template <class Id>
__global__ __launch_bounds__(1024) void adapt_plan(const Id* ids, int T, int N, F8Requests q) {
  extern __shared__ int32_t hist[];  // [16][N], behind them the tiles' first numbers [N + 1]
  __shared__ int32_t sh[4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* first_tile = hist + 16 * N;
  for (int i = tid; i < 16 * N; i += 1024) hist[i] = 0;
  __syncthreads();
  const int64_t per = ((int64_t)T + 1023) / 1024 * 64, begin = wave * per < T ? wave * per : T, end = begin + per < T ? begin + per : T;
  int with = 0, changes = 0;  // this wave's rows that have an adapter, that have another than the row before
  for (int64_t t0 = begin; t0 < end; t0 += 64) {
    const int64_t t = t0 + lane;
    const Id id = t < end ? ids[t] : -1;
    const int32_t a = id >= 0 && id < N ? (int32_t)id : -1;
    if (t < end) q.which[t] = a;
    if (a >= 0) atomicAdd(&hist[wave * N + a], 1);  // (a count: the same in any order)
    with += __popcll(__ballot(a >= 0));
    const Id id0 = t > 0 && t < end ? ids[t - 1] : id;
    changes += __popcll(__ballot(a != (id0 >= 0 && id0 < N ? (int32_t)id0 : -1)));
  }
  if (lane == 0) sh[2][wave] = with, sh[3][wave] = changes;
  __syncthreads();
  // N <= 1024: an adapter a thread
  int total = 0;
  if (tid < N)
    for (int w = 0; w < 16; ++w) {
      const int n = hist[w * N + tid];
      hist[w * N + tid] = total;
      total += n;
    }
  int rows = total, tiles = (total + kTileRows - 1) / kTileRows;  // sums up to and with this thread's
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int r = __shfl_up(rows, d), s = __shfl_up(tiles, d);
    if (lane >= d) rows += r, tiles += s;
  }
  if (lane == 63) sh[0][wave] = rows, sh[1][wave] = tiles;
  __syncthreads();
  int all_rows = 0, all_tiles = 0, all_changes = 0, none_at = 0;  // none_at: this wave's first row without an adapter, among all such
  for (int w = 0; w < 16; ++w) {
    if (w < wave) rows += sh[0][w], tiles += sh[1][w], none_at -= sh[2][w];
    all_rows += sh[0][w], all_tiles += sh[1][w], all_changes += sh[3][w];
  }
  none_at += all_rows + (int)begin;
  if (tid < N) {
    const int start = rows - total;
    for (int w = 0; w < 16; ++w) hist[w * N + tid] += start;
    q.start[tid] = start;
    first_tile[tid] = tiles - (total + kTileRows - 1) / kTileRows;
  }
  const int none_tiles = (T - all_rows + kTileRows - 1) / kTileRows;
  if (tid == 0) q.start[N] = all_rows, first_tile[N] = all_tiles, q.tiles[0] = all_tiles, q.tiles[1] = all_tiles + none_tiles, q.tiles[2] = all_changes > T / 8;
  __syncthreads();
  for (int64_t t0 = begin; t0 < end; t0 += 64) {
    const int64_t t = t0 + lane;
    const int a = t < end ? q.which[t] : -1;
    uint64_t todo = __ballot(a >= 0);
    while (todo) {
      const int of = __builtin_amdgcn_readlane(a, __builtin_ctzll(todo));
      const uint64_t same = __ballot(a == of);
      const int place = hist[wave * N + of];
      if (a == of) q.order[place + __popcll(same & ((1ull << lane) - 1))] = (int32_t)t;
      __builtin_amdgcn_wave_barrier();
      if (lane == 0) hist[wave * N + of] = place + __popcll(same);
      __builtin_amdgcn_wave_barrier();
      todo &= ~same;
    }
    const uint64_t none = __ballot(a < 0 && t < end);
    if (a < 0 && t < end) q.order[none_at + __popcll(none & ((1ull << lane) - 1))] = (int32_t)t;
    none_at += __popcll(none);
  }
  __syncthreads();
  for (int64_t i = tid; i < (int64_t)(all_tiles + none_tiles) * kTileRows; i += 1024) {
    const int tile = (int)(i / kTileRows), r = (int)(i % kTileRows);
    int of = N;  // the last adapter whose first tile is at most this one: none's tiles come behind all
    if (tile < all_tiles) {
      int lo = 0, hi = N;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_tile[mid] <= tile) lo = mid;
        else hi = mid;
      }
      of = lo;
    }
    const int from = q.start[of] + (tile - first_tile[of]) * kTileRows, left = (of < N ? q.start[of + 1] : T) - from;
    int32_t* record = q.tiles + 4 + (int64_t)tile * kTileWords;
    record[4 + r] = q.order[from + (r < left ? r : left - 1)];
    if (r == 0) record[0] = of < N ? of : -1, record[1] = left < kTileRows ? left : kTileRows, record[2] = from;
  }
}

// ------------------------------------------------------------------ an adapter's weights
// Both forms lie as the matrix instructions take them, a lane's eight values together and the lanes' in turn, so that every request of a wave is
// one kilobyte: where lanes take rows of their own a CU gets 7 bytes a clock, whatever it has under way.
//   by rank (16 x 32 x 16 products): blocks of 128 columns, of sixteen ranks, four j, 64 lanes: rank lane & 15, columns 64 (j >> 1) + 16 (lane >> 4) + 8 (j & 1)
//   by column (32 x 16 x 32): 32 columns, sixteen ranks, 64 lanes: column lane & 31, ranks 8 (lane >> 5)
__device__ __forceinline__ int64_t at_by_rank(int r, int c, int Rp) {
  return ((((int64_t)(c >> 7) * (Rp >> 4) + (r >> 4)) * 4 + ((c >> 6) & 1) * 2 + ((c >> 3) & 1)) * 64 + ((c >> 4) & 3) * 16 + (r & 15)) * 8 + (c & 7);
}
__device__ __forceinline__ int64_t at_by_column(int r, int c, int Rp) {
  return (((int64_t)(c >> 5) * (Rp >> 4) + (r >> 4)) * 64 + ((r >> 3) & 1) * 32 + (c & 31)) * 8 + (r & 7);
}
// A thread takes one rank of one padded column.  COLUMNS: W is [columns][rank], else [rank][columns].
template <bool F32, bool COLUMNS>
__device__ __forceinline__ void set_side(const void* W, int64_t ld, int rank, int columns, int Rp, uint16_t* by_column, uint16_t* by_rank, int64_t i) {
  const int c = (int)(i / Rp), r = (int)(i - (int64_t)c * Rp);
  uint16_t v = 0;
  if (r < rank && c < columns) {
    const int64_t at = COLUMNS ? c * ld + r : r * ld + c;
    v = F32 ? f32_to_bf16_rne(((const float*)W)[at]) : ((const uint16_t*)W)[at];
  }
  by_column[at_by_column(r, c, Rp)] = v;
  by_rank[at_by_rank(r, c, Rp)] = v;
}
template <bool F32>
__global__ __launch_bounds__(256) void adapt_set(F8Adapters d, int slot, int rank, const void* A, int64_t lda, const void* B, int64_t ldb, float scale) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, na = (int64_t)d.Ip * d.Rp, nb = (int64_t)d.Op * d.Rp;
  if (i < na) set_side<F32, false>(A, lda, rank, d.I, d.Rp, d.a_t + slot * na, d.a + slot * na, i);
  else if (i < na + nb) set_side<F32, true>(B, ldb, rank, d.O, d.Rp, d.b + slot * nb, d.b_t + slot * nb, i - na);
  if (i == 0) d.scale[slot] = scale;
}

// ------------------------------------------------------------------ down
enum { kBf16, kF32, kE4, kE5 };  // what the rows are given as

struct DownArgs {
  const void* X;
  const uint8_t* scale;  // of codes
  int64_t ld, srows;
  const uint16_t* down;  // [N][Rp Kp], by rank
  const float* factor;   // [N]
  float* u;              // [slices][T][Rp]
  F8Requests q;
  int32_t T, K, Kp, Rp, per;  // per: blocks of a slice
  int32_t e5, aligned;        // aligned: rows begin at 16 bytes
  uint8_t *codes, *to_scale;  // SAVE: the rows as codes, too
  int32_t sorts;              // mixed rows' codes go in the order of their adapters
};

__device__ __forceinline__ u32x4_t pack8(const float* v) {
  return u32x4_t{f8_pack_bf16x2(v[0], v[1]), f8_pack_bf16x2(v[2], v[3]), f8_pack_bf16x2(v[4], v[5]), f8_pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void unpack8(u32x4_t w, float* v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(w[k] << 16);
    v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
  }
}
// what eight values lose as bf16, and that as bf16
__device__ __forceinline__ u32x4_t rest8(const float* v, u32x4_t high, float* rest) {
  float h[8];
  unpack8(high, h);
#pragma unroll
  for (int k = 0; k < 8; ++k) rest[k] = v[k] - h[k];
  return pack8(rest);
}

// The wait between a matrix instruction and the first use of its result, by hand: the branches over fragments that are not there are ways
// that meet again, and the compiler counts the instructions of one of them.
template <int NR, int M>
__device__ __forceinline__ void settle(f32x4_t (&acc)[NR][M]) {
  asm volatile("s_nop 15\n\ts_nop 7" : "+v"(acc[0][0]));
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int m = 0; m < M; ++m) asm volatile("" : "+v"(acc[i][m]));
}

// A workgroup takes a tile's rows, or a half or quarter of them, and a slice of the blocks of 128 columns, which its waves share out; the slices'
// sums are added by who reads u.  A wave's block of rows, 8 KB, goes through LDS, its own part of it: requests cover whole rows of the block,
// while the matrix instruction wants sixteen rows' pieces side by side.  A row of pieces of 16 bytes is permuted by its number, so that
// these lie in different banks.  In a block a lane's columns are 64 q + 16 g + 8 h + 0..7.  The ranks are the matrix
// instruction's rows and the rows its columns, so nothing of one row, NaN among it, reaches another's sums.  SAVE: the rows become
// codes on the way, as f8_save makes them, rows without an adapter too: four lanes hold a row's 128 columns.  Rows that are codes are copied where
// they are mixed.
// (64 rows, for an adapter's columns are read again for every tile.)
template <int SRC, int NR>
constexpr int kFragments = SRC == kF32 ? 1 : SRC == kBf16 || NR > 1 ? 2 : 4;  // of sixteen rows

// lds: [waves][rows of a block]; then sums [waves][NR][M][64][4]
template <int SRC, int NR, bool SAVE>
__device__ __forceinline__ void down(const DownArgs& a, int block, uint8_t* lds) {
  constexpr bool kCoded = SRC == kE4 || SRC == kE5;
  constexpr int M = kFragments<SRC, NR>, kParts = 4 / M, kSize = SRC == kF32 ? 4 : SRC == kBf16 ? 2 : 1;
  constexpr int kRow = 128 * kSize, kPieces = kRow / 16, kAtOnce = 64 / kPieces, kAsks = 16 * M / kAtOnce;  // bytes and pieces of a row; rows a request, requests
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int tile = block / kParts, part = block % kParts;
  const int32_t* record = a.q.tiles + 4 + (int64_t)tile * kTileWords;
  const int32_t* rows = record + 4 + part * M * 16;
  const int of = __builtin_amdgcn_readfirstlane(record[0]), n = __builtin_amdgcn_readfirstlane(record[1]) - part * M * 16;
  // the rows that this lane asks for pieces of, and of which piece
  int64_t asked[kAsks];
#pragma unroll
  for (int q = 0; q < kAsks; ++q) asked[q] = rows[q * kAtOnce + lane / kPieces];
  int32_t t[kCoded ? M : 1];
  if constexpr (kCoded)
#pragma unroll
    for (int m = 0; m < M; ++m) t[m] = rows[m * 16 + r];
  // where the codes go, by their row in this part of the tile
  const bool sorted = SAVE && a.sorts && a.q.tiles[2], saves = SAVE && blockIdx.z == 0 && (!kCoded || sorted);
  const int first = SAVE ? __builtin_amdgcn_readfirstlane(record[2]) + part * M * 16 : 0;
  auto goes = [&](int row) { return kCoded || sorted ? first + row : rows[row]; };
  // (held: asked for again in the loop they take 7 us of 119 at 8192 x 16384 of rank 32)
  int32_t leaves[SAVE && !kCoded ? 2 * M : 1], scales_of[SAVE && !kCoded ? M : 1];
  if constexpr (SAVE && !kCoded) {
#pragma unroll
    for (int q = 0; q < 2 * M; ++q) leaves[q] = goes(q * 8 + (lane >> 3));
#pragma unroll
    for (int m = 0; m < M; ++m) scales_of[m] = goes(m * 16 + r);
  }
  const int nb = a.Kp >> 7, kb0 = blockIdx.y * a.per, kb1 = kb0 + a.per < nb ? kb0 + a.per : nb;
  if (tile >= a.q.tiles[saves ? 1 : 0] || n <= 0 || kb0 >= nb) return;  // (no slice is empty: f8_down_slices)
  auto key = [](int row) { return kCoded ? (row >> 1) & 7 : row & 15; };
  const uint8_t* x[kAsks];
#pragma unroll
  for (int q = 0; q < kAsks; ++q) x[q] = (const uint8_t*)a.X + asked[q] * a.ld * kSize;
  uint8_t* mine = lds + wave * 16 * M * kRow;
  const uint16_t* w = a.down + (int64_t)(of < 0 ? 0 : of) * a.Rp * a.Kp + (blockIdx.z * NR * 4 * 64 + lane) * 8;
  f32x4_t acc[NR][M] = {};
  // Workgroups begin at different columns: of rows a power of two apart those at one column lie in one channel of the L2, and all would ask that one
  // (8192 x 16384 of one adapter 255 us, of two 98).
  const int blocks = kb1 - kb0, turn = block * waves % blocks;
  for (int i = wave; i < blocks; i += waves) {
    const int kb = kb0 + (i + turn < blocks ? i + turn : i + turn - blocks);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the last block has been read
    if (kCoded || (a.aligned && kb * 128 + 128 <= a.K)) {
#pragma unroll
      for (int q = 0; q < kAsks; ++q) {
        const int piece = (lane % kPieces) ^ key(q * kAtOnce + lane / kPieces);
        __builtin_amdgcn_global_load_lds((f8_gptr_t)(x[q] + (int64_t)kb * kRow + piece * 16), (f8_lptr_t)(mine + q * 1024), 16, 0, 0);
      }
    } else if constexpr (!kCoded) {  // rows at any address, a row's end
#pragma unroll
      for (int q = 0; q < kAsks; ++q) {
        const int c = kb * 128 + ((lane % kPieces) ^ key(q * kAtOnce + lane / kPieces)) * (16 / kSize);
        u32x4_t v;
        if constexpr (SRC == kBf16) {
          if (kb * 128 + 128 <= a.K) {
            v = *(const f8_any2_t*)((const uint16_t*)x[q] + c);
          } else {
            float f[8];
            load8<false>(x[q], c, a.K, f);
            v = pack8(f);
          }
        } else if (kb * 128 + 128 <= a.K) {
          v = *(const f8_any4_t*)((const float*)x[q] + c);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = c + k < a.K ? ((const uint32_t*)x[q])[c + k] : 0;
        }
        *(u32x4_t*)(mine + q * 1024 + lane * 16) = v;
      }
    }
    u32x4_t wv[NR][4];
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) wv[i][j] = *(const u32x4_t*)(w + (((int64_t)kb * (a.Rp >> 4) + i) * 4 + j) * 64 * 8);
    int s[kCoded ? M : 1];
    if constexpr (kCoded)
#pragma unroll
      for (int m = 0; m < M; ++m) s[m] = a.scale[kb * a.srows + t[m]];
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    u32x4_t codes[SAVE && !kCoded ? M : 1][2];
    int bytes[SAVE && !kCoded ? M : 1];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const uint8_t* row = mine + (m * 16 + r) * kRow;
      auto piece = [&](int p) { return *(const u32x4_t*)(row + ((p ^ key(m * 16 + r)) << 4)); };
      u32x4_t xv[4], xl[SRC == kF32 ? 4 : 1], xs[SRC == kF32 ? 4 : 1];
      float v[SRC == kF32 ? 4 : 1][8];
      if constexpr (kCoded) {
        const float f = __uint_as_float((uint32_t)s[m] << 23);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const u32x4_t c = piece(4 * q + g);
          xv[2 * q] = f8_decode_bf16x8<SRC == kE5>(c.x, c.y, f);
          xv[2 * q + 1] = f8_decode_bf16x8<SRC == kE5>(c.z, c.w, f);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int p = 8 * (j >> 1) + 2 * g + (j & 1);  // by eights
          if constexpr (SRC == kBf16) {
            xv[j] = piece(p);
          } else {
            const u32x4_t p0 = piece(2 * p), p1 = piece(2 * p + 1);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] = __uint_as_float(k < 4 ? p0[k & 3] : p1[k & 3]);
            xv[j] = pack8(v[j]);
            float rest[8];
            xl[j] = rest8(v[j], xv[j], rest);
            float none[8];
            xs[j] = rest8(rest, xl[j], none);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[i][m] = mfma_bf16_16x16x32(wv[i][j], xv[j], acc[i][m]);
          if constexpr (SRC == kF32) {
            acc[i][m] = mfma_bf16_16x16x32(wv[i][j], xl[j], acc[i][m]);
            acc[i][m] = mfma_bf16_16x16x32(wv[i][j], xs[j], acc[i][m]);
          }
        }
      if constexpr (SAVE && !kCoded) {
        uint32_t most = 0;
        float y[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (SRC == kBf16) unpack8(xv[j], y[j]);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if constexpr (SRC == kF32) y[j][k] = v[j][k];
            most = max(most, f8_magnitude(y[j][k]));
          }
        }
        const auto p = __builtin_amdgcn_permlane16_swap(most, most, false, false);
        most = max(p[0], p[1]);
        const auto o = __builtin_amdgcn_permlane32_swap(most, most, false, false);
        most = max(o[0], o[1]);
        auto encode = [&](auto E5) {
          bytes[m] = f8_scale_byte<decltype(E5)::value>(most);
          const float f = f8_inverse(bytes[m]);
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float* z = &y[2 * q + (k >> 1)][4 * (k & 1)];
              codes[m][q][k] = f8_encode4<decltype(E5)::value>(z[0] * f, z[1] * f, z[2] * f, z[3] * f);
            }
        };
        if (a.e5) encode(std::true_type{});
        else encode(std::false_type{});
      }
    }
    if constexpr (SAVE) {
      if (saves) {  // through the wave's LDS, whose rows have been read: whole lines leave
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const int row = m * 16 + r;
          if constexpr (!kCoded)  // (as codes lie there from the start)
#pragma unroll
            for (int q = 0; q < 2; ++q) *(u32x4_t*)(mine + row * 128 + (((4 * q + g) ^ ((row >> 1) & 7)) << 4)) = codes[m][q];
          if (g == 0 && row < n) a.to_scale[kb * a.srows + (kCoded ? goes(row) : scales_of[kCoded ? 0 : m])] = (uint8_t)(kCoded ? s[kCoded ? m : 0] : bytes[kCoded ? 0 : m]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int q = 0; q < 2 * M; ++q) {
          const int row = q * 8 + (lane >> 3), p = lane & 7;
          const u32x4_t c = *(const u32x4_t*)(mine + row * 128 + ((p ^ ((row >> 1) & 7)) << 4));
          if (row < n) *(u32x4_t*)(a.codes + (int64_t)(kCoded ? goes(row) : leaves[kCoded ? 0 : q]) * a.Kp + kb * 128 + p * 16) = c;
        }
      }
    }
  }
  if (of < 0) return;
  settle(acc);
  __syncthreads();
  float* sums = (float*)lds;
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int m = 0; m < M; ++m) *(f32x4_t*)(sums + (((wave * NR + i) * M + m) * 64 + lane) * 4) = acc[i][m];
  __syncthreads();
  const float factor = a.factor[of];
  for (int i = threadIdx.x; i < NR * M * 64; i += blockDim.x) {
    const int row = ((i >> 6) % M) * 16 + (i & 15);
    if (row >= n) continue;
    f32x4_t sum = *(const f32x4_t*)(sums + i * 4);
    for (int v = 1; v < waves; ++v) sum += *(const f32x4_t*)(sums + (v * NR * M * 64 + i) * 4);
    const int64_t at = (int64_t)blockIdx.y * a.T + rows[row];
    *(f32x4_t*)(a.u + at * a.Rp + (blockIdx.z * NR + i / (M * 64)) * 16 + ((i >> 4) & 3) * 4) = sum * factor;
  }
}

template <int SRC>
constexpr bool kValues = SRC == kBf16 || SRC == kF32;
template <int SRC, int NR, bool SAVE>
__global__ __launch_bounds__(SAVE && kValues<SRC> ? 256 : 512, SAVE && kValues<SRC> ? (NR == 4 ? 2 : 3) : NR == 4 ? 2 : 4) void adapt_down(DownArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  kernarg_touch<DownArgs>();
  down<SRC, NR, SAVE>(a, blockIdx.x, lds);
}
// u and v of the gradients in one launch, v of dY first (us, apart and together, with the layer's input gradient and all of the adapters': 37 rows, 1000
// and 520 columns 29.6 and 25.8, 8192, 4096 and 16384 727 and 708).
struct BothArgs {
  DownArgs y, x;
  int32_t first;  // workgroups of y
};
template <int SRC, int NR>
__global__ __launch_bounds__(512, NR == 4 ? 2 : 4) void adapt_down_both(BothArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  kernarg_touch<BothArgs>();
  if ((int)blockIdx.x < a.first) down<kBf16, NR, false>(a.y, blockIdx.x, lds);
  else down<SRC, NR, false>(a.x, blockIdx.x - a.first, lds);
}

template <int SRC, int NR>
constexpr int down_lds() {  // a wave's bytes
  constexpr int rows = 16 * kFragments<SRC, NR> * (SRC == kF32 ? 512 : SRC == kBf16 ? 256 : 128), sums = NR * kFragments<SRC, NR> * 1024;
  return rows > sums ? rows : sums;
}
inline int down_waves(int most, int per) {  // a wave a block of columns at least
  while (most > 1 && most > per) most >>= 1;
  return most;
}
inline bool raise(const void* kernel, int lds) { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess; }

template <int SRC, int NR, bool SAVE>
int down_launch(const DownArgs& a, int T, int N, int slices, hipStream_t st) {
  constexpr int most = SAVE && kValues<SRC> ? 4 : 8, lds = down_lds<SRC, NR>();
  const int64_t groups = f8_request_tiles(T, N) * (4 / kFragments<SRC, NR>);
  const int waves = down_waves(most, a.per);
  if (!f8_fits_x(groups, 512)) return BSP_ERR_SHAPE;
  static const bool raised = raise((const void*)&adapt_down<SRC, NR, SAVE>, most * lds);
  if (!raised) return BSP_ERR_HIP;
  hipLaunchKernelGGL((adapt_down<SRC, NR, SAVE>), dim3((unsigned)groups, (unsigned)slices, (unsigned)(a.Rp / (16 * NR))), dim3(64 * waves),
                     (size_t)waves * lds, st, a);
  return launched();
}
template <int SRC, int NR>
int both_launch(BothArgs& a, int T, int N, int slices, hipStream_t st) {
  constexpr int lds = down_lds<SRC, NR>() > down_lds<kBf16, NR>() ? down_lds<SRC, NR>() : down_lds<kBf16, NR>();
  const int64_t tiles = f8_request_tiles(T, N), groups = tiles * (4 / kFragments<kBf16, NR> + 4 / kFragments<SRC, NR>);
  const int waves = down_waves(8, a.x.per > a.y.per ? a.x.per : a.y.per);
  if (!f8_fits_x(groups, 512)) return BSP_ERR_SHAPE;
  a.first = (int32_t)(tiles * (4 / kFragments<kBf16, NR>));
  static const bool raised = raise((const void*)&adapt_down_both<SRC, NR>, 8 * lds);
  if (!raised) return BSP_ERR_HIP;
  hipLaunchKernelGGL((adapt_down_both<SRC, NR>), dim3((unsigned)groups, (unsigned)slices, (unsigned)(a.x.Rp / (16 * NR))), dim3(64 * waves), (size_t)waves * lds, st, a);
  return launched();
}
template <class Run>
int by_rank(int Rp, Run run) {
  switch (Rp) {
    case 16: return run(std::integral_constant<int, 1>{});
    case 32: return run(std::integral_constant<int, 2>{});
    default: return run(std::integral_constant<int, 4>{});  // (128: in two halves)
  }
}
template <int SRC, bool SAVE>
int down_rank(const DownArgs& a, int T, int N, int slices, hipStream_t st) {
  return by_rank(a.Rp, [&](auto nr) { return down_launch<SRC, decltype(nr)::value, SAVE>(a, T, N, slices, st); });
}
template <int SRC>
int both_rank(BothArgs& a, int T, int N, int slices, hipStream_t st) {
  return by_rank(a.x.Rp, [&](auto nr) { return both_launch<SRC, decltype(nr)::value>(a, T, N, slices, st); });
}
DownArgs down_args(const F8Adapters& d, bool transposed, const F8Input& x, int T, const F8Requests& q, float* u, int slices) {
  DownArgs a{};
  a.X = x.X, a.scale = x.scale, a.ld = x.ld, a.srows = f8_scale_rows(T), a.down = transposed ? d.b_t : d.a, a.factor = d.scale, a.u = u, a.q = q;
  a.T = T, a.K = transposed ? d.O : d.I, a.Kp = transposed ? d.Op : d.Ip, a.Rp = d.Rp, a.e5 = x.e5;
  const int64_t size = x.dtype == BSP_F32 ? 4 : x.dtype == BSP_BF16 ? 2 : 1;
  a.aligned = (((uintptr_t)x.X | (uintptr_t)(x.ld * size)) & 15) == 0;
  a.per = (f8_blocks(a.K) + slices - 1) / slices;
  return a;
}

// ------------------------------------------------------------------ gradients
constexpr int kStep = 32;  // rows a step

struct GradArgs {
  F8Requests q;
  const uint16_t* dY;     // bf16 [T][O]
  const void* X;          // bf16 [T][I], or codes
  const uint8_t* scale;
  int64_t ldy, ldx, srows;
  const float *u, *v;     // [slices][T][Rp]
  int64_t u_step;         // T Rp
  int32_t u_slices, v_slices, Rp;
  float *dA, *dB;         // [N][R][I], [N][O][R]
  float* part;            // [slots][R I + O R]
  int32_t N, R, I, O, blocks_o, chunk;
  int32_t src;            // of X
  int32_t each;           // a chunk is an adapter
};

// Which adapter's rows chunk number k holds, and where its sums go.  The same in all lanes.
struct Chunk {
  int of, begin, rows;  // adapter (N: none), first row's place in the order, how many
  int slot;             // of the partial sums, -1: the adapter has no other chunk
};
__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}
__device__ __forceinline__ Chunk find_chunk(const F8Requests& q, int N, int length, int k) {
  const int lane = threadIdx.x & 63;
  int chunks = 0, slots = 0;  // of the adapters before
  for (int a0 = 0; a0 < N; a0 += 64) {
    const int a = a0 + lane, start = a < N ? q.start[a] : 0, n = a < N ? q.start[a + 1] - start : 0;
    const int mine = (n + length - 1) / length, kept = mine > 1 ? mine : 0;
    const int upto = chunks + wave_scan(mine, lane), slot_upto = slots + wave_scan(kept, lane);
    const uint64_t found = __ballot(k >= upto - mine && k < upto);
    if (found) {
      const int l = __builtin_ctzll(found);
      const int s = __builtin_amdgcn_readlane(start, l), c = __builtin_amdgcn_readlane(n, l), j = k - __builtin_amdgcn_readlane(upto - mine, l);
      return Chunk{a0 + l, s + j * length, c - j * length < length ? c - j * length : length,
                   __builtin_amdgcn_readlane(kept, l) ? __builtin_amdgcn_readlane(slot_upto - kept, l) + j : -1};
    }
    chunks = __builtin_amdgcn_readlane(upto, 63), slots = __builtin_amdgcn_readlane(slot_upto, 63);
  }
  return Chunk{N, 0, 0, -1};
}

template <int BYTES>
__device__ __forceinline__ u32x4_t read_columns(const uint8_t* p) {  // rows +0..3 and +4..7 of this lane's column, rows BYTES apart
  auto* q = (__attribute__((address_space(3))) s16x4_t*)(uintptr_t)p;
  const u32x2_t a = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q));
  const u32x2_t b = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + 4 * BYTES / 8));
  return u32x4_t{a.x, a.y, b.x, b.y};
}
__device__ __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// 128 columns of one side, dY (dB) or X (dA), with a chunk of an adapter's rows and RP ranks.  Four waves of 32 columns each; the other operand
// is u or v, its three parts side by side in a row of 3 RP bf16.  CODED: the rows are codes; WHOLE: all 128 columns are there.
template <int RP, bool CODED, bool WHOLE>
__device__ __forceinline__ void grad_side(const GradArgs& a, const Chunk& k, bool in_y, int kb, uint8_t* lds) {
  constexpr int NT = (3 * RP + 31) / 32;    // tiles of 32 columns of u
  constexpr int kQ = 64 * NT + 16;          // bytes from row to row of u in LDS
  constexpr int kP = kStep * 256, kBuffer = kP + kStep * kQ, kMine = RP / 8;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int columns = in_y ? a.O : a.I, c0 = kb * 128;
  const void* P = in_y ? (const void*)a.dY : a.X;
  const int64_t ld = in_y ? a.ldy : a.ldx;
  const int r0 = blockIdx.z * RP, slices = in_y ? a.u_slices : a.v_slices;
  // what this thread brings: sixteen columns of a row, and kMine values of u.  Two steps are on their way to registers while a third is
  // multiplied; nothing about that is conditional, and nothing looks at what is on its way: either would wait for it.
  const int row = tid >> 3, piece = tid & 7, c = c0 + piece * 16;
  const float* Q = (in_y ? a.u : a.v) + r0 + piece * kMine;
  const int64_t second = slices > 1 ? a.u_step : 0;
  struct Coming {
    u32x4_t p[2];
    float u[kMine], u2[kMine];  // of two slices
    int s;
  } in[2];
  auto place = [&](int i) { return a.q.order[k.begin + (i * kStep + row < k.rows ? i * kStep + row : k.rows - 1)]; };  // (past the last row: the last)
  auto read_u = [&](const float* q, float* u) {
    if constexpr (kMine >= 4) {
#pragma unroll
      for (int e = 0; e < kMine; e += 4) {
        const f32x4_t v = *(const f32x4_t*)(q + e);
        u[e] = v[0], u[e + 1] = v[1], u[e + 2] = v[2], u[e + 3] = v[3];
      }
    } else {
      const f32x2_t v = *(const f32x2_t*)q;
      u[0] = v[0], u[1] = v[1];
    }
  };
  auto ask = [&](int64_t t, Coming& to) {
    if constexpr (CODED) {
      to.p[0] = *(const u32x4_t*)((const uint8_t*)P + t * ld + c);
      to.s = a.scale[kb * a.srows + t];
    } else if constexpr (WHOLE) {
      const uint16_t* x = (const uint16_t*)P + t * ld + c;
      to.p[0] = *(const f8_any2_t*)x;
      to.p[1] = *(const f8_any2_t*)(x + 8);
    } else {
      float v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load8<false>((const uint16_t*)P + t * ld, c + 8 * h, columns, v);
        to.p[h] = pack8(v);
      }
    }
    read_u(Q + t * a.Rp, to.u);
    read_u(Q + t * a.Rp + second, to.u2);
  };
  auto write = [&](int buf, int i, const Coming& from) {
    const bool have = i * kStep + row < k.rows;  // rows past the chunk add nothing, whatever they hold
    uint8_t* to = lds + buf * kBuffer;
    u32x4_t w[2];
    if constexpr (CODED) {
      const float f = __uint_as_float((uint32_t)from.s << 23);
      const u32x4_t x = from.p[0];
      if (a.src == kE5) w[0] = f8_decode_bf16x8<true>(x.x, x.y, f), w[1] = f8_decode_bf16x8<true>(x.z, x.w, f);
      else w[0] = f8_decode_bf16x8<false>(x.x, x.y, f), w[1] = f8_decode_bf16x8<false>(x.z, x.w, f);
    } else {
      w[0] = from.p[0], w[1] = from.p[1];
    }
    const int key = (row & 3) << 1 | ((row >> 3) & 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) *(u32x4_t*)(to + row * 256 + ((piece ^ key) << 5) + 16 * h) = have ? w[h] : u32x4_t{0, 0, 0, 0};
    uint16_t* hi = (uint16_t*)(to + kP + row * kQ) + piece * kMine;
#pragma unroll
    for (int e = 0; e < kMine; e += 2) {
      const float y0 = slices > 1 ? from.u[e] + from.u2[e] : from.u[e], y1 = slices > 1 ? from.u[e + 1] + from.u2[e + 1] : from.u[e + 1];
      const float x0 = have ? y0 : 0.f, x1 = have ? y1 : 0.f;
      const uint32_t h = f8_pack_bf16x2(x0, x1);
      const float z0 = x0 - __uint_as_float(h << 16), z1 = x1 - __uint_as_float(h & 0xFFFF0000u);
      const uint32_t l = f8_pack_bf16x2(z0, z1);
      *(uint32_t*)(hi + e) = h;
      *(uint32_t*)(hi + RP + e) = l;
      *(uint32_t*)(hi + 2 * RP + e) = f8_pack_bf16x2(z0 - __uint_as_float(l << 16), z1 - __uint_as_float(l & 0xFFFF0000u));
    }
  };
  const int half = lane >> 5, trow = half * 8 + ((lane & 15) >> 2), key_r = ((lane & 15) >> 2) << 1 | half;
  const int at_p = trow * 256 + (((wave * 2 + ((lane >> 4) & 1)) ^ key_r) << 5) + (lane & 3) * 8;
  const int at_q = kP + trow * kQ + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  f32x16_t acc[NT] = {};
  const int steps = (k.rows + kStep - 1) / kStep;
  ask(place(0), in[0]);
  ask(place(1), in[1]);
  int next = place(2);
  write(0, 0, in[0]);
  ask(next, in[0]);
  next = place(3);
  __syncthreads();
  auto step = [&](int i, Coming& coming) {  // multiplies step i, writes step i + 1 from `coming`, asks for step i + 3
    const uint8_t* from = lds + (i & 1) * kBuffer;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4_t x = read_columns<256>(from + h * 16 * 256 + at_p);
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n] = mfma32(x, read_columns<kQ>(from + h * 16 * kQ + at_q + n * 64), acc[n]);
    }
    write((i + 1) & 1, i + 1, coming);
    ask(next, coming);
    next = place(i + 4);
    __syncthreads();
  };
  for (int i = 0; i < steps; i += 2) {  // (a step past the last multiplies zeros)
    step(i, in[1]);
    step(i + 1, in[0]);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) asm volatile("" : "+a"(acc[n]));
  asm volatile("s_nop 15\n\ts_nop 7");  // (see settle)
  // the parts together, the smallest first
  constexpr int kTiles = RP == 16 ? 1 : RP / 32;
  if constexpr (RP == 16) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][e] += __shfl_xor(acc[0][e], 16) + acc[1][e];
  } else {
#pragma unroll
    for (int n = 0; n < kTiles; ++n) acc[n] += acc[n + kTiles] + acc[n + 2 * kTiles];
  }
  const int64_t na = (int64_t)a.R * a.I, nb = (int64_t)a.O * a.R;
  float* to_a = k.slot < 0 ? a.dA + k.of * na : a.part + k.slot * (na + nb);
  float* to_b = k.slot < 0 ? a.dB + k.of * nb : to_a + na;
#pragma unroll
  for (int n = 0; n < kTiles; ++n) {
    const int r = r0 + n * 32 + (lane & 31);
    if (r >= a.R || (RP == 16 && (lane & 16))) continue;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int col = c0 + wave * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
      if (col >= columns) continue;
      if (in_y) to_b[(int64_t)col * a.R + r] = acc[n][e];
      else to_a[(int64_t)r * a.I + col] = acc[n][e];
    }
  }
}

// Where no adapter can have more than one chunk a workgroup takes an adapter, and one without rows gets its zeros here: a launch less.
template <int RP>
__device__ __forceinline__ void no_rows(const GradArgs& a, int of, bool in_y, int kb) {
  const int r0 = blockIdx.z * RP;
  for (int i = threadIdx.x; i < 128 * RP; i += 256) {
    const int r = r0 + (in_y ? i % RP : i / 128), c = kb * 128 + (in_y ? i / RP : i % 128);
    if (r >= a.R || c >= (in_y ? a.O : a.I)) continue;
    if (in_y) a.dB[((int64_t)of * a.O + c) * a.R + r] = 0.f;
    else a.dA[((int64_t)of * a.R + r) * a.I + c] = 0.f;
  }
}
template <int RP>
__global__ __launch_bounds__(256) void adapt_grad(GradArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kStep * (256 + 64 * ((3 * RP + 31) / 32) + 16)];
  const int y = blockIdx.y;
  const Chunk k = a.each ? Chunk{y, a.q.start[y], a.q.start[y + 1] - a.q.start[y], -1} : find_chunk(a.q, a.N, a.chunk, y);
  if (k.of >= a.N) return;
  const bool in_y = (int)blockIdx.x < a.blocks_o;
  const int kb = in_y ? blockIdx.x : blockIdx.x - a.blocks_o;
  if (k.rows == 0) no_rows<RP>(a, k.of, in_y, kb);
  else if (!in_y && a.src != kBf16) grad_side<RP, true, true>(a, k, in_y, kb, lds);
  else if (kb * 128 + 128 <= (in_y ? a.O : a.I)) grad_side<RP, false, true>(a, k, in_y, kb, lds);
  else grad_side<RP, false, false>(a, k, in_y, kb, lds);
}

// Adapters of several chunks: their sums in order; of none: zeros.
__global__ __launch_bounds__(256) void adapt_join(GradArgs a) {
  const int lane = threadIdx.x & 63, of = blockIdx.y;
  const int n = a.q.start[of + 1] - a.q.start[of], chunks = (n + a.chunk - 1) / a.chunk;
  if (chunks == 1) return;
  int slot = 0;
  for (int a0 = 0; a0 < of; a0 += 64) {
    const int b = a0 + lane, m = b < of ? (a.q.start[b + 1] - a.q.start[b] + a.chunk - 1) / a.chunk : 0;
    slot += __builtin_amdgcn_readlane(wave_scan(m > 1 ? m : 0, lane), 63);
  }
  const int64_t na = (int64_t)a.R * a.I, nb = (int64_t)a.O * a.R;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < na + nb; i += (int64_t)gridDim.x * 256) {
    float s = 0.f;
#pragma unroll 8
    for (int k = 0; k < chunks; ++k) s += a.part[(slot + k) * (na + nb) + i];
    if (i < na) a.dA[of * na + i] = s;
    else a.dB[of * nb + i - na] = s;
  }
}

// Rows of a chunk: such that there are about two workgroups a CU, which is as many as run at one time (us with two and four, the launch that joins
// included: 16384 rows, 4096 and 4096 columns of rank 16, twelve adapters 46 and 61, 8192, 4096 and 16384 of rank 32, four 86 and 100, 2048, 4096 and
// 4096 of one 17 and 34).
int chunk_of(int T, int I, int O) {
  const int64_t blocks = f8_blocks(I) + f8_blocks(O);
  const int64_t rows = ((int64_t)T * blocks / 512 + kStep - 1) / kStep * kStep;
  return rows < 128 ? 128 : (int)(rows < INT32_MAX / 2 ? rows : INT32_MAX / 2 / kStep * kStep);
}

}  // namespace

int64_t f8_request_tiles(int T, int N) { return (int64_t)T / kTileRows + (T < N + 1 ? T : N + 1); }

F8Requests f8_requests_of(const bsp_f8_requests* r) {
  int32_t* p = r->plan;
  F8Requests q{};
  q.start = p, p += (r->N + 1 + 3) & ~3;
  q.which = p, p += ((int64_t)r->T + 3) & ~(int64_t)3;
  q.order = p, p += ((int64_t)r->T + 3) & ~(int64_t)3;
  q.tiles = p;
  return q;
}
int64_t f8_requests_bytes(int T, int N) {
  return 4 * (((N + 1 + 3) & ~3) + 2 * (((int64_t)T + 3) & ~(int64_t)3) + 4 + kTileWords * f8_request_tiles(T, N));
}
int f8_launch_plan(const bsp_f8_requests* r, const void* which, bool wide, hipStream_t st) {
  const F8Requests q = f8_requests_of(r);
  const size_t lds = (size_t)(17 * r->N + 1) * 4;
  auto run = [&](auto kernel, auto* ids) {
    static const bool raised = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (17 * 1024 + 1) * 4) == hipSuccess;
    if (!raised) return (int)BSP_ERR_HIP;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(1024), lds, st, ids, r->T, r->N, q);
    return launched();
  };
  return wide ? run(adapt_plan<int64_t>, (const int64_t*)which) : run(adapt_plan<int32_t>, (const int32_t*)which);
}

F8Adapters f8_adapters_of(const bsp_f8_adapters* d) {
  F8Adapters v{};
  v.N = d->N, v.R = d->R, v.I = d->I, v.O = d->O, v.Rp = d->R <= 16 ? 16 : d->R <= 32 ? 32 : d->R <= 64 ? 64 : 128;
  v.Ip = f8_blocks(d->I) * F8_BLOCK, v.Op = f8_blocks(d->O) * F8_BLOCK;
  v.a = d->a, v.a_t = d->a_t, v.b = d->b, v.b_t = d->b_t, v.scale = d->scale;
  return v;
}
int f8_launch_set(const F8Adapters& d, int slot, int rank, const void* A, int64_t lda, const void* B, int64_t ldb, bool f32, float scale, hipStream_t st) {
  const int64_t groups = ((int64_t)(d.Ip + d.Op) * d.Rp + 255) / 256;
  if (!f8_fits_x(groups, 256)) return BSP_ERR_SHAPE;
  if (f32) hipLaunchKernelGGL(adapt_set<true>, dim3((unsigned)groups), dim3(256), 0, st, d, slot, rank, A, lda, B, ldb, scale);
  else hipLaunchKernelGGL(adapt_set<false>, dim3((unsigned)groups), dim3(256), 0, st, d, slot, rank, A, lda, B, ldb, scale);
  return launched();
}

// Into how many slices the columns are cut, of eight blocks at least, one a wave: few rows want as many workgroups as the chip has CUs.  Who reads u
// adds them: a product once for every tile of results, the gradients, which hold two on their way, for every block of 128 columns.  (8192 x 16384
// bf16, rank 32: 88, 73, 66 us in one, two and four; a launch that adds four takes 5.)
int f8_down_slices(int T, int N, int K, bool grad) {
  const int64_t tiles = f8_request_tiles(T, N);
  const int most = grad || tiles >= 64 ? 2 : 8;
  int slices = 1;
  while (slices < most && tiles * slices < 256 && f8_blocks(K) >= 16 * slices) slices *= 2;
  return slices;
}
int f8_launch_down(const F8Adapters& d, bool transposed, const F8Input& x, int T, const F8Requests& q, float* u, uint8_t* codes, uint8_t* scale, bool sorts, hipStream_t st) {
  const int slices = f8_down_slices(T, d.N, transposed ? d.O : d.I, false);
  DownArgs a = down_args(d, transposed, x, T, q, u, slices);
  a.codes = codes, a.to_scale = scale, a.sorts = sorts;
  switch (x.dtype) {
    case BSP_BF16: return codes ? down_rank<kBf16, true>(a, T, d.N, slices, st) : down_rank<kBf16, false>(a, T, d.N, slices, st);
    case BSP_F32: return codes ? down_rank<kF32, true>(a, T, d.N, slices, st) : down_rank<kF32, false>(a, T, d.N, slices, st);
    case BSP_E4M3: return codes ? down_rank<kE4, true>(a, T, d.N, slices, st) : down_rank<kE4, false>(a, T, d.N, slices, st);
    default: return codes ? down_rank<kE5, true>(a, T, d.N, slices, st) : down_rank<kE5, false>(a, T, d.N, slices, st);
  }
}
int f8_launch_down_both(const F8Adapters& d, const F8Input& x, const F8Input& dY, int T, const F8Requests& q, float* u, float* v, hipStream_t st) {
  const int nu = f8_down_slices(T, d.N, d.I, true), nv = f8_down_slices(T, d.N, d.O, true), slices = nu > nv ? nu : nv;
  BothArgs a{down_args(d, true, dY, T, q, v, nv), down_args(d, false, x, T, q, u, nu), 0};
  switch (x.dtype) {
    case BSP_BF16: return both_rank<kBf16>(a, T, d.N, slices, st);
    case BSP_E4M3: return both_rank<kE4>(a, T, d.N, slices, st);
    default: return both_rank<kE5>(a, T, d.N, slices, st);
  }
}

int64_t f8_adapt_part_bytes(const F8Adapters& d, int T) {
  const int chunk = chunk_of(T, d.I, d.O);
  const int64_t slots = T <= chunk ? 0 : 2 * (int64_t)T / chunk;  // (an adapter of several chunks has fewer than twice its rows' share)
  return slots * ((int64_t)d.R * (d.I + (int64_t)d.O)) * 4;
}
int f8_launch_adapt_grad(const F8Adapters& d, const uint16_t* dY, int64_t ldy, const F8Input& x, int T, const F8Requests& q, const float* u, const float* v,
                         float* part, float* dA, float* dB, hipStream_t st) {
  GradArgs a{};
  a.q = q, a.dY = dY, a.X = x.X, a.scale = x.scale, a.ldy = ldy, a.ldx = x.ld, a.srows = f8_scale_rows(T), a.u = u, a.v = v, a.dA = dA, a.dB = dB, a.part = part;
  a.u_step = (int64_t)T * d.Rp, a.u_slices = f8_down_slices(T, d.N, d.I, true), a.v_slices = f8_down_slices(T, d.N, d.O, true), a.Rp = d.Rp;
  a.N = d.N, a.R = d.R, a.I = d.I, a.O = d.O, a.blocks_o = f8_blocks(d.O), a.chunk = chunk_of(T, d.I, d.O);
  a.src = x.dtype == BSP_BF16 ? kBf16 : x.dtype == BSP_E4M3 ? kE4 : kE5;
  a.each = T <= a.chunk;
  const int64_t chunks = a.each ? d.N : (int64_t)T / a.chunk + (T < d.N ? T : d.N);
  const dim3 grid((unsigned)(a.blocks_o + f8_blocks(d.I)), (unsigned)chunks, d.Rp == 128 ? 2 : 1);  // (128 ranks in two halves)
  if (chunks > 65535 || !f8_fits_x(grid.x, 256)) return BSP_ERR_SHAPE;
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (d.Rp == 16) run(adapt_grad<16>);
  else if (d.Rp == 32) run(adapt_grad<32>);
  else run(adapt_grad<64>);
  if (launched() != BSP_OK) return BSP_ERR_HIP;
  if (a.each) return BSP_OK;
  const int64_t groups = ((int64_t)d.R * (d.I + (int64_t)d.O) + 1023) / 1024;
  hipLaunchKernelGGL(adapt_join, dim3((unsigned)(groups < 4096 ? groups : 4096), (unsigned)d.N), dim3(256), 0, st, a);
  return launched();
}
