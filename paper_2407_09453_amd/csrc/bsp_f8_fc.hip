// FC layers on many rows, weights and activations in 8-bit codes: Y = act(X W^t + b + residual), bound by the matrix cores.
//
// A workgroup owns 32 to 256 rows by one or two block rows of 128 channels and walks the block columns that its block rows keep (two: where
// all are kept); a step is 128 columns, both operands staged in LDS with 16-byte asynchronous copies, two to four buffers
// deep.  The weights are the matrix core's rows and the activations its columns, so a lane's four neighbouring results
// are neighbouring channels of one row of Y, and an activation's scale is one byte a lane.
// A staged row of 128 bytes is eight pieces of 16; piece p of row r lies at place p ^ (r / 2 mod 8), so sixteen rows' same
// piece, which sixteen lanes read together, lie in sixteen different bank groups.
// MO x MT tiles of 32 x 32 a wave, WO x WT waves.
// Measured: 8192 x 16384 -> 4096 390 to 440 us (2.8 to 2.5 PFLOP/s), 16384 x 4096 -> 16384 870 (2.5), 2048 x 4096 -> 4096 35, 512 x 4096 -> 4096 14.5 to 16.5,
// 197 x 2048 -> 1000 7 (fp32 results 10).  On constant operands the first two take 306 and 702 us: with random codes the card's power sets the clock, and what the
// loop leaves (91 % of a register loop's rate) is little.
// With a residual the same take 560, 1850, 59, 21 and 8.4: its values (and for fp32 results the bias too) are asked for a row at a time in the way
// out (store_tile's first branch), each waited for before the next.
#include "bsp_f8.h"
#include <type_traits>

namespace {

struct TileArgs {
  F8Rows w;
  const uint8_t *X, *scale;
  F8Epilogue q;
  int64_t ld, srows;
  int32_t T, tiles_t, tiles_o;
  float* part;  // split > 1: sums of each share of the block columns, [split][T][4 ceil(out / 4)], instead of results
  int32_t split;
  int32_t full;  // blocks in a block row, where all are kept; else 0
  F8Low low;
};

__device__ __forceinline__ i32x8_t read_fragment(const uint8_t* p, int at0, int at1) {
  const u32x4_t a = *(const u32x4_t*)(p + at0), b = *(const u32x4_t*)(p + at1);
  return i32x8_t{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

__device__ __forceinline__ f32x16_t mfma_bf16_32x32x16(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// A wave's results, 32 MO channels of 32 MT rows, to Y.  In the accumulators a lane holds four channels of a row, and stored from there a
// request would touch 32 rows.  So 32 rows at a time pass through LDS (the wave's own part, each row 16 bytes longer than
// its values, in fp32 where a residual is still to be added) and leave as whole 64 MO-byte pieces of rows.
template <int MO>
constexpr int kStoreBytes = 32 * (32 * MO * 4 + 16);

// order: where the rows go, or null: they go as they come.
template <int MO, int MT, bool F32, bool LOW>
__device__ __forceinline__ void store_tile(const F8Epilogue& q, f32x16_t (&acc)[MO][MT], uint8_t* lds, int T, int O, int64_t t0, int o0, const int32_t* order) {
  const int lane = threadIdx.x & 63;
  constexpr int kLanes = 4 * MO;  // lanes that hold a row's piece, eight channels each
  const int c = o0 + (lane % kLanes) * 8;
  if (F32 || q.residual) {  // fp32 through LDS, then four channels at a time
    constexpr int kRow = 32 * MO * 4 + 16;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int o = 0; o < MO; ++o)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          *(f32x4_t*)(lds + (lane & 31) * kRow + (o * 32 + k * 8 + (lane >> 5) * 4) * 4) =
              f32x4_t{acc[o][m][4 * k], acc[o][m][4 * k + 1], acc[o][m][4 * k + 2], acc[o][m][4 * k + 3]};
#pragma unroll 1
      for (int r = lane / (8 * MO); r < 32; r += 8 / MO) {
        int64_t t = t0 + m * 32 + r;
        const int ch = o0 + (lane % (8 * MO)) * 4;
        const f32x4_t v = *(const f32x4_t*)(lds + r * kRow + (lane % (8 * MO)) * 16);
        if (t >= T || ch >= O) continue;
        if (LOW && order) t = order[t];
        f8_store4<F32>(q, t, ch, O, v[0], v[1], v[2], v[3]);
      }
    }
    return;
  }
  constexpr int kRow = 32 * MO * 2 + 16;
  f32x4_t bias[MO][4] = {};
  if (q.bias) {
#pragma unroll
    for (int o = 0; o < MO; ++o)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int ch = o0 + o * 32 + k * 8 + (lane >> 5) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[o][k][e] = q.bias[ch + e < O ? ch + e : O - 1];
      }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int o = 0; o < MO; ++o)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = acc[o][m][4 * k + e] + bias[o][k][e];
          if (q.relu) v[e] = v[e] < 0.f ? 0.f : v[e];
        }
        *(u32x2_t*)(lds + (lane & 31) * kRow + (o * 32 + k * 8 + (lane >> 5) * 4) * 2) = u32x2_t{f8_pack_bf16x2(v[0], v[1]), f8_pack_bf16x2(v[2], v[3])};
      }
    auto rows = [&](auto WHOLE) {  // of whole pieces; or of pieces at any address, which share lines with others
#pragma unroll 4
      for (int r = lane / kLanes; r < 32; r += 64 / kLanes) {
        int64_t t = t0 + m * 32 + r;
        u32x4_t v = *(const u32x4_t*)(lds + r * kRow + (lane % kLanes) * 16);
        if (t >= T || c >= O) continue;
        if (LOW && order) t = order[t];
        if (q.gate) {
          const u32x2_t g = *(const u32x2_t*)(q.gate + t * (int64_t)f8_blocks(O) * F8_BLOCK + c);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!f8_positive((g[e >> 2] >> (8 * (e & 3))) & 0xFFu, q.gate_e5)) v[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
        uint16_t* y = (uint16_t*)q.Y + t * O + c;
        if constexpr (decltype(WHOLE)::value) {
          __builtin_nontemporal_store(v, (u32x4_t*)y);
        } else if (c + 8 <= O) {
          *(u32x4_any*)y = v;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + e < O) y[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
        }
      }
    };
    if (O % 8 == 0) rows(std::true_type{});
    else rows(std::false_type{});
  }
}

// The wait between a matrix instruction and the first use of its result, by hand: where two ways meet again behind it, a branch that is taken or
// not, the compiler counts the instructions of one of them, be it the longer (found where channel 31 of a result lost its second part).
__device__ __forceinline__ void settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <int PARTS>
struct LowParts {
  u32x4_t part[PARTS];
};
template <int PARTS, int ASK>  // ASK: slices asked for together
__device__ __forceinline__ LowParts<PARTS> low_parts(const F8Low& low, const float* u) {
  f32x4_t x0 = *(const f32x4_t*)u, x1 = *(const f32x4_t*)(u + 4);
#pragma unroll 1
  for (int s = 1; s < low.slices; s += ASK) {  // (two, four or eight)
    f32x4_t y0[ASK], y1[ASK];
#pragma unroll
    for (int e = 0; e < ASK; ++e) {
      const float* v = u + (s + e < low.slices ? s + e : s) * low.u_step;
      y0[e] = *(const f32x4_t*)v, y1[e] = *(const f32x4_t*)(v + 4);
    }
#pragma unroll
    for (int e = 0; e < ASK; ++e)
      if (s + e < low.slices) x0 += y0[e], x1 += y1[e];
  }
  LowParts<PARTS> p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a0 = (e < 2 ? x0 : x1)[2 * (e & 1)], a1 = (e < 2 ? x0 : x1)[2 * (e & 1) + 1];
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      p.part[i][e] = f8_pack_bf16x2(a0, a1);
      a0 -= __uint_as_float(p.part[i][e] << 16), a1 -= __uint_as_float(p.part[i][e] & 0xFFFF0000u);
    }
  }
  return p;
}
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2_t;
// A fragment's rows by themselves, where they belong to more than sixteen adapters: a lane multiplies its row's u with its own adapter's weights,
// sixteen channels of every 32, with ordinary instructions (us, an adapter at a time and so: 64 x 512 -> 16384 of 64 adapters 18 and 13.6, of rank 64
// 64 x 4096 -> 4096 41 and 31, 512 of 512 32 and 26).  Not in the widest tiles (16384 x 4096 -> 4096 of 32 mixed as they come: 428 and 496).
constexpr int kManyAdapters = 16;
template <int MO, int MT>
__device__ __forceinline__ void add_low_rows(const F8Low& low, f32x16_t (&acc)[MO][MT], int m, const float* u, int of, int o0) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint16_t* b = low.up + (of < 0 ? 0 : of) * low.step + (int64_t)o0 * low.rank + 4 * half * 8;
  for (int k = 0; k < low.rank; k += 16) {
    f32x4_t x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = *(const f32x4_t*)(u + k + 4 * e);
    for (int s = 1; s < low.slices; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += *(const f32x4_t*)(u + s * low.u_step + k + 4 * e);
#pragma unroll
    for (int o = 0; o < MO; ++o)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint16_t* c = b + (int64_t)o * 32 * low.rank + k * 32 + q * 64;
        u32x4_t w[4][2];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < 2; ++h) w[e][h] = *(const u32x4_t*)(c + e * 8 + h * 256);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float s = 0.f;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              s = fmaf(__uint_as_float(w[e][h][i] << 16), x[2 * h + (i >> 1)][2 * (i & 1)], s);
              s = fmaf(__uint_as_float(w[e][h][i] & 0xFFFF0000u), x[2 * h + (i >> 1)][2 * (i & 1) + 1], s);
            }
          acc[o][m][4 * q + e] += of >= 0 ? s : 0.f;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
}

// The rows' adapters: B_a u_t added to a wave's sums, one adapter of its rows after the other, the next ones' weights asked for while one is
// multiplied.  u enters as two bf16 parts (for fp32 results three), as zeros in the rows of other adapters: the rows are the matrix instruction's
// columns, and the sums go on where they are.  Zero times what is no number is none: an adapter with such weights among its rows'
// neighbours is multiplied from zero, and a lane, which holds results of one row, takes or leaves what it gives.
// Bound by the instructions of each adapter among a wave's rows, behind a product that leaves none of their time free (16384 x 4096 -> 4096 of rank
// 16, us: the product 225 to 250, with adapters 15 to 20 more; 64 x 4096 -> 16384 15, with 32 adapters' rows mixed 25).
// order: the rows' numbers where they are not multiplied as they come.
template <int MO, int MT, int PARTS>
__device__ __forceinline__ void add_low(const F8Low& low, f32x16_t (&acc)[MO][MT], int T, int64_t t0, int o0, const int32_t* order) {
  const int lane = threadIdx.x & 63;
  const uint16_t* up = low.up + (int64_t)o0 * low.rank + lane * 8;  // (as the instruction takes them: 32 channels, sixteen ranks, 64 lanes)
  const float* u[MT];
  int of[MT];
  uint64_t all[MT];
  settle();
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    int64_t t = t0 + m * 32 + (lane & 31) < T ? t0 + m * 32 + (lane & 31) : T - 1;
    if (order) t = order[t];
    u[m] = low.u + t * low.rank + (lane >> 5) * 8;
    of[m] = low.which[t];
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    all[m] = __ballot(of[m] >= 0);
    if constexpr (MO < 4) {
      uint64_t rest = all[m];
      for (int n = 0; rest && n < kManyAdapters; ++n) rest &= ~__ballot(of[m] == __builtin_amdgcn_readlane(of[m], __builtin_ctzll(rest)));
      if (!rest) continue;
      all[m] = 0;
      add_low_rows<MO, MT>(low, acc, m, u[m] - (lane >> 5) * 8, of[m], o0);
    }
  }
  for (int k = 0; k < low.rank; k += 16) {
    constexpr int kAhead = MO == 4 ? 2 : MT == 2 ? 4 : 8;
    uint64_t todo[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) todo[m] = all[m];
    int now[kAhead], last = 0;
    u32x4_t w[kAhead][MO];
    // (asked for without a condition, once more the last one's where there is no next: a wait can then be by count)
    auto ask = [&](int d) {
      int next = -1;
#pragma unroll
      for (int m = MT - 1; m >= 0; --m)
        if (todo[m]) next = __builtin_amdgcn_readlane(of[m], __builtin_ctzll(todo[m]));
#pragma unroll
      for (int m = 0; m < MT; ++m) todo[m] &= ~__ballot(of[m] == next);
      now[d] = next;
      last = next >= 0 ? next : last;
      const uint16_t* b = up + last * low.step + k * 32;
#pragma unroll
      for (int o = 0; o < MO; ++o) w[d][o] = *(const u32x4_t*)(b + (int64_t)o * 32 * low.rank);
    };
#pragma unroll
    for (int d = 0; d < kAhead; ++d) ask(d);
    LowParts<PARTS> p[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) p[m] = low_parts<PARTS, MO == 4 ? 1 : 3>(low, u[m] + k);
    while (now[0] >= 0) {
#pragma unroll
      for (int d = 0; d < kAhead; ++d) {
        if (now[d] >= 0) {
          // an exponent of ones in any half of the weights' words
          u16x2_t most = {0, 0};
#pragma unroll
          for (int o = 0; o < MO; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, w[d][o][e] & 0x7F807F80u));
          const bool odd = __any(most.x == 0x7F80 || most.y == 0x7F80);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const bool mine = of[m] == now[d];
            if (!__any(mine)) continue;
            if (!odd || __all(mine)) {
#pragma unroll
              for (int i = 0; i < PARTS; ++i) {
                u32x4_t v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mine ? p[m].part[i][e] : 0;
#pragma unroll
                for (int o = 0; o < MO; ++o) acc[o][m] = mfma_bf16_32x32x16(w[d][o], v, acc[o][m]);
              }
            } else {
              settle();
#pragma unroll
              for (int o = 0; o < MO; ++o) {
                f32x16_t sum = {};
#pragma unroll
                for (int i = 0; i < PARTS; ++i) sum = mfma_bf16_32x32x16(w[d][o], p[m].part[i], sum);
                asm volatile("" : "+v"(sum));  // (read in the block of the instruction that makes it)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[o][m][e] += mine ? sum[e] : 0.f;
                __builtin_amdgcn_sched_barrier(0);
              }
            }
          }
        }
        ask(d);
      }
    }
  }
  settle();
}

// Which tile a workgroup takes: workgroups go to the eight XCDs in turn, an XCD takes an eighth of the tiles, and its tiles follow one another
// in bands of four tiles of channels, so that what it runs at one time (32) shares four tiles' weights and eight tiles' rows in its L2.
__device__ __forceinline__ void place_tile(int b, int tiles_o, int tiles_t, int* to, int* tt) {
  const int total = tiles_o * tiles_t, each = total >> 3, more = total & 7, xcd = b & 7;
  const int j = xcd * each + (xcd < more ? xcd : more) + (b >> 3);
  const int band = j / (4 * tiles_t), r = j - band * 4 * tiles_t;
  const int wide = tiles_o - band * 4 < 4 ? tiles_o - band * 4 : 4;
  *to = band * 4 + r % wide;
  *tt = r / wide;
}

// ------------------------------------------------------------------ the kernel
// A wave overlaps its own work: it reads one half of a step (64 columns) while it multiplies the other, and one barrier a step,
// between the halves, both frees the buffer that all have read and hands over the one that has landed.  The copies of the
// step BUFS later then go into the buffer just freed and have BUFS - 1 steps to arrive; a wave waits for its own copies of
// the next step by their count, not for all that it has asked for.
template <int MO, int MT, int WO, int WT, int BUFS>
struct Wide {
  static constexpr int NO = 32 * MO * WO, NT = 32 * MT * WT, WAVES = WO * WT, R = NO / F8_BLOCK;
  static constexpr int QO = NO / 8 / WAVES, QT = NT / 8 / WAVES, COPIES = QO + QT + 1;  // requests a wave and step: weights, rows, the rows' scales
  static constexpr int SCALES = (NO + NT) * F8_BLOCK;                                   // where they lie in a buffer
  static constexpr int STAGE = SCALES + WAVES * 256;  // (a request is 256 bytes, 32 MT of them scales that the wave wants)
  static constexpr int kStored = WAVES * kStoreBytes<MO>;
  static constexpr int kLds = BUFS * STAGE > kStored ? BUFS * STAGE : kStored;
  static_assert(WAVES % 2 == 0 && NO % F8_BLOCK == 0 && NO % (8 * WAVES) == 0 && NT % (8 * WAVES) == 0 && kLds <= 160 * 1024);

  const uint8_t *payload, *X, *S;  // first block; the tile's rows, and their scales
  int64_t srows;
  int cnt, wave;
  uint32_t from_w, from_x[QT], from_s;  // this lane's places in a request
  int at[2][2], at_s, at_w, at_x;

  // 64 lanes x 16 bytes from `base` (the same in every lane) + at.  The base is hidden from the optimiser, which would keep base + at
  // of every request in two registers a lane each through the loop.
  static __device__ __forceinline__ void request(const uint8_t* base, uint32_t at, uint8_t* to) {
    asm volatile("" : "+s"(base));
    __builtin_amdgcn_global_load_lds((f8_gptr_t)(base + at), (f8_lptr_t)to, 16, 0, 0);
  }
  __device__ __forceinline__ void copy(uint8_t* to, int i, int kb) const {
    const uint8_t* w = payload + (int64_t)i * F8_BLOCK_BYTES;
    const uint8_t* x = X + (int64_t)kb * F8_BLOCK;
#pragma unroll
    for (int q = 0; q < QO; ++q) {
      const int row = q * 8 * WAVES;
      request(w + (R == 1 ? 0 : (int64_t)(row >> 7) * cnt * F8_BLOCK_BYTES) + (row & 127) * F8_BLOCK, from_w, to + wave * 1024 + row * F8_BLOCK);
    }
#pragma unroll
    for (int q = 0; q < QT; ++q) request(x, from_x[q], to + wave * 1024 + (NO + q * 8 * WAVES) * F8_BLOCK);
    const uint8_t* s = S + (int64_t)kb * srows;
    asm volatile("" : "+s"(s));
    __builtin_amdgcn_global_load_lds((f8_gptr_t)(s + from_s), (f8_lptr_t)(to + SCALES + wave * 256), 4, 0, 0);
  }
  __device__ __forceinline__ void read(const uint8_t* from, int h, i32x8_t (&w)[MO], i32x8_t (&x)[MT]) const {
#pragma unroll
    for (int o = 0; o < MO; ++o) w[o] = read_fragment(from + at_w + o * 32 * F8_BLOCK, at[h][0], at[h][1]);
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = read_fragment(from + at_x + m * 32 * F8_BLOCK, at[h][0], at[h][1]);
  }
  __device__ __forceinline__ void read_scales(const uint8_t* from, int (&s)[MT]) const {
#pragma unroll
    for (int m = 0; m < MT; ++m) s[m] = from[at_s + m * 32];
  }
  // F32: as bf16, so that nothing is lost in the sum (see f8_few)
  template <bool E5, bool F32>
  static __device__ __forceinline__ void multiply(i32x8_t (&w)[MO], i32x8_t (&x)[MT], int sw, int (&sx)[MT], f32x16_t (&acc)[MO][MT]) {
    if constexpr (F32) {
      const float fw = __uint_as_float((uint32_t)sw << 23);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4_t wj[MO], xj[MT];
#pragma unroll
        for (int o = 0; o < MO; ++o) wj[o] = f8_decode_bf16x8<false>(w[o][2 * j], w[o][2 * j + 1], fw);
#pragma unroll
        for (int m = 0; m < MT; ++m) xj[m] = f8_decode_bf16x8<E5>(x[m][2 * j], x[m][2 * j + 1], __uint_as_float((uint32_t)sx[m] << 23));
#pragma unroll
        for (int o = 0; o < MO; ++o)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[o][m] = mfma_bf16_32x32x16(wj[o], xj[m], acc[o][m]);
      }
      return;
    }
#pragma unroll
    for (int o = 0; o < MO; ++o)
#pragma unroll
      for (int m = 0; m < MT; ++m)
        acc[o][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[o], x[m], acc[o][m], 0, E5 ? 1 : 0, 0, sw, 0, sx[m]);
  }

  // Step i, whose first half has been read.  LATER: steps to come that have been asked for (all of the BUFS - 1 that fit in the
  // main loop, where this step asks for one more).  `to` is written behind the barrier alone, `from` and `next` are other
  // bytes by then: the compiler need not order its reads of LDS behind copies in flight, the waits here do.
  template <bool E5, bool F32, int LATER, bool MORE>
  __device__ __forceinline__ void step(uint8_t* __restrict__ to, const uint8_t* __restrict__ from, const uint8_t* __restrict__ next, int i, int sw, int kb,
                                       i32x8_t (&w)[2][MO], i32x8_t (&x)[2][MT], int (&sx)[2][MT], f32x16_t (&acc)[MO][MT]) const {
    constexpr int N = MO * MT, kRead = 2 * (MO + MT);
    read(from, 1, w[1], x[1]);
    multiply<E5, F32>(w[0], x[0], sw, sx[0], acc);
    if constexpr (!F32)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                   // one matrix instruction,
      __builtin_amdgcn_sched_group_barrier(0x100, (kRead + N - 1) / N, 0);  // and what it hides: reads of LDS
    }
    constexpr int kLeft = LATER > 0 ? (LATER - 1) * COPIES : 0;
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft) : "memory");  // step i + 1 has landed, and this wave has read step i
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    constexpr int kHalf = (N + 1) / 2;
    if constexpr (LATER > 0) {
      read_scales(next, sx[1]);
      read(next, 0, w[0], x[0]);
    }
    if constexpr (MORE) copy(to, i + BUFS, kb);
    multiply<E5, F32>(w[1], x[1], sw, sx[0], acc);
    if constexpr (!F32) {
#pragma unroll
    for (int k = 0; k < kHalf; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (LATER > 0) __builtin_amdgcn_sched_group_barrier(0x100, (kRead + MT + kHalf - 1) / kHalf, 0);
    }
#pragma unroll
    for (int k = 0; k < kHalf; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (MORE) __builtin_amdgcn_sched_group_barrier(0x020, (COPIES + kHalf - 1) / kHalf, 0);  // copies to LDS
    }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) sx[0][m] = sx[1][m];
  }
};

// LOW: with adapters beside the layer.
template <int MO, int MT, int WO, int WT, int BUFS, bool E5, bool F32, bool LOW>
__device__ __forceinline__ void wide(const TileArgs& a, uint8_t* lds) {
  using K = Wide<MO, MT, WO, WT, BUFS>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wo = wave / WT, wt = wave % WT;
  // a share of the block columns, and the tile
  constexpr bool kSplits = MO * MT <= 4;
  const int tiles = a.tiles_o * a.tiles_t, share = kSplits ? (int)blockIdx.x / tiles : 0;
  int tile_o, tile_t;
  place_tile((int)blockIdx.x - share * tiles, a.tiles_o, a.tiles_t, &tile_o, &tile_t);
  const int br = tile_o * K::R;
  const int64_t t0 = (int64_t)tile_t * K::NT;
  // (where all blocks are kept their places need not be read)
  const auto* ptr = (const __attribute__((address_space(4))) int32_t*)a.w.ptr;
  int n0 = a.full ? br * a.full : ptr[br], cnt = a.full ? a.full : ptr[br + 1] - n0, col_first = 0;
  if constexpr (kSplits) {
    const int from = (int)((int64_t)cnt * share / a.split), to = (int)((int64_t)cnt * (share + 1) / a.split);
    n0 += from;
    col_first = from;
    cnt = to - from;
  }
  const int last = (int)(a.T - 1 - t0 < K::NT - 1 ? a.T - 1 - t0 : K::NT - 1);  // rows past the last: its bytes, their results go nowhere

  K k;
  k.payload = a.w.payload + (int64_t)n0 * F8_BLOCK_BYTES;
  const bool mixed = LOW && a.low.mixed && *(const __attribute__((address_space(4))) int32_t*)a.low.mixed;
  k.X = (mixed ? a.low.codes : a.X) + t0 * a.ld;
  k.S = (mixed ? a.low.scale : a.scale) + t0;
  k.srows = a.srows;
  k.cnt = cnt;
  k.wave = wave;
  // this lane's 16 bytes of a request of eight rows
  const int srow = wave * 8 + (lane >> 3), piece = ((lane & 7) ^ ((srow >> 1) & 7)) * 16;
  k.from_w = srow * F8_BLOCK + piece;
#pragma unroll
  for (int q = 0; q < K::QT; ++q) {
    const int row = srow + q * 8 * K::WAVES;
    k.from_x[q] = (uint32_t)(row < last ? row : last) * (uint32_t)a.ld + piece;
  }
  // four rows' scales a lane; a scale array's last four bytes for rows past it
  const int64_t s_end = a.srows - 4 - t0;
  k.from_s = (uint32_t)(wt * MT * 32 + lane * 4 < s_end ? wt * MT * 32 + lane * 4 : s_end);
  // the pieces that this lane reads of its row of a fragment, for the two halves of a step
  const int f = (lane >> 1) & 7, g2 = (lane >> 5) * 2;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int q = 0; q < 2; ++q) k.at[h][q] = (lane & 31) * F8_BLOCK + (((4 * h + g2 + q) ^ f) << 4);
  k.at_w = wo * MO * 32 * F8_BLOCK;
  k.at_x = (K::NO + wt * MT * 32) * F8_BLOCK;
  k.at_s = K::SCALES + wave * 256 + (lane & 31);

  f32x16_t acc[MO][MT] = {};
  if (cnt > 0) {
    const int32_t* idx = a.w.idx + n0;
    const uint8_t* scl = a.w.scale + n0 + (K::R == 1 ? 0 : ((wo * MO * 32) >> 7) * cnt);
    // block columns and weight scales, one a lane: of the first steps, of those that the loop below asks for (64 at a time) and goes through, of the last
    auto column = [&](int i) { return a.full ? col_first + (i < cnt ? i : cnt - 1) : idx[i < cnt ? i : cnt - 1]; };
    auto scale = [&](int i) { return (int)scl[i < cnt ? i : cnt - 1]; };
    const int tail = cnt > BUFS ? cnt - BUFS : 0;
    const int col0 = column(lane);
    int cols = column(lane + BUFS), scales = scale(lane), tail_scales = scale(tail + lane);
#pragma unroll
    for (int j = 0; j < BUFS; ++j)
      if (j < cnt) k.copy(lds + j * K::STAGE, j, __builtin_amdgcn_readlane(col0, j));
    i32x8_t w[2][MO], x[2][MT];
    int sx[2][MT];
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(cols), "+v"(scales), "+v"(tail_scales)::"memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    k.read_scales(lds, sx[0]);
    k.read(lds, 0, w[0], x[0]);
    int cur = 0;
    auto following = [](int b) { return b == (BUFS - 1) * K::STAGE ? 0 : b + K::STAGE; };
    for (int c = 0; c < cnt - BUFS; c += 64) {
      if (c > 0) {
        cols = column(c + lane + BUFS), scales = scale(c + lane);
        asm volatile("s_waitcnt vmcnt(0)" : "+v"(cols), "+v"(scales)::"memory");
      }
      const int end = c + 64 < cnt - BUFS ? c + 64 : cnt - BUFS;
      for (int i = c; i < end; ++i) {
        const int nxt = following(cur);
        k.template step<E5, F32, BUFS - 1, true>(lds + cur, lds + cur, lds + nxt, i, __builtin_amdgcn_readlane(scales, i - c),
                                            __builtin_amdgcn_readlane(cols, i - c), w, x, sx, acc);
        cur = nxt;
      }
    }
    auto rest = [&](auto later) {  // the step with `later` steps behind it
      constexpr int L = decltype(later)::value;
      if (cnt > L) {
        const int nxt = following(cur);
        k.template step<E5, F32, L, false>(lds + cur, lds + cur, lds + nxt, 0, __builtin_amdgcn_readlane(tail_scales, cnt - 1 - L - tail), 0, w, x, sx, acc);
        cur = nxt;
      }
    };
    if constexpr (BUFS > 3) rest(std::integral_constant<int, 3>{});
    if constexpr (BUFS > 2) rest(std::integral_constant<int, 2>{});
    rest(std::integral_constant<int, 1>{});
    rest(std::integral_constant<int, 0>{});
  }
  const int32_t* order = mixed ? a.low.order : nullptr;
  if constexpr (LOW)
    if (share == 0) add_low<MO, MT, F32 ? 3 : 2>(a.low, acc, a.T, t0 + wt * MT * 32, tile_o * K::NO + wo * MO * 32, order);
  __syncthreads();
  if constexpr (kSplits) {
    if (a.split > 1) {
      const int ld = (a.w.out + 3) & ~3;
      const F8Epilogue sums{a.part + (int64_t)share * a.T * ld, nullptr, nullptr, nullptr, 0, 0};
      store_tile<MO, MT, true, LOW>(sums, acc, lds + wave * kStoreBytes<MO>, a.T, ld, t0 + wt * MT * 32, tile_o * K::NO + wo * MO * 32, order);
      return;
    }
  }
  store_tile<MO, MT, F32, LOW>(a.q, acc, lds + wave * kStoreBytes<MO>, a.T, a.w.out, t0 + wt * MT * 32, tile_o * K::NO + wo * MO * 32, order);
}

template <int MO, int MT, int WO, int WT, int BUFS, bool E5, bool F32>
__global__ __launch_bounds__(64 * WO * WT) void f8_wide(TileArgs a) {
  extern __shared__ uint8_t lds[];
  kernarg_touch<TileArgs>();
  wide<MO, MT, WO, WT, BUFS, E5, F32, false>(a, lds);
}
template <int MO, int MT, int WO, int WT, int BUFS, bool E5, bool F32>
__global__ __launch_bounds__(64 * WO * WT) void f8_wide_low(TileArgs a) {
  extern __shared__ uint8_t lds[];
  kernarg_touch<TileArgs>();
  wide<MO, MT, WO, WT, BUFS, E5, F32, true>(a, lds);
}

// The shares' sums, in their order, and what follows a product: a thread takes four channels of a row.
template <bool F32>
__global__ __launch_bounds__(256) void f8_join(const float* part, int split, int T, int O, F8Epilogue q) {
  const int quads = (O + 3) >> 2;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = i / quads, rows = (int64_t)T * quads;
  if (i >= rows) return;
  f32x4_t s = {};
#pragma unroll 8
  for (int k = 0; k < split; ++k) s += *(const f32x4_t*)(part + (k * rows + i) * 4);
  f8_store4<F32>(q, t, (int)(i - t * quads) * 4, O, s[0], s[1], s[2], s[3]);
}

template <int NO, int NT>
int launch(void (*kernel)(TileArgs), bool raised, int threads, int lds, TileArgs a, hipStream_t st) {
  if (!raised) return BSP_ERR_HIP;
  a.tiles_o = (a.w.out + NO - 1) / NO;
  a.tiles_t = (int)(((int64_t)a.T + NT - 1) / NT);
  if (!f8_fits_x((int64_t)a.tiles_o * a.tiles_t * a.split, threads)) return BSP_ERR_SHAPE;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles_o * a.tiles_t * a.split)), dim3(threads), lds, st, a);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}
bool raise(const void* kernel, int lds) { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess; }

template <int MO, int MT, int WO, int WT, int BUFS, bool E5, bool F32, bool LOW>
int launch_wide(const TileArgs& a, hipStream_t st) {
  using K = Wide<MO, MT, WO, WT, BUFS>;
  constexpr auto kernel = LOW ? &f8_wide_low<MO, MT, WO, WT, BUFS, E5, F32> : &f8_wide<MO, MT, WO, WT, BUFS, E5, F32>;
  static const bool raised = raise((const void*)kernel, K::kLds);
  return launch<K::NO, K::NT>(kernel, raised, 64 * K::WAVES, K::kLds, a, st);
}

// Which tile: the smaller of the chip's rate on it and of the steps' own latency, one after the other.  `alone`: us a step where a CU has one
// workgroup, `shared`: where it has as many as fit; `rate`: TFLOP/s of padded work with the chip full.  Measured on
// T x I -> O of 65 .. 16384 x 512 .. 16384 -> 512 .. 16384, all blocks kept and half of them (us; 256x256, 128x256, 128x128, 128x64, 128x32):
//   16384 x 4096 -> 16384  873 1079 1062 1307 2439     2048 x 4096 -> 4096  44 35 34 43 80     512 x 4096 -> 4096  43 30 23 15 21
//   65 x 4096 -> 4096  37 29 18 13.5 11     4096 x 512 -> 512  12 9.5 6.6 5.8 7.2     2048 x 4096 -> 4096, half kept  - 24 25 29 57
struct Tile {
  int o, t, fit;
  double alone, shared, rate;
};
constexpr Tile kTiles[] = {{256, 256, 1, 1.15, 1.15, 2500}, {128, 256, 1, 0.75, 0.75, 2150}, {128, 128, 2, 0.40, 0.85, 2200}, {128, 64, 2, 0.25, 0.50, 1700}, {128, 32, 1, 0.18, 0.18, 1000}};

struct Plan {
  int tile, split;
};
// Where tiles are too few for the chip the block columns are cut into shares, of at least four steps each, whose sums a second launch joins: that
// costs it 3 us and the memory's time (us, one share and as planned: 243 x 18816 -> 384 40 and 15.3, 256 x 16384 -> 1024 35 and 19.5).
// fp32 results take twice the time a step, at half the rate (64 x 4096 -> 4096 fp32 17.2 us in one share, 13.6 in two, 8192 x 4096 -> 4096 1180 TFLOP/s).
Plan plan_of(int O, int64_t nnzb, int T, bool full, bool f32) {
  const double steps = (double)nnzb / f8_blocks(O);
  Plan best{2, 1};
  double least = 1e30;
  for (int k = f32 ? 2 : full && f8_blocks(O) % 2 == 0 ? 0 : 1; k < 5; ++k) {
    const Tile& v = kTiles[k];
    const double groups = (double)((f8_blocks(O) * F8_BLOCK + v.o - 1) / v.o) * (double)(((int64_t)T + v.t - 1) / v.t);
    for (int split = 1; split == 1 || (k >= 2 && groups * split <= 256 && steps >= 4.0 * split && split <= 64); split *= 2) {
      const double all = groups * split;
      const double rounds = all <= 256 ? v.alone : v.shared * (double)(int64_t)((all + 256 * v.fit - 1) / (256 * v.fit));
      const double us = rounds * steps / split, at_rate = groups * steps * v.o * v.t * 256e-6 / v.rate;
      const double join = split > 1 ? 3.0 + (double)T * O * 4 * 2 * split / 3e6 : 0;
      const double worse = (us > at_rate ? us : at_rate) * (f32 ? 2.1 : 1) + join;
      if (worse < least) least = worse, best = Plan{k, split};
    }
  }
  return best;
}

template <bool E5, bool LOW>
int launch_any(const TileArgs& a, int k, bool f32, hipStream_t st) {
  if (f32) {
    switch (k) {
      case 3: return launch_wide<2, 1, 2, 2, 3, E5, true, LOW>(a, st);
      case 4: return launch_wide<1, 1, 4, 1, 4, E5, true, LOW>(a, st);
      default: return launch_wide<2, 2, 2, 2, 2, E5, true, LOW>(a, st);
    }
  }
  switch (k) {
    case 0: return launch_wide<4, 2, 2, 4, 2, E5, false, LOW>(a, st);
    case 1: return launch_wide<4, 2, 1, 4, 3, E5, false, LOW>(a, st);
    case 2: return launch_wide<2, 2, 2, 2, 2, E5, false, LOW>(a, st);
    case 3: return launch_wide<2, 1, 2, 2, 3, E5, false, LOW>(a, st);
    default: return launch_wide<1, 1, 4, 1, 4, E5, false, LOW>(a, st);
  }
}

}  // namespace

namespace {
bool all_kept(const F8Rows& w) { return w.nnzb == (int64_t)f8_blocks(w.out) * f8_blocks(w.in); }
}  // namespace

int f8_tile_split(const F8Rows& w, int T, bool f32) { return plan_of(w.out, w.nnzb, T, all_kept(w), f32).split; }

int f8_launch_tile(const F8Rows& w, const F8Input& x, int T, const F8Low& low, const F8Epilogue& q, bool f32, float* part, hipStream_t st) {
  const bool full = all_kept(w);
  const Plan plan = plan_of(w.out, w.nnzb, T, full, f32);
  TileArgs a{w, (const uint8_t*)x.X, x.scale, q, x.ld, f8_scale_rows(T), T, 0, 0, part, plan.split, full ? f8_blocks(w.in) : 0, low};
  if (low.rank) return x.e5 ? launch_any<true, true>(a, plan.tile, f32, st) : launch_any<false, true>(a, plan.tile, f32, st);
  return x.e5 ? launch_any<true, false>(a, plan.tile, f32, st) : launch_any<false, false>(a, plan.tile, f32, st);
}

int f8_launch_join(const float* part, int split, int T, int O, const F8Epilogue& q, bool f32, hipStream_t st) {
  const int64_t groups = ((int64_t)T * ((O + 3) / 4) + 255) / 256;
  if (!f8_fits_x(groups, 256)) return BSP_ERR_SHAPE;
  if (f32) hipLaunchKernelGGL(f8_join<true>, dim3((unsigned)groups), dim3(256), 0, st, part, split, T, O, q);
  else hipLaunchKernelGGL(f8_join<false>, dim3((unsigned)groups), dim3(256), 0, st, part, split, T, O, q);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}
