// The weights' gradient of an FC layer from the 8-bit checkpoint of its input: dW[o][i] = sum_t dY[t][o] X[t][i] for kept blocks
// only, and the bias's, db[o] = sum_t dY[t][o].  Bound by the matrix cores and LDS on many rows (busy 48 and 45 % of the time), by the steps' latency on few:
// 8192, 4096 x 16384 1010 us (1.09 PFLOP/s), half of the blocks of 8192, 8192 x 8192 585, of 2048, 4096 x 4096 59; 4096, 512 x 512 20.
//
// A scale of the checkpoint belongs to a row t and 128 columns, and t is what the product sums over, so no scaled matrix
// instruction fits; code x power of two is exact in bf16, and the product runs on the bf16 matrix cores with fp32 sums.
// A workgroup takes one block row (128 outputs) and C of its kept blocks, whichever they are: the gradients' 128 columns are
// staged once for all of them.  Codes become bf16 on their way into LDS (a conversion of two values takes the scale along).
// Both operands are summed over their rows: LDS holds them as they lie in memory, row after row, and the transposing LDS read
// hands a lane four rows of its column.  It takes four rows of 32 bytes from a group of sixteen lanes, and half a wave two
// neighbouring chunks of them: the chunks of a row are permuted by the row (bits 0 and 1, then 3), so that these eight lie in different banks.
// Two buffers of 32 rows; what is written into one was asked for, into registers, two or four steps before.
// Where a matrix has too few blocks for the chip the rows are cut into ranges whose sums meet in a second launch, in order.
#include "bsp_f8.h"

#include <type_traits>

namespace {

constexpr int kStep = 32;  // rows a step
constexpr int kTile = kStep * 256;                     // 32 rows of 128 bf16

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef const __attribute__((address_space(1))) uint8_t* global_t;

__device__ __forceinline__ u32x4_t read_columns(const uint8_t* p) {  // rows +0..3 and +4..7 of this lane's column
  auto* q = (__attribute__((address_space(3))) s16x4_t*)(uintptr_t)p;
  const u32x2_t a = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q));
  const u32x2_t b = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + 4 * 256 / 8));
  return u32x4_t{a.x, a.y, b.x, b.y};
}

__device__ __forceinline__ int chunk_key(int t) { return (t & 3) << 1 | ((t >> 3) & 1); }

// the gradients of a row of fewer than eight, and zeros
__device__ __forceinline__ u32x4_t gradients_few(const uint16_t* row, int O) {
  uint32_t v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = row[k < O ? k : O - 1];
    v[k] = k < O ? v[k] : 0;
  }
  return u32x4_t{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
}

// Column sums of one block row's gradients over one range of rows: a thread adds eight columns of every 32nd (16th) row, eight rows asked for
// at once (2966 columns of 4052 rows: 22 us; one by one where a row ends inside a thread's columns 180).
template <int THREADS>
__device__ __forceinline__ void column_sums(const F8GradArgs& a, int br, int range, int64_t t_begin, int64_t t_end, float* sums) {
  constexpr int kRows = THREADS / 16, kAtOnce = 8;
  const int piece = threadIdx.x & 15, o = br * F8_BLOCK + piece * 8;
  const int from = o + 8 <= a.O || a.O < 8 ? o : a.O - 8;  // at a row's end its last eight
  float s[8] = {};
  auto add = [&](auto get) {
    for (int64_t t = t_begin + (threadIdx.x >> 4); t < t_end; t += kRows * kAtOnce) {
      u32x4_t v[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) v[j] = get(a.dY + (t + j * kRows < t_end ? t + j * kRows : t_end - 1) * a.ldy);
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += t + j * kRows < t_end ? __uint_as_float(k & 1 ? v[j][k >> 1] & 0xFFFF0000u : v[j][k >> 1] << 16) : 0.f;
    }
  };
  if (a.O < 8) {
    if (o < a.O) add([&](const uint16_t* row) { return gradients_few(row, a.O); });
  } else if (o < a.O) {
    add([&](const uint16_t* row) { return u32x4_t(*(const u32x4_any*)(row + from)); });
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (from + k >= o) sums[(threadIdx.x >> 4) * 129 + (from + k - br * F8_BLOCK)] = s[k];
  __syncthreads();
  if (threadIdx.x < F8_BLOCK && br * F8_BLOCK + (int)threadIdx.x < a.O) {
    float v = 0.f;
    for (int r = 0; r < THREADS / 16; ++r) v += sums[r * 129 + threadIdx.x];
    (a.split == 1 ? a.db : a.part_db + (int64_t)range * a.O)[br * F8_BLOCK + threadIdx.x] = v;
  }
}

// C blocks on WAVES waves: four and two of the workgroups, or three of one block, on a CU, or eight and one, or two of one block.  Four waves of one workgroup and four of
// another do not keep in step from barrier to barrier, and read less of LDS for each product (us at 2048 x 4096 -> 4096 half kept, one block: 61 on eight waves, 57.6
// on four; 4096 x 8192 -> 2048 110 and 102; 8192 x 4096 -> 16384, two blocks: 1115 and 1051); where a workgroup has a CU to itself eight waves are faster (37, 1000 x 520
// 7.9 and 9.8), and of four blocks four waves would be one a SIMD.
// E5: e5m2 codes.  THIN: fewer than eight outputs, read one by one.
template <int C, int WAVES, bool E5, bool THIN>
__global__ __launch_bounds__(64 * WAVES, C > 1 ? 2 : WAVES == 4 ? 3 : 4) void f8_grad(F8GradArgs a) {
  constexpr int THREADS = 64 * WAVES;
  constexpr int MO = 8 * C / WAVES, WO = 4 / MO;  // 32-row tiles of outputs a wave, waves side by side over the 128 outputs
  constexpr int kBuffer = (1 + C) * kTile;
  constexpr int kAhead = MO > 1 ? 2 : 4;  // steps that are on their way to registers (the accumulators of four blocks leave room for two)
  constexpr int kRow = THREADS / kStep, kYs = 16 / kRow;  // threads that bring a row; of eight gradients each
  constexpr int kCodes = MO > 1 ? 16 : 8, kPieces = C * F8_BLOCK / kCodes / kRow, kApart = kRow * kCodes / F8_BLOCK;  // runs of codes a thread brings, each a block, or two, on
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  kernarg_touch<F8GradArgs>();
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int groups = a.groups;  // of C blocks in a block row; 0: the column sums alone are wanted
  const int steps = (int)(((int64_t)a.T + kStep - 1) / kStep), per = (steps + a.split - 1) / a.split;
  // Ranges of rows in eights: each XCD (workgroups go to the eight in turn) takes its own, with all the blocks, which share what they read in its L2.
  int b = blockIdx.x, range = blockIdx.y;
  if ((a.split & 7) == 0) {
    const unsigned id = blockIdx.y * gridDim.x + blockIdx.x, j = id >> 3, turn = j / gridDim.x;
    range = (int)(turn * 8 + (id & 7)), b = (int)(j - turn * gridDim.x);
  }
  const int64_t t_begin = (int64_t)range * per * kStep;
  const int64_t t_end = t_begin + (int64_t)per * kStep < a.T ? t_begin + (int64_t)per * kStep : a.T;
  // Workgroups go to the eight XCDs in turn.  Four neighbouring groups of a block row go to one, with the same groups of seven other rows: what an
  // XCD runs at one time shares eight rows' gradients and four groups' codes in its L2.  Block rows are dealt to the XCDs one by
  // one, so that rows that keep more blocks than others do not meet on one.
  const int quads = (groups + 3) >> 2, clusters = quads * a.nbo, behind = (clusters + 7) / 8 * 32;
  if (b >= behind) {  // the workgroups behind: one block row's column sums each
    column_sums<THREADS>(a, b - behind, range, t_begin, t_end, (float*)lds);
    return;
  }
  const int cluster = (b >> 5) * 8 + (b & 7), quad = cluster / a.nbo, br = cluster - quad * a.nbo;
  const int first = (quad * 4 + ((b >> 3) & 3)) * C;
  if (cluster >= clusters || first >= a.nbi) return;
  const int n0 = __builtin_amdgcn_readfirstlane(a.row_ptr[br]), cnt = __builtin_amdgcn_readfirstlane(a.row_ptr[br + 1]) - n0;
  if (a.split == 1 && cnt < a.nbi) {  // of the C block columns from `first` those that are not kept become zeros
    for (int c = first; c < first + C && c < a.nbi; ++c) {
      bool kept = false;
      for (int i = lane; i < cnt; i += 64) kept |= a.col_idx[n0 + i] == c;
      if (__ballot(kept)) continue;
      const int col = c * F8_BLOCK + (tid & 127);
      if (col < a.I)
        for (int r = tid >> 7; r < F8_BLOCK && br * F8_BLOCK + r < a.O; r += THREADS / 128) a.dW[((int64_t)br * F8_BLOCK + r) * a.I + col] = 0.f;
    }
  }
  const int has = cnt - first < C ? cnt - first : C;  // kept blocks first .. first + has - 1 of the row
  if (has <= 0) return;

  // what this thread brings: eight gradients, and 8 C codes of one row
  const int row = tid / kRow, piece = tid % kRow;
  // eight gradients at once: at a row's end its last eight, which are moved into place when they are written
  uint32_t col_y[kYs];
  int past[kYs];  // of them
#pragma unroll
  for (int q = 0; q < kYs; ++q) {
    const int o = br * F8_BLOCK + (piece + q * kRow) * 8;
    col_y[q] = (uint32_t)(o + 8 <= a.O || THIN ? o : a.O - 8) * 2;
    past[q] = o + 8 <= a.O || (THIN && piece + q == 0) ? 0 : o + 8 - a.O < 8 ? o + 8 - a.O : 8;
  }
  const int64_t Kp = (int64_t)f8_blocks(a.I) * F8_BLOCK, srows = f8_scale_rows(a.T);
  const int j_in = (piece * kCodes) >> 7, at_in = (piece * kCodes) & 127;  // the first run's block, and its columns in that; the next lies two blocks on
  uint32_t col_x[kPieces], col_s[kPieces];
#pragma unroll
  for (int p = 0; p < kPieces; ++p) {
    const int kb = a.col_idx[n0 + first + (j_in + kApart * p < has ? j_in + kApart * p : 0)];
    col_x[p] = (uint32_t)kb * F8_BLOCK + at_in;
    col_s[p] = (uint32_t)(kb * srows);
  }
  u32x4_t y_in[kAhead][kYs];
  u32x2_t x_in[kAhead][kPieces][kCodes / 8];
  int s_in[kAhead][kPieces];
  const int key = chunk_key(row);
  // A run of sixteen codes becomes a chunk of 32 bytes in two writes; every other row takes its second half first, so that a write of
  // four rows touches all banks.
  const uint32_t swap = kCodes == 16 && (row & 1) ? 8 : 0;
  const int to_y = row * 256 + ((piece >> 1) ^ key) * 32 + (piece & 1) * 16;
  const int to_x = (1 + j_in) * kTile + row * 256 + ((at_in >> 4) ^ key) * 32 + (kCodes == 8 ? (at_in & 8) * 2 : swap * 2);
  // To registers: eight gradients and the codes of row r of those that follow by, bx, bs, which are the same in all lanes.  Nothing here looks
  // at what it asks for: that would wait for it.  (A lane's places are hidden from the optimiser, which would keep each in two registers
  // and add the base there.)
  auto ask = [&](global_t by, global_t bx, global_t bs, uint32_t r, int j) {
    asm volatile("" : "+s"(by), "+s"(bx), "+s"(bs));
#pragma unroll
    for (int q = 0; q < kYs; ++q) {
      if constexpr (THIN) y_in[j][q] = gradients_few((const uint16_t*)by + r * a.ldy, a.O);
      else {
        uint32_t at = r * (uint32_t)a.ldy * 2 + col_y[q];
        asm volatile("" : "+v"(at));
        y_in[j][q] = *(const __attribute__((address_space(1))) u32x4_any*)(by + at);
      }
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      uint32_t at[kCodes / 8], at_s = r + col_s[p];
#pragma unroll
      for (int h = 0; h < kCodes / 8; ++h) {
        at[h] = r * (uint32_t)Kp + col_x[p] + (swap ^ 8 * h);
        asm volatile("" : "+v"(at[h]));
        x_in[j][p][h] = *(const __attribute__((address_space(1))) u32x2_t*)(bx + at[h]);
      }
      asm volatile("" : "+v"(at_s));
      s_in[j][p] = bs[at_s];
    }
  };
  // The range's rows that make no whole step come first, as step 0; n steps in all.
  const int total = t_begin < t_end ? (int)(t_end - t_begin) : 0, n = (total + kStep - 1) / kStep, odd = total - (n - 1) * kStep;
  auto load = [&](int i, int j) {  // step i, or the last
    const int s = i < n ? i : n - 1;
    const int64_t from = t_begin + (s > 0 ? odd + (s - 1) * kStep : 0);
    const int most = s > 0 ? kStep - 1 : odd - 1;
    ask((global_t)(a.dY + from * a.ldy), (global_t)(a.codes + from * Kp), (global_t)(a.scale + from), row < most ? row : most, j);
  };
  // To LDS.  CHECK: step 0, whose missing rows add nothing.  ENDS: the last outputs' block row.
  auto write = [&](int buf, int j, auto ENDS, auto CHECK) {
    const bool in = !decltype(CHECK)::value || row < odd;
#pragma unroll
    for (int q = 0; q < kYs; ++q) {
      u32x4_t y = in ? y_in[j][q] : u32x4_t{0, 0, 0, 0};
      if constexpr (decltype(ENDS)::value) {
#pragma unroll
        for (int d = 1; d < 8; d *= 2) {  // down by `past` values of two bytes, zeros from above
          const u32x4_t v = d == 1 ? u32x4_t{y.x >> 16 | y.y << 16, y.y >> 16 | y.z << 16, y.z >> 16 | y.w << 16, y.w >> 16}
                          : d == 2 ? u32x4_t{y.y, y.z, y.w, 0} : u32x4_t{y.z, y.w, 0, 0};
          y = past[q] & d ? v : y;
        }
        y = past[q] == 8 ? u32x4_t{0, 0, 0, 0} : y;
      }
      *(u32x4_t*)(lds + buf * kBuffer + (to_y ^ 128 * q)) = y;  // the second run lies four chunks on
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {  // (a block more than there are: sums that go nowhere)
      const float s = __uint_as_float((uint32_t)s_in[j][p] << 23);
#pragma unroll
      for (int h = 0; h < kCodes / 8; ++h) {
        const u32x2_t c = in ? x_in[j][p][h] : u32x2_t{0, 0};
        *(u32x4_t*)(lds + buf * kBuffer + kApart * p * kTile + (to_x ^ 16 * h)) = f8_decode_bf16x8<E5>(c.x, c.y, s);
      }
    }
  };

  const int wo = wave % WO, wi = wave / WO;  // wi: 64 columns of the C blocks'
  const int key_r = ((lane & 15) >> 2) << 1 | (lane >> 5), trow = (lane >> 5) * 8 + ((lane & 15) >> 2);
  int at_o[MO], at_i[2];
#pragma unroll
  for (int m = 0; m < MO; ++m) at_o[m] = trow * 256 + (((wo * MO * 2 + m * 2 + ((lane >> 4) & 1)) ^ key_r) << 5) + (lane & 3) * 8;
#pragma unroll
  for (int m = 0; m < 2; ++m) at_i[m] = (1 + (wi >> 1)) * kTile + trow * 256 + ((((wi & 1) * 4 + m * 2 + ((lane >> 4) & 1)) ^ key_r) << 5) + (lane & 3) * 8;
  f32x16_t acc[MO][2] = {};
  auto read = [&](int buf, int k, u32x4_t (&y)[MO], u32x4_t (&x)[2]) {
#pragma unroll
    for (int m = 0; m < 2; ++m) x[m] = read_columns(lds + buf * kBuffer + k * 256 + at_i[m]);
#pragma unroll
    for (int m = 0; m < MO; ++m) y[m] = read_columns(lds + buf * kBuffer + k * 256 + at_o[m]);
  };
  auto multiply = [&](u32x4_t (&y)[MO], u32x4_t (&x)[2]) {
#pragma unroll
    for (int m = 0; m < MO; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        acc[m][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, y[m]), __builtin_bit_cast(bf16x8_t, x[i]), acc[m][i], 0, 0, 0);
  };

  // Step i in buffer i mod 2, a half of it (sixteen rows) read while the other is multiplied; one barrier, between the halves, behind which
  // the next step's buffer is whole and this one's is free for the step after that.  Nothing inside is conditional, so that
  // a wait for what a register asked for can be by count: it is on one and on four blocks a workgroup.  On two the
  // compiler moves the shift of the later step's scales up and waits for all that is under way, every second step.
  auto run = [&](auto ENDS) {
    u32x4_t y[2][MO], x[2][2];
    auto meet = [&]() {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    constexpr int kReads = 2 * (MO + 2), kMul = 2 * MO;
    // where the loop's copies come from: the step 2 + kAhead further on, or the last
    int behind = n - 3 - kAhead;  // steps after that one
    const int64_t ahead = t_begin + (behind > 0 ? odd + (1 + kAhead) * (int64_t)kStep : n > 1 ? odd + (n - 2) * (int64_t)kStep : 0);
    const uint32_t r_ahead = n > 1 || row < odd ? row : odd - 1;
    global_t by = (global_t)(a.dY + ahead * a.ldy), bx = (global_t)(a.codes + ahead * Kp), bs = (global_t)(a.scale + ahead);
    auto step = [&](auto U) {  // U: its number mod kAhead
      constexpr int u = decltype(U)::value & 1, slot = (decltype(U)::value + 2) % kAhead;
      read(u, 16, y[1], x[1]);
      multiply(y[0], x[0]);
#pragma unroll
      for (int k = 0; k < kMul; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                           // a matrix instruction,
        __builtin_amdgcn_sched_group_barrier(0x100, (kReads + kMul - 1) / kMul, 0);  // reads of LDS behind it
      }
      meet();
      read(u ^ 1, 0, y[0], x[0]);
      write(u, slot, ENDS, std::false_type{});
      ask(by, bx, bs, r_ahead, slot);
      const int64_t on = behind > 0 ? kStep : 0;
      by += on * 2 * a.ldy, bx += on * Kp, bs += on;
      --behind;
      multiply(y[1], x[1]);
#pragma unroll
      for (int k = 0; k < kMul; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, (kReads + kMul / 2 - 1) / (kMul / 2), 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);  // conversions, and the writes that follow the reads
        if (k >= kMul / 2) __builtin_amdgcn_sched_group_barrier(0x200, 2, 0);
      }
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j) load(j, j);
    write(0, 0, ENDS, std::true_type{});
    load(kAhead, 0);
    write(1, 1, ENDS, std::false_type{});
    load(1 + kAhead, 1);
    meet();
    read(0, 0, y[0], x[0]);
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    constexpr std::integral_constant<int, 2> k2{};
    constexpr std::integral_constant<int, 3> k3{};
    int i = 0;
    for (; i + kAhead <= n; i += kAhead) {
      step(k0);
      step(k1);
      if constexpr (kAhead == 4) {
        step(k2);
        step(k3);
      }
    }
    if (i < n) step(k0);
    if (i + 1 < n) step(k1);
    if constexpr (kAhead == 4)
      if (i + 2 < n) step(k2);
  };
  if (n > 0) {
    if (br == a.nbo - 1 && (a.O & 127)) run(std::true_type{});
    else run(std::false_type{});
  }

  if (wi >> 1 >= has) return;
  const int kb = a.col_idx[n0 + first + (wi >> 1)];
  const bool whole = a.split == 1;
  float* out = whole ? a.dW + (int64_t)br * F8_BLOCK * a.I + (int64_t)kb * F8_BLOCK
                     : a.part + ((int64_t)range * a.nnzb + n0 + first + (wi >> 1)) * F8_BLOCK_BYTES;
  const int64_t ld = whole ? a.I : F8_BLOCK;
  const int rows = whole ? a.O - br * F8_BLOCK : F8_BLOCK, cols = whole ? a.I - kb * F8_BLOCK : F8_BLOCK;
#pragma unroll
  for (int m = 0; m < MO; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = (wi & 1) * 64 + i * 32 + (lane & 31);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int q = (wo * MO + m) * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
        if (q < rows && c < cols) out[q * ld + c] = acc[m][i][r];
      }
    }
}

// The sums over the ranges of rows, in their order: a kept block's entries, zeros for the others, and the bias's gradient.  A workgroup
// takes eight rows of a block at a time, a thread four entries; every sixteenth of the rows, or (many blocks, most of them zeros: the start
// of a workgroup is what counts: 24 x 156 blocks of which 37 are kept, 4052 rows, 183 us for the call with two rows a workgroup, 93 so) every fourth.
__global__ __launch_bounds__(256) void f8_grad_finish(F8GradArgs a) {
  const int cell = blockIdx.x, br = cell / a.nbi, kb = cell - br * a.nbi, c = (threadIdx.x & 31) * 4;
  if (a.db && kb == 0 && blockIdx.y == 0 && threadIdx.x < F8_BLOCK && br * F8_BLOCK + (int)threadIdx.x < a.O) {
    const float* p = a.part_db + br * F8_BLOCK + threadIdx.x;
    float v = 0.f;
#pragma unroll 16
    for (int s = 0; s < a.split; ++s) v += p[s * (int64_t)a.O];
    a.db[br * F8_BLOCK + threadIdx.x] = v;
  }
  const int n0 = a.row_ptr[br], n1 = a.row_ptr[br + 1];
  int n = -1;
  for (int i = n0 + (threadIdx.x & 63); i < n1; i += 64) n = a.col_idx[i] == kb ? i : n;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) n = max(n, __shfl_xor(n, d));
  const int left = a.I - kb * F8_BLOCK - c;  // columns from this thread's on
  if (!a.dW || left <= 0) return;
  for (int r = (int)blockIdx.y * 8 + (threadIdx.x >> 5); r < F8_BLOCK && br * F8_BLOCK + r < a.O; r += gridDim.y * 8) {
    f32x4_t v = {};
    if (n >= 0) {
      const float* p = a.part + (int64_t)n * F8_BLOCK_BYTES + r * F8_BLOCK + c;
#pragma unroll 8
      for (int s = 0; s < a.split; ++s) v += *(const f32x4_any*)(p + s * (a.nnzb * F8_BLOCK_BYTES));
    }
    float* out = a.dW + ((int64_t)br * F8_BLOCK + r) * a.I + (int64_t)kb * F8_BLOCK + c;
    if (left >= 4) {
      *(f32x4_any*)out = v;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < left) out[k] = v[k];
    }
  }
}

// Kept blocks a workgroup: more of them share a block row's gradients and take longer, so it goes by how often the chip is filled.  The model counts two workgroups of
// one or two blocks a CU or one of four (single blocks on four waves would fit three; their step was taken from those on eight); us a step where it is full: 0.62, 0.98,
// 0.94, and 6 a round to begin and end.  Measured (us for one, two, four blocks):
//   all kept: 8192 x 4096 -> 16384 1241 1051 1017, 8192 x 8192 -> 8192 1183 981 971 (930, 1120, 1133 TFLOP/s), 2048 x 4096 -> 4096 84 75 75, 2048 x 4096 -> 4097 104 109 121
//   under random masks: 8192 x 8192 -> 8192 half 663 583 645, a quarter 386 391 444, 2048 x 4096 -> 4096 half 61 66 67, 3000 x 16384 -> 1024 0.3 57 63 87,
//   4096 x 4096 -> 4096 a quarter 72 79 113, 0.7 140 120 123, 4052 x 19902 -> 2966 a quarter 256 298 248
int blocks_each(const F8GradArgs& a) {
  const double steps = (double)(((int64_t)a.T + kStep - 1) / kStep), row = (double)a.nnzb / a.nbo;
  const bool full = a.nnzb == (int64_t)a.nbo * a.nbi;
  int best = 1;
  double least = 1e30;
  for (int c = 1; c <= 4; c *= 2) {
    const double step = c == 1 ? 0.62 : c == 2 ? 0.98 : 0.94;
    const int64_t slots = c == 4 ? 256 : 512;
    double rounds, whole;
    if (full) {
      const int64_t groups = (int64_t)a.nbo * ((a.nbi + c - 1) / c), left = groups % slots;
      // a last round takes half the time where a CU has one workgroup instead of two, and less than a whole one where most have none
      const double part = left == 0 ? 0 : left <= 256 && slots == 512 ? 0.5 : slots == 512 || groups < slots ? 1 : 0.7;
      rounds = (double)(groups / slots) + part, whole = (double)((groups + slots - 1) / slots);
    } else {
      // rows keep differing numbers of blocks: the last group of a row is half full on average, and XCDs have more or fewer, which the smaller workgroups even out
      whole = a.nbo * (row / c + (c - 1) / (2.0 * c)) / (double)slots;
      rounds = c == 1 ? 1.07 * whole : whole + (c == 2 ? 0.25 : 0.4);
      const double lowest = c == 1 ? 0.7 : c == 2 ? 0.5 : 0.8;
      if (rounds < lowest) rounds = lowest;
    }
    const double us = rounds * steps * step + 6 * whole;
    if (us < least) least = us, best = c;
  }
  return best;
}

template <int C, int WAVES, bool E5, bool THIN = false>
int launch(F8GradArgs a, hipStream_t st) {
  constexpr int lds = 2 * (1 + C) * kTile;
  static const bool raised = hipFuncSetAttribute((const void*)&f8_grad<C, WAVES, E5, THIN>, hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
  if (!raised) return BSP_ERR_HIP;
  a.groups = a.dW ? (a.nbi + C - 1) / C : 0;
  const int64_t groups = ((int64_t)a.nbo * ((a.groups + 3) / 4) + 7) / 8 * 32;
  if (!f8_fits_x(groups + a.nbo, 64 * WAVES)) return BSP_ERR_SHAPE;
  hipLaunchKernelGGL((f8_grad<C, WAVES, E5, THIN>), dim3((unsigned)(groups + (a.db ? a.nbo : 0)), (unsigned)a.split), dim3(64 * WAVES), lds, st, a);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}

}  // namespace

// ... and where single blocks are a workgroup for every other CU or fewer (more blocks in ranges were not measured), ranges of at least four steps: a step takes 0.5 us where a CU has one workgroup, 0.65 where it has two, and
// the ranges' sums cost a launch and are written and read (us at 16384 rows, 1024 x 1024 in 4 and 8 ranges 74 and 55, 2048 x 1024 in 2 and 4 135 and 101; 2000 rows, 51
// blocks of 4096 x 4096 in 5 and 10 39 and 51).
int f8_grad_split(int64_t nnzb, int T) {
  const int64_t steps = ((int64_t)T + kStep - 1) / kStep;
  if (nnzb == 0 || nnzb > 128) return 1;
  int best = 1;
  double least = 0.5 * (double)steps;
  for (int64_t s = 2; s * 4 <= T / kStep && s * nnzb <= 512; ++s) {
    if (s > 8 && (s & 7)) continue;
    const double us = (double)((steps + s - 1) / s) * (s * nnzb <= 256 ? 0.5 : 0.65) + 4 + 0.033 * (double)(nnzb * s);
    if (us < least) least = us, best = (int)s;
  }
  return best;
}

int f8_launch_grad(const F8GradArgs& a, hipStream_t st) {
  // the second launch: every block of the matrix, or (the bias's gradient alone) one a block row
  F8GradArgs f = a;
  if (!f.dW) f.nbi = 1;
  if (!f8_fits_x((int64_t)f.nbo * f.nbi, 256)) return BSP_ERR_SHAPE;
  int rc;
  if (a.O < 8) rc = a.e5 ? launch<1, 8, true, true>(a, st) : launch<1, 8, false, true>(a, st);
  else switch (a.split > 1 ? 1 : blocks_each(a)) {
    case 4: rc = a.e5 ? launch<4, 8, true>(a, st) : launch<4, 8, false>(a, st); break;
    case 2: rc = a.e5 ? launch<2, 4, true>(a, st) : launch<2, 4, false>(a, st); break;
    default:
      if (a.split == 1 && a.nnzb > 256) rc = a.e5 ? launch<1, 4, true>(a, st) : launch<1, 4, false>(a, st);
      else rc = a.e5 ? launch<1, 8, true>(a, st) : launch<1, 8, false>(a, st);
  }
  if (rc != BSP_OK || a.split == 1) return rc;
  const int cells = f.nbo * f.nbi;
  hipLaunchKernelGGL(f8_grad_finish, dim3((unsigned)cells, !f.dW ? 1 : cells >= 1024 ? 4 : 16), dim3(256), 0, st, f);
  return hipGetLastError() == hipSuccess ? BSP_OK : BSP_ERR_HIP;
}
