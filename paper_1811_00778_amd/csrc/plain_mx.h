// Products of microscaled matrices: y = act(x w^T + bias) + residual, w of four-bit numbers, x of four or eight bits.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows by 16 rows over 128 numbers, four blocks of 32, and scales every block's sum by the two
// blocks' powers of two.  Lane l holds of its row l mod 16, with g = l / 16: of four-bit numbers the 16 bytes of block g, of eight-bit ones bytes 16 g .. 16 g + 15 of
// the first and of the last 64; and of its row the byte of block g in one of four bytes of a register.  w is the first operand: a lane's four sums are of w's rows
// 4 g .. 4 g + 3 and x's row l mod 16.  F products side by side take rows F i + j (i: row of the instruction, j: product), so that a lane's sums of
// all of them are 4 F columns side by side, and the scales of four products one 32-bit word.
//
// What the instruction sums, by measurement (every sum of eight random codes of both formats, 131072 of them): the products of eight consecutive four-by-eight-bit pairs are
// cut, toward zero, to multiples of 2^(p + q - 13), p and q the largest of the factors' exponents in a pair (numbers below the normal ones count with the least normal exponent), and the
// groups' sums join in 32 bits.  Pairs of four-bit numbers lie within those 13 bits: exact.  Eight-bit x does not, so it goes in two halves: numbers from 2 on, whose products with w
// are multiples of 2^-3 (2^-2 0.5) beside 2^(8 + 2), and numbers below, multiples of 2^-10 (2^-9 0.5) beside 2^(0 + 2).  Neither loses a bit: sums are of exact products, in 32
// bits.  It takes twice the instructions; in one, what lies beside a large product was lost, also where large ones cancel, and 16-bit results were off by up to all of themselves.
#pragma once
#include "plain_rows.h"

namespace hcnn {

struct MxArgs {
  GemmArgs g;                  // M, N, the ending, the sums
  const uint8_t *x, *x_scales, *w, *w_scales;
  size_t x_bytes, w_bytes;     // of a row
  size_t x_pitch, w_pitch;     // bytes from a block's row scales to the next block's: multiples of 64, so that whole 64 rows can be read
  uint32_t steps;              // of 128 numbers
  uint32_t part;               // steps of each of g.splits parts of the sum
  uint64_t first;              // tile that the launch begins with
};

#if defined(__HIP_DEVICE_COMPILE__)
typedef int hcnn_int8 __attribute__((ext_vector_type(8)));
#endif

// A lane's part of an operand of one instruction
template <int F>
struct MxFrag {
#if defined(__HIP_DEVICE_COMPILE__)
  hcnn_word4 v[F == kMx8 ? 2 : 1];
  __device__ __forceinline__ hcnn_int8 words() const {
    hcnn_int8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = (int)v[0][i];
      r[i + 4] = F == kMx8 ? (int)v[F == kMx8 ? 1 : 0][i] : 0;
    }
    return r;
  }
#endif
};

#if defined(__HIP_DEVICE_COMPILE__)
// acc += (16 rows of w) x (16 rows of x) over a step; the scales' bytes JW and JX of the words
template <int F, int JW, int JX>
__device__ __forceinline__ void mx_mma(hcnn_float4& acc, const MxFrag<kMx4>& w, const MxFrag<F>& x, uint32_t sw, uint32_t sx) {
  const hcnn_int8 wv = w.words(), xv = x.words();
  if constexpr (F == kMx4) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc, 4, 4, JW, (int)sw, JX, (int)sx);
  } else {
    hcnn_int8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // bytes with 0x40: magnitudes of 2 or more
      const uint32_t b = (uint32_t)xv[i], up = b & 0x40404040u, mask = (up << 2) - (up >> 6);
      hi[i] = (int)(b & mask);
      lo[i] = (int)(b & ~mask);
    }
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, hi, acc, 4, 0, JW, (int)sw, JX, (int)sx);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, lo, acc, 4, 0, JW, (int)sw, JX, (int)sx);
  }
}
#endif

// number k of a row, for the checker
template <int F>
HCNN_HD float mx_at(const uint8_t* codes, size_t row_bytes, const uint8_t* scales, size_t pitch, size_t row, uint32_t k) {
  const uint8_t* line = codes + row * row_bytes;
  const uint32_t code = F == kMx8 ? line[k] : line[k / 2] >> (k % 2 * 4) & 15, byte = scales[k / 32 * pitch + row];
  return mx_value<F>(code) * (byte == 255 ? std::numeric_limits<float>::quiet_NaN() : mx_scale(byte));
}

// Each i of 0 .. COUNT - 1 as a compile-time constant (the instruction takes the scales' byte as one)
template <class Each, int... I>
HCNN_HD void each_of(std::integer_sequence<int, I...>, Each&& each) { (each(std::integral_constant<int, I>{}), ...); }

// The simple form, for few rows or columns and small sizes: a workgroup computes 16 MF rows by 16 NF columns, its waves share the steps; operands come straight from
// memory to the registers that the products read, kDeep steps asked for at a time, and no wave waits for another before the sums join in LDS.  One row of eight bits through 4096 ->
// 16384 (36 MB of weights): 9.8 us by the profiler, 3.7 TB/s with the launch; 4096 -> 4096 5.0 in a graph of 20.  Few rows are bound by that stream, more of them by the operands that every workgroup reads
// for itself: 517 x 1031 -> 777 of eight bits in 64 x 16 11.8 us, in 64 x 64 11.4 (graphs of 10); from about a 64 x 64 for each of four on a compute unit on the tiles are faster.
template <class T, int F, int MF, int NF>
struct MxStrip {
  static constexpr int kWaves = MF * NF == 16 ? 4 : 8, kThreads = kWaves * 64, kDeep = MF * NF == 16 ? 2 : 4;
  static constexpr uint32_t kRows = MF * 16, kCols = NF * 16;
  static constexpr int kPhases = 2;
  static constexpr size_t kLdsBytes = (size_t)kWaves * kRows * kCols * 4;
  struct Regs {};
  static size_t grid(const GemmArgs& g) { return (size_t)((g.M + kRows - 1) / kRows) * ((g.N + kCols - 1) / kCols); }
#if defined(__HIP_DEVICE_COMPILE__)
  // Row f i + j of R, from row r0 on, of step s
  template <int OF, int COUNT>
  __device__ __forceinline__ static void frags(MxFrag<OF> (&to)[COUNT], const uint8_t* const (&at)[COUNT], uint32_t s) {
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
      const char* p = reinterpret_cast<const char*>(at[j]) + (size_t)s * (OF == kMx8 ? 128 : 64);
      const U4 a = ld16(p);
      to[j].v[0] = hcnn_word4{a.x, a.y, a.z, a.w};
      if constexpr (OF == kMx8) {
        const U4 b = ld16(p + 64);
        to[j].v[1] = hcnn_word4{b.x, b.y, b.z, b.w};
      }
    }
  }
  template <int COUNT>
  __device__ __forceinline__ static uint32_t scale(const uint8_t* at, size_t pitch, uint32_t s) {
    const uint8_t* p = at + (size_t)s * 4 * pitch;
    if constexpr (COUNT == 4) return *reinterpret_cast<const uint32_t*>(p);
    else return *p;
  }
#endif
  template <int PH>
  HCNN_HD static void phase(const MxArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    float* lds = reinterpret_cast<float*>(lds_words);              // [wave][kRows][kCols]
    const uint32_t wave = (uint32_t)tid / 64, lane = (uint32_t)tid % 64, i = lane % 16, g = lane / 16;
    const uint32_t tn = (a.g.N + kCols - 1) / kCols;
    const uint64_t tile = a.first + bid;
    const uint32_t m0 = (uint32_t)(tile / tn) * kRows, n0 = (uint32_t)(tile % tn) * kCols;
    if constexpr (PH == 0) {
      hcnn_float4 acc[MF][NF];
#pragma unroll
      for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int n = 0; n < NF; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][n][e] = 0.0f;
#if defined(__HIP_DEVICE_COMPILE__)
      // (rows beyond the last one: the last one, their sums are dropped; the scales have room for whole 64 rows)
      const uint8_t *xp[MF], *wp[NF];
#pragma unroll
      for (int m = 0; m < MF; ++m) xp[m] = a.x + (size_t)(m0 + i * MF + m < a.g.M ? m0 + i * MF + m : a.g.M - 1) * a.x_bytes + g * 16;
#pragma unroll
      for (int n = 0; n < NF; ++n) wp[n] = a.w + (size_t)(n0 + i * NF + n < a.g.N ? n0 + i * NF + n : a.g.N - 1) * a.w_bytes + g * 16;
      const uint8_t *sx = a.x_scales + g * a.x_pitch + m0 + i * MF, *sw = a.w_scales + g * a.w_pitch + n0 + i * NF;
      for (uint32_t s0 = wave_uniform(wave); s0 < a.steps; s0 += kWaves * kDeep) {
        MxFrag<F> x[kDeep][MF];
        MxFrag<kMx4> w[kDeep][NF];
        uint32_t bx[kDeep], bw[kDeep];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
          const uint32_t s = s0 + d * kWaves;
          if (s < a.steps) {
            frags(w[d], wp, s);
            frags(x[d], xp, s);
            bx[d] = scale<MF>(sx, a.x_pitch, s);
            bw[d] = scale<NF>(sw, a.w_pitch, s);
          }
        }
#pragma unroll
        for (int d = 0; d < kDeep; ++d)
          if (s0 + d * kWaves < a.steps)
            each_of(std::make_integer_sequence<int, MF * NF>{}, [&](auto c) {
              constexpr int m = c.value / NF, n = c.value % NF;
              mx_mma<F, n, m>(acc[m][n], w[d][n], x[d][m], bw[d], bx[d]);
            });
      }
#else
      for (uint32_t s = wave; s < a.steps; s += kWaves)
        for (uint32_t m = 0; m < MF; ++m)
          for (uint32_t n = 0; n < NF; ++n)
            for (uint32_t e = 0; e < 4; ++e) {
              const uint32_t row = m0 + i * MF + m, col = n0 + (4 * g + e) * NF + n;
              if (row >= a.g.M || col >= a.g.N) continue;
              for (uint32_t k = s * 128; k < s * 128 + 128; ++k)
                acc[m][n][e] += mx_at<F>(a.x, a.x_bytes, a.x_scales, a.x_pitch, row, k) * mx_at<kMx4>(a.w, a.w_bytes, a.w_scales, a.w_pitch, col, k);
            }
#endif
#pragma unroll
      for (int m = 0; m < MF; ++m) {
        float* to = lds + ((size_t)wave * kRows + i * MF + m) * kCols + 4 * g * NF;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < NF; ++n) to[e * NF + n] = acc[m][n][e];
      }
    } else {
      for (uint32_t q = tid; q < kRows * kCols / 4; q += kThreads) {
        const uint32_t m[1] = {m0 + q / (kCols / 4)}, n = n0 + q % (kCols / 4) * 4;
        if (m[0] >= a.g.M || n >= a.g.N) continue;
        float v[1][4] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[0][e] += lds[(size_t)w * kRows * kCols + q * 4 + e];
        float bias[4] = {};
        if (a.g.bias) load_row(static_cast<const T*>(a.g.bias) + n, a.g.N - n, bias);
        finish<T>(a.g, m, n, bias, v);
      }
    }
  }
};

// The form for many rows and columns.  What bounds it: a tile of 256 x 256 takes 34 KB of operands for every step of 128 numbers, which the matrix unit goes through in
// 0.55 us (four bits; 8192 x 16384 -> 16384 with the operands' loads and reads left out: 644 us); the loads alone, 13 TB/s out of the dies' caches of the 17 that they give, take 772,
// products and loads 950, 4.6 PFLOP/s.  Every tile's outputs leave at memory's rate with nothing beside them: 72 of the 304 us of 8192 x 4096 -> 16384 (3.6 PFLOP/s).  Of
// eight bits, two instructions for one, 690 us (1.6 PFLOP/s) there, 1.7 on the longer sum, the matrix unit busy for 0.64 of it: the instructions alone give 2.1.  Measured and left out: four waves of 128 x 128 in place of eight of 128 x 64 (406 us: nothing beside a wave's ending),
// slots of one step (324), 128 x 256 in two workgroups a compute unit, also started half a tile apart (345, 348: their operands are half as many again).
// A workgroup computes a tile of BM x BN outputs in WM x WN waves, 16 FM rows by 16 FN columns each; operands come to LDS past
// the registers, in slots: of four-bit x two steps (128 bytes of every row, two slots), of eight-bit x one step (128 bytes of x's rows, 64 of w's; three slots), with
// their scales.  A lane's operands of x go through a ring of kAhead places, read that many products ahead; w's of a step have two places.  The last kAhead
// of a slot's operands are in registers when the barrier comes: behind it the slot is filled anew while their products run, and the next slot's first are read.
//   LDS: lines of 256 bytes (all 64 banks), 16 pieces of 16 bytes, piece p of line l at p ^ turn(l).  The 16 rows of one read lie four apart: turn takes 16 values in
// them, so that they spread evenly over the banks.  (Lines of 128 bytes have eight values: two rows of a read would share each.)
template <int BYTES, int ROWS, int THREADS>
struct MxTileRows {
  static constexpr uint32_t kPieces = BYTES / 16, kLineRows = 256 / BYTES;          // of a row; rows of a line
  static constexpr int kEach = ROWS * BYTES / 16 / THREADS;
  static constexpr uint32_t kLdsBytes = ROWS * BYTES;
  static_assert(ROWS * BYTES % (16 * THREADS) == 0, "every thread has the same number of pieces");
  HCNN_HD static uint32_t turn(uint32_t line) { return line / (4 / kLineRows) & 15; }
  HCNN_HD static uint32_t place(uint32_t row, uint32_t piece) {
    const uint32_t line = row / kLineRows, p = row % kLineRows * kPieces + piece;
    return line * 256 + ((p ^ turn(line)) << 4);
  }
  // (row, piece) that lies at LDS piece c
  HCNN_HD static void at(uint32_t c, uint32_t* row, uint32_t* piece) {
    const uint32_t line = c / 16, p = (c % 16) ^ turn(line);
    *row = line * kLineRows + p / kPieces;
    *piece = p % kPieces;
  }
  // Byte offset of a thread's piece i from the slot's first bytes in the tile's first row.  Rows beyond X: the last one.
  HCNN_HD static uint32_t offset(size_t ld, uint32_t X, uint32_t x0, int tid, int i) {
    uint32_t row, piece;
    at((uint32_t)(tid + i * THREADS), &row, &piece);
    if (x0 + row >= X) row = X - 1 - x0;
    return (uint32_t)(row * ld) + piece * 16;
  }
  // (every piece of a thread has this number within its row)
  static_assert(THREADS % 256 == 0, "the threads take whole turns of lines");
  HCNN_HD static uint32_t piece_of(int tid) {
    uint32_t row, piece;
    at((uint32_t)tid, &row, &piece);
    return piece;
  }
};
// BYTES (16 or 4) of every lane of a wave to LDS, side by side
template <int BYTES>
HCNN_HD void load_to_lds(const uint8_t* base, uint32_t off, uint32_t at, [[maybe_unused]] char* lds, [[maybe_unused]] int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
  static_assert(BYTES == 16 || BYTES == 4, "what the instruction takes");
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  if constexpr (BYTES == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(off), "s"(base) : "memory", "m0");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(at), "v"(off), "s"(base) : "memory", "m0");
#pragma clang diagnostic pop
#else
  __builtin_memcpy(lds + at + lane * BYTES, base + off, BYTES);
#endif
}
// Byte of LDS at which the workgroup's memory begins
HCNN_HD uint32_t lds_start([[maybe_unused]] const uint32_t* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
  return wave_uniform((uint32_t)(uintptr_t)lds);          // (the low half of an LDS pointer is its offset)
#else
  return 0;
#endif
}
// What is on its way to LDS past the registers has arrived, all but the last N loads
template <int N>
HCNN_HD void direct_all_but() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
#endif
}

// 16 numbers of each of a wave's 16 x 4 lanes, four lanes (16 apart) side by side in a row, to memory in 64 bytes of every row at a time: the lanes' pieces of 16 bytes
// change places first.  (Stores of a lane's own pieces write 16 of every 32 or 64 bytes at a time: 8192 x 128 -> 16384 took 82 us in place of 78, of which 52 are the outputs at 5.2 TB/s.)
template <class T>
HCNN_HD void store_quads(T* p, [[maybe_unused]] uint32_t g, const float (&v)[16], bool here) {     // p: the lane's own first number; here: the row is there
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int P = sizeof(T);                                     // pieces: two of 16-bit numbers, four of 32
  constexpr uint32_t kPer16 = 16 / sizeof(T);
  T t[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) t[i] = Num<T>::narrow(v[i]);
  uint32_t w[P][4];
  __builtin_memcpy(w, t, sizeof(t));
  auto swap = [](auto wide, uint32_t& a, uint32_t& b) {
    typedef unsigned two __attribute__((ext_vector_type(2)));
    two r;
    if constexpr (decltype(wide)::value) r = __builtin_bit_cast(two, __builtin_amdgcn_permlane32_swap(a, b, false, false));
    else r = __builtin_bit_cast(two, __builtin_amdgcn_permlane16_swap(a, b, false, false));
    a = r.x;
    b = r.y;
  };
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if constexpr (P == 2) {
      swap(std::false_type{}, w[0][d], w[1][d]);
      swap(std::true_type{}, w[0][d], w[1][d]);
    } else {
      swap(std::false_type{}, w[0][d], w[1][d]);
      swap(std::false_type{}, w[P - 2][d], w[P - 1][d]);
      swap(std::true_type{}, w[0][d], w[P - 2][d]);
      swap(std::true_type{}, w[1][d], w[P - 1][d]);
    }
  }
  if (!here) return;
  T* row = p - 16 * g;                                             // the four lanes' first number
#pragma unroll
  for (int i = 0; i < P; ++i) {
    U4 x;
    __builtin_memcpy(&x, w[i], 16);
    st16(reinterpret_cast<char*>(row + (i * 4 + g) * kPer16), x);
  }
#else
  if (here) store_row(p, v);
#endif
}

template <class T, int F, int BM, int BN, int WM, int WN, int EPI>
struct MxTile {
  static constexpr int kThreads = WM * WN * 64;
  static constexpr int kLoopPhases = 4, kPhases = 5;                   // a round of the loop: two steps
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int kMinWavesPerSimd = FM * FN > 32 ? 1 : 2;
  static constexpr int kScaleLoads = (BM + BN) / 64 / (WM * WN);       // of a wave for a step: 64 rows each
  static_assert(FM % 4 == 0 && FN % 4 == 0 && kScaleLoads * 64 * WM * WN == BM + BN && 256 % BM == 0 && 256 % BN == 0, "whole groups of four products");
  static constexpr int kSteps = F == kMx4 ? 2 : 1, kSlots = F == kMx4 ? 2 : 3;       // steps of a slot
  static constexpr int kAhead = F == kMx4 ? 4 : 2;
  typedef MxTileRows<128, BM, kThreads> X;
  typedef MxTileRows<F == kMx4 ? 128 : 64, BN, kThreads> W;
  static constexpr uint32_t kScaleBytes = 4 * (BM + BN);               // of a step: [x's blocks][BM], [w's blocks][BN]
  static constexpr uint32_t kScales = X::kLdsBytes + W::kLdsBytes, kSlot = kScales + kSteps * kScaleBytes;
  static constexpr size_t kLdsBytes = (size_t)kSlots * kSlot;
  static constexpr int kLoads = X::kEach + W::kEach + kSteps * kScaleLoads;          // of a thread for a slot
  static_assert(kLdsBytes <= 160 * 1024, "the slots fit LDS");
#if defined(__HIP_DEVICE_COMPILE__)
  struct Operands { MxFrag<F> x[kAhead]; MxFrag<kMx4> w[2][FN]; uint32_t sx[2][FM / 4], sw[2][FN / 4]; };
#else
  struct Operands { float x[kAhead][128], w[2][FN * 4][128]; };
#endif
  struct Regs {
    uint32_t iter;
    uint32_t m0, n0, split, steps;              // steps: of the part
    // the next slot to be brought: its first step, its place, its bytes of the tile's first rows and of the scales that this wave brings, and from a step's to the next's
    // (behind the last slot: the last one again, to a place that nobody reads)
    uint32_t at_step, at_slot, wave_lds;
    const uint8_t *x, *w, *scales[kScaleLoads];
    size_t scale_step[kScaleLoads];
    uint32_t here;                              // the slot that is read
    uint32_t ox[X::kEach], ow[W::kEach], os[kScaleLoads];
    uint32_t back;                              // from a piece of a second step to the one in its place in a slot that has one step only
    Operands op;
    hcnn_float4 acc[FM][FN];
  };
  static constexpr bool wave_sync(int ph) { return ph == 1 || ph == 3 || (ph == 0 && F == kMx4); }
  HCNN_HD static uint32_t loop_count(const MxArgs& a) { return (a.part + 1) / 2; }
  static size_t grid(const GemmArgs& g) { return (size_t)((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN) * g.splits; }
  // Tiles go round the eight dies as those of Gemm do
  HCNN_HD static void begin(const MxArgs& a, unsigned bid, int tid, uint32_t* lds, Regs& r) {
    const uint32_t tm = (a.g.M + BM - 1) / BM, tn = (a.g.N + BN - 1) / BN, all = tm * tn * a.g.splits;
    const uint32_t die = bid % 8, each = all / 8, rest = all % 8;
    uint32_t at = die * each + (die < rest ? die : rest) + bid / 8;
    r.split = at / (tm * tn);
    at -= r.split * (tm * tn);
    constexpr uint32_t kBand = 4;
    const uint32_t band = at / (kBand * tn), high = tm - band * kBand < kBand ? tm - band * kBand : kBand;
    at -= band * kBand * tn;
    r.m0 = (band * kBand + at % high) * BM;
    r.n0 = at / high * BN;
    const uint32_t step0 = r.split * a.part;
    r.steps = step0 >= a.steps ? 0 : a.steps - step0 < a.part ? a.steps - step0 : a.part;
    r.x = a.x + r.m0 * a.x_bytes + (size_t)step0 * (F == kMx8 ? 128 : 64);
    r.w = a.w + r.n0 * a.w_bytes + (size_t)step0 * 64;
    r.at_step = r.at_slot = r.here = 0;
    r.wave_lds = lds_start(lds) + wave_uniform((uint32_t)tid / 64) * 1024;
#pragma unroll
    for (int i = 0; i < X::kEach; ++i) r.ox[i] = X::offset(a.x_bytes, a.g.M, r.m0, tid, i);
#pragma unroll
    for (int i = 0; i < W::kEach; ++i) r.ow[i] = W::offset(a.w_bytes, a.g.N, r.n0, tid, i);
    r.back = kSteps == 2 && X::piece_of(tid) >= 4 ? 64 : 0;
    // scales: a wave's 64 words are 64 x 4 of the bytes [blocks][BM] and [blocks][BN]; beyond the rows, the last word that is there
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
      const uint32_t word = (uint32_t)(tid + i * kThreads) * 4, of_w = wave_uniform(word >= 4 * BM), in = of_w ? word - 4 * BM : word;
      const uint32_t block = of_w ? in / BN : in / BM, row = of_w ? r.n0 + in % BN : r.m0 + in % BM;
      const size_t pitch = of_w ? a.w_pitch : a.x_pitch;
      r.scales[i] = (of_w ? a.w_scales : a.x_scales) + (size_t)step0 * 4 * pitch;
      r.scale_step[i] = 4 * pitch;
      r.os[i] = (uint32_t)(block * pitch + (row < pitch ? row : pitch - 4));
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) r.acc[i][j][e] = 0.0f;
    for (int s = 0; s < kSlots; ++s) {
#pragma unroll
      for (int d = 0; d < kLoads; ++d) bring(d, tid, lds, r);
      brought(r);
    }
    direct_all_but<(kSlots - 1) * kLoads>();
  }
  HCNN_HD static void begin_next(const MxArgs&, unsigned, int tid, uint32_t* lds, Regs& r) {
    const char* slot = reinterpret_cast<const char*>(lds);
    read_w(slot, 0, 0, tid, r);
#pragma unroll
    for (int q = 0; q < kAhead; ++q) read_x(slot, 0, 0, q, tid, r);
  }
  // Load d of the thread's for the next slot
  HCNN_HD static void bring(int d, int tid, uint32_t* lds, const Regs& r) {
    char* base = reinterpret_cast<char*>(lds);
    const uint32_t back = kSteps == 2 && r.at_step + 1 == r.steps ? r.back : 0;
    if (d < X::kEach) {
      load_to_lds<16>(r.x, r.ox[d] - back, r.wave_lds + r.at_slot + d * kThreads * 16, base, tid & 63);
    } else if (d < X::kEach + W::kEach) {
      const int i = d - X::kEach;
      load_to_lds<16>(r.w, r.ow[i] - back, r.wave_lds + r.at_slot + X::kLdsBytes + i * kThreads * 16, base, tid & 63);
    } else {
      const int s = (d - X::kEach - W::kEach) / kScaleLoads, i = (d - X::kEach - W::kEach) % kScaleLoads;
      const uint32_t wave_scales = r.wave_lds - wave_uniform((uint32_t)tid / 64) * 768;
      load_to_lds<4>(r.scales[i] + (s && r.at_step + 1 < r.steps ? r.scale_step[i] : 0), r.os[i], wave_scales + r.at_slot + kScales + s * kScaleBytes + i * kThreads * 4, base, tid & 63);
    }
  }
  HCNN_HD static void brought(Regs& r) {
    r.at_slot = r.at_slot == (kSlots - 1) * kSlot ? 0 : r.at_slot + kSlot;
    const uint32_t on = r.at_step + kSteps < r.steps ? kSteps : 0;
    r.at_step += on;
    r.x += on * (F == kMx8 ? 128 : 64);
    r.w += on * 64;
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) r.scales[i] += on ? kSteps * r.scale_step[i] : 0;
  }
  HCNN_HD static uint32_t x_row(int tid, int q) { return (uint32_t)tid / 64 / WN * (FM * 16) + q / 4 * 64 + tid % 16 * 4 + q % 4; }
  HCNN_HD static uint32_t w_row(int tid, int j) { return (uint32_t)tid / 64 % WN * (FN * 16) + j / 4 * 64 + tid % 16 * 4 + j % 4; }
  // Operand q of x, and all of w's, of step s of a slot, for step `to` of a round
#if defined(__HIP_DEVICE_COMPILE__)
  __device__ __forceinline__ static hcnn_word4 word4(const char* p) { return *reinterpret_cast<const hcnn_word4*>(p); }
  __device__ __forceinline__ static void read_x(const char* slot, int s, int, int q, int tid, Regs& r) {
    const uint32_t g = tid % 64 / 16, row = x_row(tid, q);
    MxFrag<F>& to = r.op.x[q % kAhead];
    to.v[0] = word4(slot + X::place(row, F == kMx8 ? g : s * 4 + g));
    if constexpr (F == kMx8) to.v[1] = word4(slot + X::place(row, 4 + g));
  }
  __device__ __forceinline__ static void read_w(const char* slot, int s, int to, int tid, Regs& r) {
    const uint32_t g = tid % 64 / 16;
    const char* scales = slot + kScales + s * kScaleBytes;
#pragma unroll
    for (int j = 0; j < FN; ++j) r.op.w[to][j].v[0] = word4(slot + X::kLdsBytes + W::place(w_row(tid, j), F == kMx8 ? g : s * 4 + g));
#pragma unroll
    for (int c = 0; c < FN / 4; ++c) r.op.sw[to][c] = *reinterpret_cast<const uint32_t*>(scales + 4 * BM + g * BN + w_row(tid, c * 4));
#pragma unroll
    for (int c = 0; c < FM / 4; ++c) r.op.sx[to][c] = *reinterpret_cast<const uint32_t*>(scales + g * BM + x_row(tid, c * 4));
  }
  template <int Q>
  __device__ __forceinline__ static void products(int s, Regs& r) {
    each_of(std::make_integer_sequence<int, FN>{}, [&](auto j) {
      mx_mma<F, j.value % 4, Q % 4>(r.acc[Q][j.value], r.op.w[s][j.value], r.op.x[Q % kAhead], r.op.sw[s][j.value / 4], r.op.sx[s][Q / 4]);
    });
  }
#else
  // (the checker takes the numbers with their scales)
  template <int G>
  HCNN_HD static float number(const char* line, uint32_t k, uint8_t byte) {
    const uint8_t b = static_cast<uint8_t>(line[G == kMx8 ? k : k / 2]);
    return mx_value<G>(G == kMx8 ? b : b >> (k % 2 * 4) & 15) * (byte == 255 ? std::numeric_limits<float>::quiet_NaN() : mx_scale(byte));
  }
  HCNN_HD static void read_x(const char* slot, int s, int, int q, int tid, Regs& r) {
    const uint32_t row = x_row(tid, q);
    for (uint32_t k = 0; k < 128; ++k) {
      const uint32_t byte = F == kMx8 ? k : s * 64 + k / 2;
      const char* piece = slot + X::place(row, byte / 16);
      r.op.x[q % kAhead][k] = number<F>(piece + byte % 16 - (F == kMx8 ? k : k / 2), k, (uint8_t)slot[kScales + s * kScaleBytes + k / 32 * BM + row]);
    }
  }
  HCNN_HD static void read_w(const char* slot, int s, int to, int tid, Regs& r) {
    for (uint32_t j = 0; j < FN; ++j)
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t row = w_row((tid & ~63) + 4 * (tid % 64 / 16) + e, j);
        for (uint32_t k = 0; k < 128; ++k) {
          const uint32_t byte = (F == kMx8 ? 0 : s * 64) + k / 2;
          const char* piece = slot + X::kLdsBytes + W::place(row, byte / 16);
          r.op.w[to][j * 4 + e][k] = number<kMx4>(piece + byte % 16 - k / 2, k, (uint8_t)slot[kScales + s * kScaleBytes + 4 * BM + k / 32 * BN + row]);
        }
      }
  }
  template <int Q>
  HCNN_HD static void products(int s, Regs& r) {
    for (uint32_t j = 0; j < FN; ++j)
      for (uint32_t e = 0; e < 4; ++e)
        for (uint32_t k = 0; k < 128; ++k) r.acc[Q][j][e] += r.op.x[Q % kAhead][k] * r.op.w[s][j * 4 + e][k];
  }
#endif
  template <int PH>
  HCNN_HD static void phase(const MxArgs& a, unsigned, int tid, uint32_t* lds, Regs& r) {
    if constexpr (PH < 4) {
      constexpr int S = PH / 2;                                        // step of the round
      const uint32_t step = r.iter * 2 + S;
      if (step >= r.steps) return;                                     // (the same for all threads of the workgroup)
      constexpr bool kLast = kSteps == 1 || S == 1;                    // step of the slot
      constexpr int kHere = kSteps == 2 ? S : 0, kNext = kSteps == 2 ? 1 - S : 0;
      const char* base = reinterpret_cast<const char*>(lds);
      if constexpr (PH % 2 == 0) {
        each_of(std::make_integer_sequence<int, FM - kAhead>{}, [&](auto q) {
          products<q.value>(S, r);
          read_x(base + r.here, kHere, S, q.value + kAhead, tid, r);
          sched_fence();
        });
        // the next slot has arrived (the barrier behind this makes it so for all waves); the one behind it may still be on its way
        if constexpr (kLast) direct_all_but<(kSlots - 2) * kLoads>();
      } else {
        // the step's last products, the next one's first operands (behind the last step: of nothing, and not used), and from here on nobody reads this slot
        if (kLast) r.here = r.here == (kSlots - 1) * kSlot ? 0 : r.here + kSlot;
        const char* next = base + r.here;
        read_w(next, kNext, 1 - S, tid, r);
        each_of(std::make_integer_sequence<int, kAhead>{}, [&](auto i) {
          products<FM - kAhead + i.value>(S, r);
          read_x(next, kNext, 1 - S, i.value, tid, r);
          if constexpr (kLast) {
            constexpr int kGroup = (kLoads + kAhead - 1) / kAhead;
#pragma unroll
            for (int d = 0; d < kGroup; ++d)
              if (i.value * kGroup + d < kLoads) bring(i.value * kGroup + d, tid, lds, r);
          }
          sched_fence();
        });
        if (kLast) brought(r);
      }
    } else {
      direct_done();                                                   // (nothing may still be on its way to LDS when the workgroup ends)
      // (the groups and rows as compile-time constants: a loop that the compiler does not unroll would keep the sums in memory)
      each_of(std::make_integer_sequence<int, FN / 4>{}, [&](auto c) {
        // 16 columns side by side: sums 4 e + j of the group's products j
        constexpr int j0 = c.value * 4;
        const uint32_t n = r.n0 + w_row(tid & ~63, j0) + 16 * (tid % 64 / 16);
        if (n >= a.g.N) return;
        const uint32_t left = a.g.N - n;
        float bias[16] = {};
        if (EPI == kEpiOut && a.g.bias) load_row(static_cast<const T*>(a.g.bias) + n, left, bias);
        each_of(std::make_integer_sequence<int, FM / 2>{}, [&](auto p) {
          constexpr int q0 = p.value * 2;
          uint32_t m[2];
          float v[2][16];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            m[q] = r.m0 + x_row(tid, q0 + q);
            if (m[q] >= a.g.M) m[q] = ~0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) v[q][e] = r.acc[q0 + q][j0 + e % 4][e / 4];
          }
          if constexpr (EPI == kEpiOut) {
            size_t row[2];
            finish_values<T>(a.g, m, n, bias, v, row);
            // (whole groups of 64 columns: the same for all lanes of the wave)
            const bool whole = r.n0 + w_row(tid & ~63, j0) + 64 <= a.g.N;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              T* to = static_cast<T*>(a.g.out) + row[q] * a.g.ld_out + n;
              if (whole) store_quads(to, tid % 64 / 16, v[q], m[q] != ~0u);
              else if (m[q] != ~0u) store_row(to, left, v[q]);
            }
          } else {
            const uint32_t quads = (left + 3) / 4 * 4;                 // (rows of sums have room for whole quads)
#pragma unroll
            for (int q = 0; q < 2; ++q)
              if (m[q] != ~0u) store_row(a.g.sums + ((size_t)r.split * a.g.M + m[q]) * a.g.ld_sums + n, quads, v[q]);
          }
        });
      });
    }
  }
};

}  // namespace hcnn
