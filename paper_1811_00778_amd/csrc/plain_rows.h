// Kernels of the plain network that work along the rows of a matrix: dropout, the root-mean-square norm and its gradient, microscaled formats.
// They are bound by memory: every number is read once and written once where a row fits the registers of the threads that share it.
#pragma once
#include "philox.h"
#include "plain_kernels.h"

namespace hcnn {

template <class T> constexpr int kChunk = 16 / (int)sizeof(T);       // numbers of a thread's access

// ---------------------------------------------------------------- microscaled formats
// Blocks of 32 numbers of a row share a power of two 2^e, held as the byte e + 127; numbers are e2m1 (four bits) or e4m3 (eight), as in the OCP
// Microscaling Formats specification (2023): e = floor(log2 A) - kMxTop for a block whose largest magnitude is A (at least -127), numbers are x 2^-e to
// nearest, ties to even, at most the format's largest.  A block of zeros has e = 0; one with an infinity or a NaN the byte 255, which
// stands for NaN, and codes of 0.
enum { kMxNone = 0, kMx4 = 4, kMx8 = 8 };
template <int F> constexpr int kMxTop = F == kMx4 ? 2 : 8;           // exponent of the largest number
HCNN_HD uint32_t mx_byte(uint32_t top, int emax) {                   // top: bits of the largest magnitude
  if (top >= 0x7f800000u) return 255;
  if (top == 0) return 127;
  const int e = (int)(top >> 23) - emax;                             // (numbers below 2^-126 have an exponent of 0 here: far below the least)
  return e > 0 ? (uint32_t)e : 0;
}
HCNN_HD float mx_back(uint32_t byte) { return bits_float((254 - byte) << 23); }                        // 2^-e; byte < 253
HCNN_HD float mx_scale(uint32_t byte) { return bits_float(byte == 0 ? 0x00400000u : byte << 23); }   // 2^e; byte < 255
// what a code stands for (without the scale)
template <int F>
HCNN_HD float mx_value(uint32_t code) {
  if constexpr (F == kMx4) {
    const uint32_t m = code & 7, e = m >> 1;
    const float v = e ? bits_float((e + 126) << 23 | (m & 1) << 22) : (float)m * 0.5f;
    return code & 8 ? -v : v;
  } else {
    const uint32_t m = code & 127, e = m >> 3;
    const float v = m == 127 ? std::numeric_limits<float>::quiet_NaN() : e ? bits_float((e + 120) << 23 | (m & 7) << 20) : (float)m * 0.001953125f;
    return code & 128 ? -v : v;
  }
}
// nearest code of a number below twice the format's largest power of two
template <int F>
HCNN_HD uint32_t mx_code_plain(float q) {
  const uint32_t b = float_bits(q), sign = b >> 31;
  float a = bits_float(b & 0x7fffffffu);
  constexpr float kMost = F == kMx4 ? 6.0f : 448.0f;
  constexpr int kLeast = F == kMx4 ? 127 : 121, kBits = F == kMx4 ? 1 : 3;      // biased exponent of the smallest normal; bits behind the point
  if (a > kMost) a = kMost;
  uint32_t e = float_bits(a) >> 23;
  if (e < (uint32_t)kLeast) e = kLeast;
  // in steps of 2^(e - 127 - kBits): adding 2^23 of them rounds to a whole number of steps, ties to even
  const float magic = bits_float((e + 23 - kBits) << 23);
  volatile float sum = a + magic;
  const uint32_t steps = float_bits(sum) & 0x7fffffu;
  // (a number rounded up to the next power of two has twice 2^kBits steps: its code follows from the same sum)
  return sign << (F - 1) | (((e - kLeast) << kBits) + steps);
}
// codes of W scaled numbers, the first one lowest
template <int F, int W>
HCNN_HD uint64_t mx_codes(const float (&q)[W]) {
#if defined(__HIP_DEVICE_COMPILE__)
  uint32_t w[2] = {0, 0};
  if constexpr (F == kMx4) {
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], q[0], q[1], 1.0f, 0);
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], q[2], q[3], 1.0f, 1);
    if constexpr (W == 8) {
      w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], q[4], q[5], 1.0f, 2);
      w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[0], q[6], q[7], 1.0f, 3);
    }
  } else {
    // (the conversion makes numbers beyond the largest NaN)
    float c[W];
#pragma unroll
    for (int i = 0; i < W; ++i) c[i] = __builtin_amdgcn_fmed3f(q[i], -448.0f, 448.0f);
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      w[i / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[i], c[i + 1], (int)w[i / 4], false);
      w[i / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[i + 2], c[i + 3], (int)w[i / 4], true);
    }
  }
  return (uint64_t)w[1] << 32 | w[0];
#else
  uint64_t r = 0;
  for (int i = 0; i < W; ++i) r |= (uint64_t)mx_code_plain<F>(q[i]) << (F * i);
  return r;
#endif
}
// A microscaled matrix: codes [rows][row_bytes], 0 behind a row's numbers up to whole 128; the blocks' bytes [columns up to whole 128 / 32][pitch >= rows], so
// that the rows' bytes of a block lie side by side: a matrix instruction's operand takes 16 rows of one block in a lane's 16.
struct MxOut {
  uint8_t *codes, *scales;
  size_t row_bytes, pitch;
};
// W scaled numbers of row `row` at column c, and their block's byte by one of its threads
template <int F, int W>
HCNN_HD void mx_store(const MxOut& o, size_t row, uint32_t c, const float (&q)[W], uint32_t byte) {
  const uint64_t codes = mx_codes<F>(q);
  uint8_t* to = o.codes + row * o.row_bytes + c / 8 * F;
  if constexpr (F * W == 64) {
    *reinterpret_cast<uint64_t*>(to) = codes;
  } else if constexpr (F * W == 32) {
    *reinterpret_cast<uint32_t*>(to + (W == 4 ? c % 8 / 4 * 4 : 0)) = (uint32_t)codes;
  } else {
    *reinterpret_cast<uint16_t*>(to + c % 8 / 4 * 2) = (uint16_t)codes;
  }
  if (c % 32 == 0) o.scales[c / 32 * o.pitch + row] = (uint8_t)byte;
}
// The largest of the threads of a block (32 / W neighbours); the checker looks at the block's numbers instead
template <int W, class Numbers>
HCNN_HD uint32_t block_top(uint32_t own, uint32_t c, Numbers&& numbers) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int d = 1; d < 32 / W; d *= 2) {
    const uint32_t other = (uint32_t)__shfl_xor((int)own, d);
    own = own > other ? own : other;
  }
  return own;
#else
  uint32_t top = 0;
  for (uint32_t at = c / 32 * 32; at < c / 32 * 32 + 32; at += W) {
    float v[W];
    numbers(at, v);
    for (int i = 0; i < W; ++i)
      if ((float_bits(v[i]) & 0x7fffffffu) > top) top = float_bits(v[i]) & 0x7fffffffu;
  }
  (void)own;
  return top;
#endif
}
template <int W>
HCNN_HD uint32_t top_of(const float (&v)[W]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const uint32_t b = float_bits(v[i]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
  return top;
}
// v's numbers that exist; the others are 0
template <class T, int W>
HCNN_HD void load_some(const T* row, uint32_t c, uint32_t n, float (&v)[W]) {
  if (c < n) load_row(row + c, n - c, v);
  else
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = 0.0f;
}

// A launch over the chunks of all rows: a workgroup takes kThreads * EACH consecutive ones.
struct Chunks {
  uint64_t all;                // chunks
  FastDiv per_row;
  uint32_t groups;             // workgroups
};
struct Chunk { size_t row; uint32_t at; };
// Where the run that begins at chunk `first` of all begins (first: the same in the workgroup)
HCNN_HD Chunk chunk_of(const Chunks& s, uint64_t first) {
  const uint64_t row = first / s.per_row.d;
  return Chunk{(size_t)row, (uint32_t)(first - row * s.per_row.d)};
}
HCNN_HD Chunk chunk_behind(const Chunks& s, Chunk c, uint32_t i) {
  const uint32_t at = c.at + i, q = quot(at, s.per_row);
  return Chunk{c.row + q, at - q * s.per_row.d};
}

// Bound by memory: 16384 x 4096 bfloat16 numbers to four bits with their values, 304 MB, in 60 us a call among others (5.0 TB/s), 67 by the profiler; by its launch at 1021 x 517.  The rounding is the conversion
// instruction's (nearest, ties to even; beyond the largest cut to it, for eight bits before the instruction), the scaling in front of it exact.
// A workgroup takes tiles of 128 columns by as many rows as it has threads for (16, of 32-bit numbers 8): the rows' bytes of a block's scales, which lie side by side, leave
// together (a row's worth of columns at a time, with a byte here and there: two us more).
struct QuantizeArgs {
  Chunks tiles;                // rows: groups of Quantize::kRows; chunks: tiles of 128 columns
  const void* x;
  size_t ldx;
  uint32_t rows, n;
  MxOut to;
  void* values;                // what the codes and scales stand for (may be null)
  size_t ld_values;
};
template <class T, int F>
struct Quantize {
  static constexpr int kThreads = 256, W = kChunk<T>, EACH = 4, kAcross = 128 / W, kRows = kThreads / kAcross;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const QuantizeArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    for (uint64_t run = bid; run * EACH < a.tiles.all; run += a.tiles.groups) {
      const uint64_t first = run * EACH;
      const Chunk start = chunk_of(a.tiles, first);
      float v[EACH][W];
      size_t row[EACH];
      uint32_t c[EACH];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const Chunk k = chunk_behind(a.tiles, start, (uint32_t)i);
        row[i] = first + i < a.tiles.all ? k.row * kRows + tid / kAcross : a.rows;
        c[i] = k.at * 128 + tid % kAcross * W;
        if (row[i] < a.rows) load_some(static_cast<const T*>(a.x) + row[i] * a.ldx, c[i], a.n, v[i]);
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        // (the threads of a block are of one row)
        if (row[i] >= a.rows) continue;
        const uint32_t top = block_top<W>(top_of(v[i]), c[i], [&](uint32_t at, float (&u)[W]) { load_some(static_cast<const T*>(a.x) + row[i] * a.ldx, at, a.n, u); });
        const uint32_t byte = mx_byte(top, kMxTop<F>);
        const float back = byte == 255 ? 0.0f : mx_back(byte);
        float q[W];
#pragma unroll
        for (int e = 0; e < W; ++e) q[e] = byte == 255 ? 0.0f : v[i][e] * back;
        mx_store<F>(a.to, row[i], c[i], q, byte);
        if (a.values && c[i] < a.n) {
          const uint64_t codes = mx_codes<F>(q);
          const float scale = byte == 255 ? std::numeric_limits<float>::quiet_NaN() : mx_scale(byte);
#pragma unroll
          for (int e = 0; e < W; ++e) q[e] = mx_value<F>((uint32_t)(codes >> (F * e)) & ((1u << F) - 1)) * scale;
          store_row(static_cast<T*>(a.values) + row[i] * a.ld_values + c[i], a.n - c[i], q);
        }
      }
    }
  }
};

// ---------------------------------------------------------------- dropout
// y = residual + (word >= threshold ? x * scale : 0): word c mod 4 of the generator's four for the counter (c div 4, row, stream, kKindDropout 2^24) decides
// about column c of a row.  The mask is a function of (seed, stream, row, column): the backward pass forms it again, whatever type or strides it has.
// Bound by memory: the words cost five multiply-adds and ten exclusive-ors a number, less than half of the time that 16-bit numbers take.  8192 x 16384 bfloat16 with the
// residual, 805 MB, in 147 us a call among others (5.5 TB/s), 157 by the profiler; 8192 x 800 in 32 bits 9.8 and 10.4.
constexpr uint32_t kKindDropout = 4;         // (the samplers of polynomials are kinds 1 to 3)
struct DropoutArgs {
  Chunks chunks;
  const void *x, *residual;
  void* y;
  size_t ldx, ld_residual, ldy;
  uint32_t n;
  uint32_t threshold, none;    // none: nothing is kept
  float scale;
  uint64_t seed;
  uint32_t stream;
};
template <class T, bool RESIDUAL>
struct Dropout {
  static constexpr int kThreads = 256, W = kChunk<T>, EACH = 2;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const DropoutArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    for (uint64_t run = bid; run * (kThreads * EACH) < a.chunks.all; run += a.chunks.groups) {
      const uint64_t first = run * (kThreads * EACH);
      const Chunk start = chunk_of(a.chunks, first);
      float x[EACH][W], r[EACH][W];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const Chunk k = chunk_behind(a.chunks, start, (uint32_t)(i * kThreads + tid));
        if (first + i * kThreads + tid >= a.chunks.all) continue;
        load_row(static_cast<const T*>(a.x) + k.row * a.ldx + k.at * W, a.n - k.at * W, x[i]);
        if (RESIDUAL) load_row(static_cast<const T*>(a.residual) + k.row * a.ld_residual + k.at * W, a.n - k.at * W, r[i]);
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (first + i * kThreads + tid >= a.chunks.all) continue;
        const Chunk k = chunk_behind(a.chunks, start, (uint32_t)(i * kThreads + tid));
        const uint32_t c = k.at * W;
#pragma unroll
        for (int q = 0; q < W; q += 4) {
          const PhiloxWords words = philox4x32_10((c + q) / 4, (uint32_t)k.row, a.stream, kKindDropout << 24, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float kept = words.w[e] >= a.threshold && !a.none ? x[i][q + e] * a.scale : 0.0f;
            x[i][q + e] = RESIDUAL ? kept + r[i][q + e] : kept;
          }
        }
        store_row(static_cast<T*>(a.y) + k.row * a.ldy + c, a.n - c, x[i]);
      }
    }
  }
};

// ---------------------------------------------------------------- root-mean-square norm
// Sums over the LANES threads of a row, THREADS of a workgroup, of COUNT 64-bit numbers a thread: within a wave by exchanges, between waves (or, in the checker,
// between all threads) through LDS.  give(), a barrier where a row has more than a wave, total().
template <int LANES, int THREADS, int COUNT>
struct RowSum {
  static constexpr size_t kLdsBytes = (size_t)COUNT * THREADS * 8;
#if defined(__HIP_DEVICE_COMPILE__)
  __device__ __forceinline__ static void give(double* lds, int tid, double (&v)[COUNT]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
#pragma unroll
      for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v[i] += __shfl_xor(v[i], d);
      if (LANES > 64 && tid % 64 == 0) lds[i * (THREADS / 64) + tid / 64] = v[i];
    }
  }
  __device__ __forceinline__ static void total(const double* lds, int tid, double (&v)[COUNT]) {
    if constexpr (LANES > 64) {
      const int first = tid / LANES * (LANES / 64);
#pragma unroll
      for (int i = 0; i < COUNT; ++i) {
        v[i] = 0.0;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) v[i] += lds[i * (THREADS / 64) + first + w];
      }
    }
  }
#else
  HCNN_HD static void give(double* lds, int tid, double (&v)[COUNT]) {
    for (int i = 0; i < COUNT; ++i) lds[i * THREADS + tid] = v[i];
  }
  HCNN_HD static void total(const double* lds, int tid, double (&v)[COUNT]) {
    for (int i = 0; i < COUNT; ++i) {
      v[i] = 0.0;
      for (int l = 0; l < LANES; ++l) v[i] += lds[i * THREADS + tid / LANES * LANES + l];
    }
  }
#endif
};

// 1 / sqrt(mean of squares + eps) as one * two: rows of numbers near the largest have an inverse below the smallest normal 32-bit number
struct RowScale { float one, two; double whole; };
HCNN_HD RowScale row_scale(double squares, double per, double eps) {
  RowScale r;
  r.whole = 1.0 / sqrt(squares * per + eps);
  r.two = r.whole < 7.888609052210118e-31 ? 5.421010862427522e-20f : 1.0f;        // 2^-100; 2^-64
  r.one = (float)(r.whole < 7.888609052210118e-31 ? r.whole * 18446744073709551616.0 : r.whole);
  return r;
}
// A 64-bit number rounded to odd at 21 bits: what is rounded to fewer bits after this is rounded as if from the 64 bits.  (Below 2^-129 the conversion rounds to nearest.)
HCNN_HD float to_odd(double x) {
  uint64_t b;
  __builtin_memcpy(&b, &x, 8);
  const uint64_t kept = (b >> 32 | ((uint32_t)b != 0)) << 32;
  double y;
  __builtin_memcpy(&y, &kept, 8);
  return (float)y;
}
// The same of a number whose 32-bit one is no normal number: rounded to odd at 32 bits' least step
HCNN_HD float to_odd_small(double x) {
  const double steps = __builtin_fabs(x) * 0x1p149;
  if (!(steps < 0x1p20)) return to_odd(x);
  const uint32_t whole = (uint32_t)steps;
  return __builtin_copysignf(bits_float(whole | (whole != steps)), (float)x);
}

struct NormRowsArgs {
  const void *x, *residual, *weight;       // residual, weight may be null
  size_t ldx, ld_residual;
  uint32_t rows, n;
  uint32_t first;                           // row that the launch begins with
  double per, eps;                          // per: 1 / n
  void *h, *y;                              // h: x + residual, rounded (may be null)
  size_t ldh, ldy;
  MxOut to;                                 // F: in y's place
};
// y = h / sqrt(mean of h^2 + eps) * weight, h = x + residual in 32 bits.  LANES threads share a row and hold it in their registers, EL numbers each; EL = 0: rows
// of any length, read a second time for y.  Squares are summed in 64 bits: none of a 32-bit number's leaves the range, and no sum of a row's is rounded to fewer
// bits than the numbers have.  With F the numbers are scaled and weighted in 64 bits and rounded to odd on the way to 32, so that they are rounded to the
// format's few bits once: rounded to 32 bits on the way, one in a million next to a border would end on its other side.  Bound by memory: 8192 x 4096 bfloat16 with the
// residual in and its sum out, 268 MB, in 43 us by the profiler (6.2 TB/s, part of it out of the last cache), 51 a call among others; one row of 4096 into eight bits 4.6 us by the profiler, two waits for
// memory and the launch.
template <class T, int LANES, int EL, int F>
struct NormRows {
  static constexpr int kThreads = LANES > 256 ? LANES : 256, W = kChunk<T>, kLines = kThreads / LANES;
  static constexpr int kHeld = EL ? EL / W : 1;
#if defined(HCNN_HOSTEMU)
  static constexpr bool kBehind = F != kMxNone;       // (the checker's threads look at each other's numbers for a block's scale: sums leave in a phase of their own)
#else
  static constexpr bool kBehind = false;
#endif
  static constexpr int kPhases = kBehind ? 3 : 2;
  typedef RowSum<LANES, kThreads, 1> Sum;
  static constexpr size_t kLdsBytes = Sum::kLdsBytes;
  struct Regs { float h[kHeld][W]; double sum[1]; };
  static constexpr bool wave_sync(int) { return LANES <= 64; }
  // h at column c of the row, stored where `keep`
  HCNN_HD static void numbers(const NormRowsArgs& a, size_t row, uint32_t c, bool keep, float (&h)[W]) {
    load_some(static_cast<const T*>(a.x) + row * a.ldx, c, a.n, h);
    if (c >= a.n) return;
    if (a.residual) {
      float r[W];
      load_row(static_cast<const T*>(a.residual) + row * a.ld_residual + c, a.n - c, r);
#pragma unroll
      for (int e = 0; e < W; ++e) h[e] += r[e];
    }
    if (keep && a.h) store_row(static_cast<T*>(a.h) + row * a.ldh + c, a.n - c, h);
  }
  HCNN_HD static void add(const float (&h)[W], double& sum) {
#pragma unroll
    for (int e = 0; e < W; ++e) sum += (double)h[e] * h[e];
  }
  HCNN_HD static void weights(const NormRowsArgs& a, uint32_t c, float (&w)[W]) {
    if (a.weight) load_some(static_cast<const T*>(a.weight), c, a.n, w);
    else
#pragma unroll
      for (int e = 0; e < W; ++e) w[e] = 1.0f;
  }
  // in place of h: the row's numbers that are rounded to few bits (F)
  HCNN_HD static void fine(const NormRowsArgs& a, const RowScale& s, uint32_t c, float (&h)[W]) {
    if (c >= a.n) return;                   // (0 behind the row, also where the row is NaN)
    float w[W];
    double v[W];
    weights(a, c, w);
    bool small = false;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      v[e] = (double)h[e] * w[e] * s.whole;
      h[e] = to_odd(v[e]);
      small |= (float_bits(h[e]) & 0x7fffffffu) < 0x00800000u;
    }
    if (small) {
#pragma unroll
      for (int e = 0; e < W; ++e) h[e] = to_odd_small(v[e]);
    }
  }
  HCNN_HD static void finish_chunk(const NormRowsArgs& a, size_t row, uint32_t c, const RowScale& s, float (&h)[W]) {
    if constexpr (F == kMxNone) {
      if (c >= a.n) return;
      float w[W];
      weights(a, c, w);
#pragma unroll
      for (int e = 0; e < W; ++e) h[e] = h[e] * s.two * s.one * w[e];
      store_row(static_cast<T*>(a.y) + row * a.ldy + c, a.n - c, h);
    } else {
      fine(a, s, c, h);
      const uint32_t top = block_top<W>(top_of(h), c, [&](uint32_t at, float (&u)[W]) {
        numbers(a, row, at, false, u);
        fine(a, s, at, u);
      });
      const uint32_t byte = mx_byte(top, kMxTop<F>);
      const float back = byte == 255 ? 0.0f : mx_back(byte);
#pragma unroll
      for (int e = 0; e < W; ++e) h[e] = byte == 255 ? 0.0f : h[e] * back;
      if (c < a.to.row_bytes / F * 8) mx_store<F>(a.to, row, c, h, byte);
    }
  }
  template <int PH>
  HCNN_HD static void phase(const NormRowsArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs& r) {
    double* lds = reinterpret_cast<double*>(lds_words);
    const size_t row = a.first + (size_t)bid * kLines + tid / LANES;
    const uint32_t lane = (uint32_t)tid % LANES;
    const bool here = row < a.rows;
    const uint32_t end = F == kMxNone ? a.n : (a.n + 127) / 128 * 128;
    if constexpr (PH == 0) {
      r.sum[0] = 0.0;
      if (here) {
        if constexpr (EL > 0) {
#pragma unroll
          for (int i = 0; i < kHeld; ++i) numbers(a, row, (i * LANES + lane) * W, !kBehind, r.h[i]);
#pragma unroll
          for (int i = 0; i < kHeld; ++i) add(r.h[i], r.sum[0]);
        } else {
          for (uint32_t c = lane * W; c < a.n; c += LANES * W) {
            numbers(a, row, c, false, r.h[0]);
            add(r.h[0], r.sum[0]);
          }
        }
      }
      Sum::give(lds, tid, r.sum);
    } else if constexpr (PH == 2) {
      float h[W];
      for (uint32_t c = lane * W; here && c < a.n; c += LANES * W) numbers(a, row, c, true, h);
    } else if (here) {
      Sum::total(lds, tid, r.sum);
      const RowScale s = row_scale(r.sum[0], a.per, a.eps);
      if constexpr (EL > 0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) finish_chunk(a, row, (i * LANES + lane) * W, s, r.h[i]);
      } else {
        // (the sum leaves now: it may take the place of x or the residual, which the row's second reading needs)
        for (uint32_t c = lane * W; c < end; c += LANES * W) {
          numbers(a, row, c, !kBehind, r.h[0]);
          finish_chunk(a, row, c, s, r.h[0]);
        }
      }
    }
  }
};

// Gradient from h as it is stored: with u = h / sqrt(mean of h^2 + eps), both sums of a row in one pass,
//   dx = (w dy - u mean(w dy u)) / sqrt(...) + dh,   dw = sum over rows of dy u.
// Bound by memory: 8192 x 4096 bfloat16 with dh, 268 MB, in 60 us by the profiler and 5.4 for the columns' sums (without the next row's loads ahead, and with sums of 16 columns a
// workgroup, 76 and 18).  30011 x 77 in 32 bits 14 and 4: two fifths of the threads' numbers lie beyond the row.
// A workgroup takes rows_each rows, kLines at a time; the columns' sums stay in its threads' registers and leave once, in 32 bits, for QuadSums.
struct NormGradArgs {
  const void *dy, *h, *weight, *dh;         // weight, dh may be null
  size_t ld_dy, ldh, ld_dh;
  uint32_t rows, n, rows_each;              // rows_each: a multiple of the rows taken at a time
  double per, eps;
  void* dx;
  size_t ld_dx;
  float* part;                              // [workgroups][ld_part] (null: no dw)
  size_t ld_part;
  double* inverse;                          // EL = 0: [rows] 1 / sqrt(mean of squares + eps), for NormColumns
};
template <class T, int LANES, int EL>
struct NormGrad {
  static constexpr int kThreads = LANES > 256 ? LANES : 256, W = kChunk<T>, kLines = kThreads / LANES;
  static constexpr int kHeld = EL ? EL / W : 1;
  static constexpr int kLoopPhases = 2, kPhases = 4;
  // (the host gives a compute unit as many workgroups: with one fewer there, 8192 x 4096 took twice the time)
  static constexpr int kMinWavesPerSimd = kThreads == 1024 ? 4 : EL == 16 ? (sizeof(T) == 4 ? 2 : 3) : sizeof(T) == 4 ? 4 : 5;
  typedef RowSum<LANES, kThreads, 2> Sum;
  static constexpr size_t kSumBytes = 2 * Sum::kLdsBytes;                        // two, taken in turn: a barrier an iteration
  static constexpr size_t kLdsBytes = kSumBytes + (kLines > 1 ? (size_t)kLines * LANES * EL * 4 : 0);
  // A row as it lies in memory (the next one is asked for before the sums of this one are known, where the registers have room for it) and the weights, for all rows
  static constexpr bool kNext = LANES < 1024 || EL < 16;
  struct Raw { U4 v[kHeld]; };
  struct Regs {
    uint32_t iter;
    Raw w, dy, h, dh;
    U4 now[kHeld];                          // dh of the row at hand
    float dyf[kHeld][W], hf[kHeld][W], dw[kHeld][W];
    double sum[2];
  };
  static constexpr bool wave_sync(int ph) { return ph == 1 || (ph == 0 && LANES <= 64); }
  HCNN_HD static uint32_t loop_count(const NormGradArgs& a) { return a.rows_each / kLines; }
  HCNN_HD static size_t row_of(const NormGradArgs& a, unsigned bid, int tid, uint32_t iter) { return (size_t)bid * a.rows_each + (size_t)iter * kLines + tid / LANES; }
  HCNN_HD static void widened(const U4& v, float (&to)[W]) {
    T t[W];
    __builtin_memcpy(t, &v, 16);
#pragma unroll
    for (int e = 0; e < W; ++e) to[e] = Num<T>::widen(t[e]);
  }
  // (`otherwise` where there is no such number, or no row)
  HCNN_HD static void load(const T* row, uint32_t n, uint32_t lane, float otherwise, Raw& r) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const uint32_t c = (i * LANES + lane) * W;
      U4 v;
      if (row && c + W <= n) {
        v = ld16(reinterpret_cast<const char*>(row + c));
      } else {
        T t[W];
#pragma unroll
        for (int e = 0; e < W; ++e) t[e] = row && c + e < n ? row[c + e] : Num<T>::narrow(otherwise);
        __builtin_memcpy(&v, t, 16);
      }
      r.v[i] = v;
    }
  }
  HCNN_HD static void ask(const NormGradArgs& a, size_t row, uint32_t lane, Regs& r) {
    if (row >= a.rows) return;
    load(static_cast<const T*>(a.dy) + row * a.ld_dy, a.n, lane, 0.0f, r.dy);
    load(static_cast<const T*>(a.h) + row * a.ldh, a.n, lane, 0.0f, r.h);
    load(a.dh ? static_cast<const T*>(a.dh) + row * a.ld_dh : nullptr, a.n, lane, 0.0f, r.dh);
  }
  HCNN_HD static void begin(const NormGradArgs& a, unsigned bid, int tid, uint32_t*, Regs& r) {
    if constexpr (EL > 0) {
      const uint32_t lane = (uint32_t)tid % LANES;
      load(static_cast<const T*>(a.weight), a.n, lane, 1.0f, r.w);
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) r.dw[i][e] = 0.0f;
      if (kNext) ask(a, row_of(a, bid, tid, 0), lane, r);
    }
  }
  HCNN_HD static void add(const float (&g)[W], const float (&h)[W], double (&sum)[2]) {
#pragma unroll
    for (int e = 0; e < W; ++e) {
      sum[0] += (double)h[e] * h[e];
      sum[1] += (double)g[e] * h[e];
    }
  }
  // g = weight dy, h: to dx and, in h's place, u
  HCNN_HD static void finish_chunk(const RowScale& s, float mean, const float (&g)[W], float (&h)[W], float (&dx)[W]) {
#pragma unroll
    for (int e = 0; e < W; ++e) h[e] *= s.one;
    if (s.two != 1.0f) {
#pragma unroll
      for (int e = 0; e < W; ++e) h[e] *= s.two;
    }
#pragma unroll
    for (int e = 0; e < W; ++e) dx[e] = (g[e] - h[e] * mean) * s.one;
    if (s.two != 1.0f) {
#pragma unroll
      for (int e = 0; e < W; ++e) dx[e] *= s.two;
    }
  }
  // rows of any length
  HCNN_HD static void load_long(const NormGradArgs& a, size_t row, uint32_t c, float (&dy)[W], float (&h)[W]) {
    load_some(static_cast<const T*>(a.dy) + row * a.ld_dy, c, a.n, dy);
    load_some(static_cast<const T*>(a.h) + row * a.ldh, c, a.n, h);
    if (a.weight) {
      float w[W];
      load_some(static_cast<const T*>(a.weight), c, a.n, w);
#pragma unroll
      for (int e = 0; e < W; ++e) dy[e] *= w[e];
    }
  }
  template <int PH>
  HCNN_HD static void phase(const NormGradArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs& r) {
    double* lds = reinterpret_cast<double*>(reinterpret_cast<char*>(lds_words) + r.iter % 2 * Sum::kLdsBytes);
    const uint32_t lane = (uint32_t)tid % LANES, line = (uint32_t)tid / LANES;
    const size_t row = row_of(a, bid, tid, r.iter);
    const bool here = row < a.rows;
    if constexpr (PH == 0) {
      r.sum[0] = r.sum[1] = 0.0;
      if (here) {
        if constexpr (EL > 0) {
          if (!kNext) ask(a, row, lane, r);
#pragma unroll
          for (int i = 0; i < kHeld; ++i) {
            float g[W];
            widened(r.dy.v[i], r.dyf[i]);
            widened(r.h.v[i], r.hf[i]);
            widened(r.w.v[i], g);
            r.now[i] = r.dh.v[i];
#pragma unroll
            for (int e = 0; e < W; ++e) g[e] *= r.dyf[i][e];
            add(g, r.hf[i], r.sum);
          }
          if (kNext && r.iter + 1 < loop_count(a)) ask(a, row + kLines, lane, r);
        } else {
          for (uint32_t c = lane * W; c < a.n; c += LANES * W) {
            load_long(a, row, c, r.dyf[0], r.hf[0]);
            add(r.dyf[0], r.hf[0], r.sum);
          }
        }
      }
      Sum::give(lds, tid, r.sum);
    } else if constexpr (PH == 1) {
      if (!here) return;
      Sum::total(lds, tid, r.sum);
      const RowScale s = row_scale(r.sum[0], a.per, a.eps);
      const float mean = (float)(r.sum[1] * a.per * s.whole);
      if constexpr (EL > 0) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
          const uint32_t c = (i * LANES + lane) * W;
          float g[W], dx[W], d[W];
          widened(r.w.v[i], g);
          widened(r.now[i], d);
#pragma unroll
          for (int e = 0; e < W; ++e) g[e] *= r.dyf[i][e];
          finish_chunk(s, mean, g, r.hf[i], dx);
#pragma unroll
          for (int e = 0; e < W; ++e) {
            dx[e] += d[e];
            r.dw[i][e] += r.dyf[i][e] * r.hf[i][e];
          }
          if (c < a.n) store_row(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.n - c, dx);
        }
      } else {
        if (lane == 0 && a.inverse) a.inverse[row] = s.whole;
        for (uint32_t c = lane * W; c < a.n; c += LANES * W) {
          float dx[W], d[W];
          load_long(a, row, c, r.dyf[0], r.hf[0]);
          finish_chunk(s, mean, r.dyf[0], r.hf[0], dx);
          if (a.dh) {
            load_row(static_cast<const T*>(a.dh) + row * a.ld_dh + c, a.n - c, d);
#pragma unroll
            for (int e = 0; e < W; ++e) dx[e] += d[e];
          }
          store_row(static_cast<T*>(a.dx) + row * a.ld_dx + c, a.n - c, dx);
        }
      }
    } else if constexpr (EL > 0) {
      if (!a.part) return;
      float* lines = reinterpret_cast<float*>(reinterpret_cast<char*>(lds_words) + kSumBytes);        // [kLines][LANES * EL]
      constexpr uint32_t kCols = LANES * EL;
      float* to = a.part + (size_t)bid * a.ld_part;
      if constexpr (PH == 2) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
          const uint32_t c = (i * LANES + lane) * W;
          if constexpr (kLines > 1) {
            // (store_row is for memory, not for LDS)
#pragma unroll
            for (int e = 0; e < W; ++e) lines[line * kCols + c + e] = r.dw[i][e];
          } else if (c < a.n) {
            store_row(to + c, (a.n - c + 3) / 4 * 4, r.dw[i]);                          // (rows of parts have room for whole quads)
          }
        }
      } else if (kLines > 1) {
        for (uint32_t c = tid; c < kCols && c < a.n; c += kThreads) {
          float s = 0.0f;
#pragma unroll
          for (int l = 0; l < kLines; ++l) s += lines[l * kCols + c];
          to[c] = s;
        }
      }
    }
  }
};
// Sums of the workgroups' sums: a workgroup takes 32 columns, a quad for each of 32 threads, which share the parts.
template <class T>
struct QuadSums {
  static constexpr int kThreads = 256, kSide = 32;
  static constexpr int kPhases = 2;
  static constexpr size_t kLdsBytes = kThreads * 16;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const ColumnSumArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    float* lds = reinterpret_cast<float*>(lds_words);              // [kSide][32]
    if constexpr (PH == 0) {
      const uint32_t n = bid * 32 + tid % 8 * 4;
      float s[4] = {};
      if (n < a.N) {
#pragma unroll 8
        for (uint32_t b = tid / 8; b < a.blocks; b += kSide) {
          float v[4];
          load_row(a.part + b * a.ld_part + n, v);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] += v[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) lds[tid * 4 + e] = s[e];
    } else if (tid < 32 && bid * 32 + tid < a.N) {
      float s = 0.0f;
#pragma unroll
      for (int l = 0; l < kSide; ++l) s += lds[l * 32 + tid];
      static_cast<T*>(a.out)[bid * 32 + tid] = Num<T>::narrow(s);
    }
  }
};
// The columns' sums of rows that do not fit the registers: a workgroup takes kThreads * 4 columns of rows_each rows
template <class T>
struct NormColumns {
  static constexpr int kThreads = 256, kCols = kThreads * 4;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const NormGradArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    const uint32_t blocks = (a.n + kCols - 1) / kCols, rb = bid / blocks, c = bid % blocks * kCols + tid * 4;
    if (c >= a.n) return;
    const uint32_t m0 = rb * a.rows_each, m1 = a.rows - m0 < a.rows_each ? a.rows : m0 + a.rows_each;
    float sum[4] = {};
#pragma unroll 4
    for (uint32_t m = m0; m < m1; ++m) {
      float dy[4], h[4];
      load_row(static_cast<const T*>(a.dy) + m * a.ld_dy + c, a.n - c, dy);
      load_row(static_cast<const T*>(a.h) + m * a.ldh + c, a.n - c, h);
      const double inverse = a.inverse[m];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += dy[e] * (float)(h[e] * inverse);
    }
    store_row(a.part + (size_t)rb * a.ld_part + c, a.n - c, sum);
  }
};

}  // namespace hcnn
