// Kernels of the plain (unencrypted) network's training: matrix products with what follows them, softmax cross entropy, the
// norm of many gradients.  Sums, statistics and norms are held in 32 bits or more; 16-bit numbers are widened on the way in
// and rounded once on the way out (to nearest, ties to even).
#pragma once
#include <cmath>
#include <limits>

#include "platform.h"

namespace hcnn {

// ---------------------------------------------------------------- numbers
struct Half { uint16_t bits; };        // IEEE binary16
struct Bfloat { uint16_t bits; };      // the upper half of a binary32

HCNN_HD float bits_float(uint32_t b) { float f; __builtin_memcpy(&f, &b, 4); return f; }
HCNN_HD uint32_t float_bits(float f) { uint32_t b; __builtin_memcpy(&b, &f, 4); return b; }

template <class T> struct Num;
template <> struct Num<float> {
  HCNN_HD static float widen(float x) { return x; }
  HCNN_HD static float narrow(float x) { return x; }
};
template <> struct Num<Bfloat> {
  HCNN_HD static float widen(Bfloat x) { return bits_float((uint32_t)x.bits << 16); }
  HCNN_HD static Bfloat narrow(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(Bfloat, (__bf16)x);
#else
    const uint32_t b = float_bits(x);
    if ((b & 0x7fffffffu) > 0x7f800000u) return Bfloat{(uint16_t)(b >> 16 | 0x40)};       // a NaN stays one
    return Bfloat{(uint16_t)((b + 0x7fffu + (b >> 16 & 1)) >> 16)};
#endif
  }
};
template <> struct Num<Half> {
  HCNN_HD static float widen(Half x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return (float)__builtin_bit_cast(_Float16, x);
#else
    const uint32_t s = (uint32_t)(x.bits >> 15) << 31, e = x.bits >> 10 & 31, m = x.bits & 1023;
    if (e == 31) return bits_float(s | 0x7f800000u | m << 13);
    if (e) return bits_float(s | (e + 112) << 23 | m << 13);
    const float v = (float)m * 5.9604644775390625e-8f;                                    // m * 2^-24
    return s ? -v : v;
#endif
  }
  HCNN_HD static Half narrow(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(Half, (_Float16)x);
#else
    const uint32_t b = float_bits(x), s = b >> 16 & 0x8000, a = b & 0x7fffffffu;
    if (a > 0x7f800000u) return Half{(uint16_t)(s | 0x7e00)};
    if (a >= 0x477ff000u) return Half{(uint16_t)(s | 0x7c00)};                            // rounds to 2^16 or more
    if (a < 0x38800000u) {                                                                // below 2^-14: steps of 2^-24
      const float steps = bits_float(a) * 16777216.0f;                                    // exact
      return Half{(uint16_t)(s | (uint32_t)(int)std::nearbyint(steps))};
    }
    return Half{(uint16_t)(s | ((a + 0xfffu + (a >> 13 & 1)) - 0x38000000u) >> 13)};
#endif
  }
};

// 2^x and e^x to about one unit of the last place of the exponent function unit (e^x: and |x| 2^-24 for the product)
HCNN_HD float exp2_of(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_exp2f(x);
#else
  return std::exp2(x);
#endif
}
HCNN_HD float exp_of(float x) { return exp2_of(x * 1.44269504088896340736f); }

// ---------------------------------------------------------------- accesses of any alignment
// The device's global accesses take any address; types of alignment 1 tell the compiler so.
#if defined(__HIP_DEVICE_COMPILE__)
typedef uint32_t hcnn_any4 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t hcnn_any2 __attribute__((ext_vector_type(2), aligned(1)));
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wold-style-cast"
__device__ __forceinline__ U4 ld16(const char* p) {
  const hcnn_any4 v = *(const hcnn_any4 __attribute__((address_space(1)))*)p;
  U4 r; r.x = v.x; r.y = v.y; r.z = v.z; r.w = v.w;
  return r;
}
__device__ __forceinline__ void st16(char* p, U4 v) { *(hcnn_any4 __attribute__((address_space(1)))*)p = hcnn_any4{v.x, v.y, v.z, v.w}; }
__device__ __forceinline__ uint64_t ld8(const char* p) { return __builtin_bit_cast(uint64_t, (hcnn_any2)*(const hcnn_any2 __attribute__((address_space(1)))*)p); }
__device__ __forceinline__ void st8(char* p, uint64_t v) { *(hcnn_any2 __attribute__((address_space(1)))*)p = __builtin_bit_cast(hcnn_any2, v); }
#pragma clang diagnostic pop
#else
HCNN_HD U4 ld16(const char* p) { U4 v; __builtin_memcpy(&v, p, 16); return v; }
HCNN_HD void st16(char* p, U4 v) { __builtin_memcpy(p, &v, 16); }
HCNN_HD uint64_t ld8(const char* p) { uint64_t v; __builtin_memcpy(&v, p, 8); return v; }
HCNN_HD void st8(char* p, uint64_t v) { __builtin_memcpy(p, &v, 8); }
#endif

// W numbers in a row (4, 8 or 16), widened
template <class T, int W>
HCNN_HD void load_row(const T* p, float (&v)[W]) {
  T t[W];
  if constexpr (W * sizeof(T) == 8) {
    const uint64_t w = ld8(reinterpret_cast<const char*>(p));
    __builtin_memcpy(t, &w, 8);
  } else {
#pragma unroll
    for (size_t i = 0; i < W * sizeof(T); i += 16) {
      const U4 w = ld16(reinterpret_cast<const char*>(p) + i);
      __builtin_memcpy(reinterpret_cast<char*>(t) + i, &w, 16);
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = Num<T>::widen(t[i]);
}
template <class T, int W>
HCNN_HD void store_row(T* p, const float (&v)[W]) {
  T t[W];
#pragma unroll
  for (int i = 0; i < W; ++i) t[i] = Num<T>::narrow(v[i]);
  if constexpr (W * sizeof(T) == 8) {
    uint64_t w;
    __builtin_memcpy(&w, t, 8);
    st8(reinterpret_cast<char*>(p), w);
  } else {
#pragma unroll
    for (size_t i = 0; i < W * sizeof(T); i += 16) {
      U4 w;
      __builtin_memcpy(&w, reinterpret_cast<char*>(t) + i, 16);
      st16(reinterpret_cast<char*>(p) + i, w);
    }
  }
}
// ... of which only the first `left` exist
template <class T, int W>
HCNN_HD void load_row(const T* p, uint32_t left, float (&v)[W]) {
  if (left >= W) return load_row(p, v);
#pragma unroll
  for (uint32_t q = 0; q < W; q += 4) {
    float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (left >= q + 4) load_row(p + q, t);
    else
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (q + i < left) t[i] = Num<T>::widen(p[q + i]);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[q + i] = t[i];
  }
}
template <class T, int W>
HCNN_HD void store_row(T* p, uint32_t left, const float (&v)[W]) {
  if (left >= W) return store_row(p, v);
#pragma unroll
  for (uint32_t q = 0; q < W; q += 4) {
    const float t[4] = {v[q], v[q + 1], v[q + 2], v[q + 3]};
    if (left >= q + 4) store_row(p + q, t);
    else
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (q + i < left) p[q + i] = Num<T>::narrow(t[i]);
  }
}

// ---------------------------------------------------------------- room in binary16
// The power of two that brings numbers, the largest of them of magnitude `top` (its bits), to below 2^15, the largest to 2^14 or more (numbers below
// 2^-86: times 2^100); and its inverse.
HCNN_HD uint32_t room_exponent(uint32_t top) { return top >> 23 > 41 ? top >> 23 : 41; }
HCNN_HD float room_of(uint32_t top) { return bits_float((268 - room_exponent(top)) << 23); }
HCNN_HD float room_back(uint32_t top) { return bits_float((room_exponent(top) - 14) << 23); }

// ---------------------------------------------------------------- activations
enum { kActNone = 0, kActSquare = 1, kActRelu = 2, kActGelu = 3, kActSilu = 4, kActCount = 5 };
HCNN_HD float recip(float x) {            // to about one unit of the last place
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_rcpf(x);
#else
  return 1.0f / x;
#endif
}
// P(X <= z) of a normal X, and bell = e^(-z^2 / 2).  The tail is bell * Q(t) with t = 1 / (1 + c |z|), the form of Hastings' approximations (1955), and
// Q a polynomial without constant term: c and Q fit P(X <= -a) e^(a^2 / 2) on 0 <= a <= 14 in the sense of the least largest relative error, by least
// squares whose weights are raised where the error is large, for 40 c between 0.15 and 0.8.  Relative errors of the tail: 1.4e-7 of the
// fit, below 1e-6 + 1e-7 z^2 in 32 bits (measured 5e-7 down to z = -2, 1.3e-6 to -5, 8e-6 to -13), where the rounding of z^2 in the exponent is most of
// it.  It costs a third of the library's erf (134 M numbers of a layer's ending: 100 us, now 55).
HCNN_HD float normal_cdf(float z, float* bell) {
  const float t = recip(1.0f + 0.23333333333f * fabsf(z)), e = exp2_of(-0.72134752044f * z * z);
  float q = -0.06778094120f;
  q = q * t + 0.23061270695f;
  q = q * t - 0.17640544687f;
  q = q * t + 0.20500715358f;
  q = q * t + 0.02320650282f;
  q = q * t + 0.10073172775f;
  q = q * t + 0.09145269742f;
  q = q * t + 0.09317556141f;
  q = q * t * e;
  *bell = e;
  return z < 0.0f ? q : 1.0f - q;
}
HCNN_HD float act_of(float z, int act) {
  float bell;
  switch (act) {
    case kActSquare: return z * z;
    case kActRelu: return z > 0.0f || z != z ? z : 0.0f;
    case kActGelu: return z * normal_cdf(z, &bell);
    case kActSilu: return z * recip(1.0f + exp_of(-z));
  }
  return z;
}
template <int B, int W>
HCNN_HD void act_all(float (&v)[B][W], int act) {
  switch (act) {
#define PLAIN_ACT(A)                    \
  case A:                               \
    _Pragma("unroll") for (int i = 0; i < B * W; ++i) v[i / W][i % W] = act_of(v[i / W][i % W], A); \
    break
    PLAIN_ACT(kActSquare);
    PLAIN_ACT(kActRelu);
    PLAIN_ACT(kActGelu);
    PLAIN_ACT(kActSilu);
#undef PLAIN_ACT
  }
}
HCNN_HD float slope_of(float z, int act) {
  switch (act) {
    case kActSquare: return 2.0f * z;
    case kActRelu: return z > 0.0f || z != z ? 1.0f : 0.0f;
    case kActGelu: {
      float bell;
      const float c = normal_cdf(z, &bell);
      return c + z * bell * 0.39894228040143267794f;
    }
    case kActSilu: {
      const float s = recip(1.0f + exp_of(-z));
      return s * (1.0f + z * (1.0f - s));
    }
  }
  return 1.0f;
}

// ---------------------------------------------------------------- matrix products
// out[m][n] = sum_k a(m, k) b(n, k).  An operand is stored with its contraction index k contiguous (kAlongK: a[m][k]) or with
// its output index contiguous (kAcrossK: a[k][m]).  A workgroup computes a tile of BM x BN outputs in WM x WN waves; a stage is 128
// bytes of k (64 numbers of 16 bits, 32 of 32) in two steps, and LDS holds two stages.  While a step's products run, the next step's operands go
// from LDS to registers.  One barrier a stage, between its steps: behind it the stage's operands are all in registers, the stage after
// next comes from memory to its place, and the next one, which was asked for a stage earlier, has arrived.  (Four stages of half the size in the same
// memory and a load's time of two: a barrier for half as many products cost 8 %.)
//   kAlongK  in LDS [row][8 pieces of 16 bytes], piece p of a row at p ^ (row mod 8): the 16 rows x 4 pieces that a wave reads at once
//            spread evenly over the banks
//   kAcrossK in LDS [k][rows] as it lies in memory, in granules of 16 rows; 16-bit numbers are read with the transposing LDS read
//            (16 lanes: 4 k x 16 rows in, 4 k of one row out), 32-bit ones word by word
// Products: v_mfma_f32_16x16x32 (16 bits) and v_mfma_f32_16x16x4_f32.  A lane's 16 bytes of an operand are k 8 g .. 8 g + 7 (16 bits) or
// 4 g .. 4 g + 3 (32 bits) of a row, g = lane / 16; both operands use the same order, so that the sum is the same whatever the instruction
// calls these k.  b is the first operand: a lane then holds four consecutive n of a row m = lane mod 16, and, by the choice of b's rows for
// each product (GemmOperand), 4 FN consecutive n in all: whole 128-byte lines of 16-bit numbers for each row leave without a way through LDS
// (that way, in two halves of the tile with a barrier before and behind each, took 7 of 110 us of a tile with 4096 k).
enum { kAlongK = 0, kAcrossK = 1 };
enum { kCountNone = 0, kCountM = 1, kCountK = 2 };         // what GemmArgs::count limits

struct GemmArgs {
  const void *a, *b;
  size_t lda, ldb;             // numbers from one stored row to the next
  size_t a_extent, b_extent;   // numbers from the first to the last one that exists, inclusive
  uint32_t M, N, K;
  const uint32_t* count;       // device count of the rows that take part, see count_of
  uint32_t count_of;
  const void* kept;            // the operand with those rows only (a with kCountM, b with kCountK), read where they are not all rows
  size_t ld_kept;
  uint32_t kept_always;        // ... or in any case
  const uint32_t* rows;        // row of the output that m goes to (null: m)
  uint32_t splits;             // parts of k, each summed by workgroups of its own
  // what becomes of the sums
  float* sums;                 // [splits][M][ld_sums] where kEpiSums
  size_t ld_sums;              // a multiple of 8
  const float* addend;         // [M][ld_sums], added to the sums of the first part (may be null; may be `sums`)
  const float* alpha;          // device factor of the sums (may be null)
  const uint32_t* top;         // [M] binary16: the sums of row m are room_of(top[m]) times too large (may be null)
  int act;
  const void* bias;            // [N]
  const void* residual;
  void *out, *z;
  size_t ld_residual, ld_out, ld_z;
  // softmax
  float* stats;                // [tiles of n][2][ld_stats]: largest score, sum of exponentials relative to it
  size_t ld_stats;
  const uint32_t* target;      // [rows that take part]
  float* target_score;
  const float* lse;
  float delta_scale;
  uint32_t n_offset;           // class of column 0
};

// What the linear layer makes of B x W sums: W in a row, of the rows m[.] of the output (~0: none).  `bias`: of these columns, 0 where there is none.
template <class T, int B, int W>
HCNN_HD void finish(const GemmArgs& a, const uint32_t (&m)[B], uint32_t n, const float (&bias)[W], float (&v)[B][W]) {
  const uint32_t left = a.N - n;
  size_t row[B];
  float r[B][W];
#pragma unroll
  for (int i = 0; i < B; ++i) {
    row[i] = a.rows && m[i] != ~0u ? a.rows[m[i]] : m[i];
    if (a.residual && m[i] != ~0u) load_row(static_cast<const T*>(a.residual) + row[i] * a.ld_residual + n, left, r[i]);
  }
  if (a.alpha) {
    const float alpha = *a.alpha;
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) v[i][e] *= alpha;
  }
  if constexpr (std::is_same_v<T, Half>)
    if (a.top) {
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const float back = m[i] != ~0u ? room_back(a.top[m[i]]) : 0.0f;
#pragma unroll
        for (int e = 0; e < W; ++e) v[i][e] *= back;
      }
    }
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int e = 0; e < W; ++e) v[i][e] += bias[e];
  if (a.z) {
#pragma unroll
    for (int i = 0; i < B; ++i)
      if (m[i] != ~0u) store_row(static_cast<T*>(a.z) + row[i] * a.ld_z + n, left, v[i]);
  }
  act_all(v, a.act);
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) v[i][e] += r[i][e];
  }
#pragma unroll
  for (int i = 0; i < B; ++i)
    if (m[i] != ~0u) store_row(static_cast<T*>(a.out) + row[i] * a.ld_out + n, left, v[i]);
}

enum { kEpiOut = 0, kEpiSums = 1, kEpiStats = 2, kEpiDelta = 3 };

template <class T> struct GemmNum {
  static constexpr uint32_t kPer16 = 16 / sizeof(T);       // numbers in 16 bytes
  static constexpr uint32_t kStage = 128 / sizeof(T);      // k of a stage
};

// One operand's way through a workgroup: BX rows of the output index, THREADS threads.  The 16 rows that a wave takes for one product are four
// runs of four, GROUP rows apart: with GROUP = 4 sixteen rows in a row; b takes 4 x its products of a wave, so that the sums of a lane
// in all of them lie side by side.
template <class T, int LAYOUT, int BX, int THREADS, int GROUP = 4>
struct GemmOperand {
  static constexpr uint32_t kPer16 = GemmNum<T>::kPer16, kStage = GemmNum<T>::kStage;
  static constexpr int kPieces = BX * 8;                                       // of 16 bytes in a stage
  static constexpr int kEach = (kPieces + THREADS - 1) / THREADS;
  static constexpr uint32_t kRowPieces = LAYOUT == kAlongK ? 8 : BX / kPer16;  // in a stored row of the stage
  static constexpr uint32_t kGranules = BX / 16;
  static constexpr uint32_t kLdsBytes = BX * 128;

  HCNN_HD static bool mine(int tid, int i) { return kPieces % THREADS == 0 || tid + i * THREADS < kPieces; }

  // 16 bytes of the numbers at `off`; those that do not exist are left 0
  HCNN_HD static U4 piece(const T* p, size_t off, size_t extent) {
    if (off + kPer16 <= extent) return ld16(reinterpret_cast<const char*>(p + off));
    T t[kPer16] = {};
#pragma unroll
    for (uint32_t e = 0; e < kPer16; ++e)
      if (off + e < extent) t[e] = p[off + e];
    U4 v;
    __builtin_memcpy(&v, t, 16);
    return v;
  }
  // the first `left` numbers of a piece
  HCNN_HD static U4 first(U4 v, uint32_t left) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = i < left ? w[i] : 0u;
      else w[i] = 2 * i + 1 < left ? w[i] : 2 * i < left ? w[i] & 0xffffu : 0u;
    }
    U4 r; r.x = w[0]; r.y = w[1]; r.z = w[2]; r.w = w[3];
    return r;
  }
  // Pieces of the stage that begins at k0, of the rows from x0 on.  Rows beyond X and what lies beyond them may hold anything (their sums
  // are dropped), k beyond K are 0 in both operands.
  HCNN_HD static void load(const T* p, size_t ld, size_t extent, uint32_t X, uint32_t K, uint32_t x0, uint32_t k0, int tid, U4 (&r)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (mine(tid, i)) r[i] = load_one(p, ld, extent, X, K, x0, k0, (uint32_t)(tid + i * THREADS));
  }
  HCNN_HD static U4 load_one(const T* p, size_t ld, size_t extent, uint32_t X, uint32_t K, uint32_t x0, uint32_t k0, uint32_t c) {
    const uint32_t line = c / kRowPieces, at = c % kRowPieces * kPer16;
    U4 v{};
    {
      if constexpr (LAYOUT == kAlongK) {
        uint32_t x = x0 + line;
        if (x >= X) x = X - 1;
        const uint32_t k = k0 + at;
        if (k < K) {
          v = piece(p, x * ld + k, extent);
          if (K - k < kPer16) v = first(v, K - k);
        }
      } else {
        const uint32_t k = k0 + line, x = x0 + at;
        if (k < K && x < X) {
          v = piece(p, k * ld + x, extent);
        }
      }
    }
    return v;
  }
  // ... straight to LDS, DEEP pieces at a time: for the one stage of a sum that is not whole
  template <int DEEP>
  HCNN_HD static void copy(const T* p, size_t ld, size_t extent, uint32_t X, uint32_t K, uint32_t x0, uint32_t k0, char* lds, int tid) {
#pragma unroll 1
    for (int i0 = 0; i0 < kEach; i0 += DEEP) {
      U4 v[DEEP];
#pragma unroll
      for (int i = 0; i < DEEP; ++i)
        if (i0 + i < kEach && mine(tid, i0 + i)) v[i] = load_one(p, ld, extent, X, K, x0, k0, (uint32_t)(tid + (i0 + i) * THREADS));
#pragma unroll
      for (int i = 0; i < DEEP; ++i) {
        const uint32_t c = (uint32_t)(tid + (i0 + i) * THREADS);
        if (i0 + i < kEach && mine(tid, i0 + i)) *reinterpret_cast<U4*>(lds + place(c / kRowPieces, c % kRowPieces)) = v[i];
      }
    }
  }
  HCNN_HD static uint32_t place(uint32_t line, uint32_t pc) {                  // byte of piece pc of stored row `line`
    if constexpr (LAYOUT == kAlongK) return line * 128 + ((pc ^ turn(line)) << 4);
    else return line * (BX * sizeof(T)) + (moved(line, pc) << 4);
  }
  // kAlongK: piece p of row x lies at p ^ turn(x), which takes eight values in the 16 rows that are read at once
  HCNN_HD static uint32_t turn(uint32_t x) { return (x & 3) + (x / GROUP & 1) * 4; }
  // kAcrossK: piece pc of stored row k lies at moved(k, pc), its own inverse: within its granule of 16 numbers and the granules by the bits
  // of k in which the lanes of one read differ, as far as those do not differ in the granule or the piece themselves.
  HCNN_HD static uint32_t moved(uint32_t k, uint32_t pc) {
    constexpr uint32_t kIn = sizeof(T) == 2 ? 2 : 4, kMask = kGranules & (kGranules - 1) ? 0 : kGranules - 1;   // pieces of a granule
    uint32_t granule, piece = 0;
    if constexpr (sizeof(T) == 2) {
      granule = GROUP == 4 ? (k & 3) + (k >> 3 & 1) * 4 : GROUP == 8 ? (k & 3) * 2 : (k & 1) * 4;
      if (GROUP == 16) piece = k >> 1 & 1;
    } else {
      granule = GROUP == 4 ? k >> 2 & 3 : GROUP == 8 ? (k >> 3 & 1) * 2 : 0;
      piece = GROUP == 4 ? 0 : GROUP == 8 ? k >> 2 & 1 : k >> 2 & 3;
    }
    return (pc / kIn ^ (granule & kMask)) * kIn + (pc % kIn ^ piece);
  }
  HCNN_HD static void store(char* lds, int tid, const U4 (&r)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (!mine(tid, i)) continue;
      const uint32_t c = (uint32_t)(tid + i * THREADS);
      *reinterpret_cast<U4*>(lds + place(c / kRowPieces, c % kRowPieces)) = r[i];
    }
  }
  // ---- memory to LDS without registers: whole stages of operands whose stored rows all start on 16 bytes.  The LDS side of such a load
  // is fixed (a wave writes 64 x 16 bytes in a row), so that the order of the pieces within a stored row is made on the memory side.
  HCNN_HD static uint32_t numbers(uint32_t c) {                                 // of a row at LDS piece c, from the stage's first number
    const uint32_t line = c / kRowPieces, pc = c % kRowPieces;
    if constexpr (LAYOUT == kAlongK) return (pc ^ turn(line)) * kPer16;
    else return moved(line, pc) * kPer16;
  }
  // Byte offsets of a thread's pieces from direct_base, for the whole sum.  Rows beyond X read a row that exists, pieces beyond X the
  // row's first one.
  HCNN_HD static void direct_offsets(size_t ld, uint32_t X, uint32_t x0, int tid, uint32_t (&off)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (!mine(tid, i)) continue;
      const uint32_t c = (uint32_t)(tid + i * THREADS), line = c / kRowPieces, at = numbers(c);
      if constexpr (LAYOUT == kAlongK) {
        const uint32_t x = x0 + line < X ? line : X - 1 - x0;
        off[i] = (uint32_t)((x * ld + at) * sizeof(T));
      } else {
        off[i] = (uint32_t)((line * ld + (x0 + at < X ? at : 0)) * sizeof(T));
      }
    }
  }
  HCNN_HD static const T* direct_base(const T* p, size_t ld, uint32_t x0, uint32_t k0) {
    if constexpr (LAYOUT == kAlongK) return p + x0 * ld + k0;
    else return p + k0 * ld + x0;
  }
  // May the stage at k0 be read whole?  Its k exist, and a last piece that reaches beyond the row's numbers reads memory of the operand.
  HCNN_HD static bool direct_stage(size_t ld, size_t extent, uint32_t X, uint32_t K, uint32_t k0) {
    if (k0 + kStage > K) return false;
    if constexpr (LAYOUT == kAlongK) return true;
    return X % kPer16 == 0 || (size_t)(k0 + kStage - 1) * ld + X / kPer16 * kPer16 + kPer16 <= extent;
  }
  HCNN_HD static void direct(const T* base, char* lds, int tid, int i, const uint32_t (&off)[kEach]) {
    if (mine(tid, i)) to_lds(base, off[i], lds + ((tid & ~63) + i * THREADS) * 16, tid & 63);
  }
  // 16 bytes of every lane of a wave to LDS, side by side
  HCNN_HD static void to_lds(const T* base, uint32_t off, char* lds, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t at = wave_uniform((uint32_t)(uintptr_t)lds);             // (the low half of an LDS pointer is its offset)
    // (as an instruction of its own: of the builtin the compiler only knows that it writes LDS, and has every later LDS read wait for it)
    // (m0: what the compiler has put there for an access of its own is gone; its warning that m0 is reserved is about allocating it)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(off), "s"(base) : "memory", "m0");
#pragma clang diagnostic pop
#else
    __builtin_memcpy(lds + lane * 16, reinterpret_cast<const char*>(base) + off, 16);
#endif
  }
  // row of lane i (of 16) for product j
  HCNN_HD static uint32_t row_of(uint32_t j, uint32_t i) { return GROUP == 4 ? j * 16 + i : i / 4 * GROUP + j * 4 + i % 4; }
  // 16 bytes of the lane's row of step s of a stage, for product j of the wave whose first row is `base` (a multiple of 16)
#if defined(__HIP_DEVICE_COMPILE__)
  __device__ __forceinline__ static hcnn_word4 read(const char* lds, uint32_t base, uint32_t j, uint32_t s, uint32_t lane) {
    const uint32_t g = lane / 16, i = lane % 16;
    if constexpr (LAYOUT == kAlongK) {
      return *reinterpret_cast<const hcnn_word4*>(lds + place(base + row_of(j, i), s * 4 + g));
    } else if constexpr (sizeof(T) == 2) {
      // (lanes 4 l .. 4 l + 3 of 16 point at the four runs of rows at k = l)
      typedef short four __attribute__((ext_vector_type(4)));
      typedef four __attribute__((address_space(3)))* lptr;
      const uint32_t k = s * 32 + g * 8 + i / 4, x = base + row_of(j, i % 4 * 4);
      const four lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(lds + place(k, x / 8) + x % 8 * 2));
      const four hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(lds + place(k + 4, x / 8) + x % 8 * 2));
      typedef uint32_t two __attribute__((ext_vector_type(2)));
      const two l = __builtin_bit_cast(two, lo), h = __builtin_bit_cast(two, hi);
      return hcnn_word4{l.x, l.y, h.x, h.y};
    } else {
      hcnn_word4 v;
      const uint32_t x = base + row_of(j, i);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e)
        v[e] = *reinterpret_cast<const uint32_t*>(lds + place(s * 16 + g * 4 + e, x / 4) + x % 4 * 4);
      return v;
    }
  }
#endif
  // number (row, k) of the stage, for the checker
  HCNN_HD static float at(const char* lds, uint32_t row, uint32_t k) {
    T t;
    if constexpr (LAYOUT == kAlongK) __builtin_memcpy(&t, lds + place(row, k / kPer16) + k % kPer16 * sizeof(T), sizeof(T));
    else __builtin_memcpy(&t, lds + place(k, row / kPer16) + row % kPer16 * sizeof(T), sizeof(T));
    return Num<T>::widen(t);
  }
};

#if defined(__HIP_DEVICE_COMPILE__)
typedef float hcnn_float4 __attribute__((ext_vector_type(4)));
// acc += b (16 n) x a (16 m) over a step
template <class T>
__device__ __forceinline__ void mma(hcnn_float4& acc, hcnn_word4 b, hcnn_word4 a) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)b[j]), __builtin_bit_cast(float, (uint32_t)a[j]), acc, 0, 0, 0);
  } else if constexpr (std::is_same_v<T, Half>) {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, b), __builtin_bit_cast(v8, a), acc, 0, 0, 0);
  } else {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, b), __builtin_bit_cast(v8, a), acc, 0, 0, 0);
  }
}
#else
struct hcnn_float4 {
  float v[4];
  HCNN_HD float& operator[](int i) { return v[i]; }
  HCNN_HD float operator[](int i) const { return v[i]; }
};
#endif

// What is on its way to LDS past the registers has arrived
HCNN_HD void direct_done() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#endif
}

template <class T, int LA, int LB, int BM, int BN, int WM, int WN, int EPI, bool DIRECT>
struct Gemm {
  static constexpr int kThreads = WM * WN * 64;
  static constexpr int kLoopPhases = 2;
  static constexpr int kPhases = EPI == kEpiStats ? 4 : 3;
  static constexpr int kMinWavesPerSimd = 2;
  static constexpr uint32_t kStage = GemmNum<T>::kStage;
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  typedef GemmOperand<T, LA, BM, kThreads> A;
  // 16-bit sums: a lane's lie side by side, 32 bytes of a row; 32-bit ones: those of four lanes do, 64 bytes of a row in one store
  static constexpr int kGroup = sizeof(T) == 2 ? 4 * FN : 4;
  typedef GemmOperand<T, LB, BN, kThreads, kGroup> B;
  static constexpr uint32_t kBuffer = A::kLdsBytes + B::kLdsBytes;
  static constexpr size_t kLdsBytes = 2 * kBuffer;
  static_assert(EPI != kEpiStats || BM * WN * 4 * 8 <= kLdsBytes, "the statistics fit the stages' memory");

  // Operands of the running step.  The next one's take the place of an a as soon as its products are under way; b and the last kAhead
  // of a have two places, so that their reads come first and the step's end does not wait for one that was just asked for.
  static constexpr int kAhead = LA == kAlongK && FM >= 8 ? 2 : 0;
  static constexpr uint32_t kStep = kStage / 2;
#if defined(__HIP_DEVICE_COMPILE__)
  struct Step { hcnn_word4 a[FM + kAhead], b[2][FN]; };
#else
  struct Step { float a[FM + kAhead][kStep], b[2][FN * 4][kStep]; };
#endif
  struct Regs {
    uint32_t iter;
    uint32_t m0, n0, k_begin, k_end, M, split;
    const T *a, *b;
    size_t lda, ldb, a_extent, b_extent;
    U4 ra[A::kEach], rb[B::kEach];               // the next stage, unless DIRECT
    uint32_t oa[A::kEach], ob[B::kEach];         // DIRECT: offsets of the pieces
    Step step;
    hcnn_float4 acc[FM][FN];
  };

  HCNN_HD static uint32_t counted(const GemmArgs& a, uint32_t which, uint32_t all) {
    if (a.count_of != which) return all;
    const uint32_t c = wave_uniform(*a.count);
    return c < all ? c : all;
  }
  // stages of each part of k
  HCNN_HD static uint32_t loop_count(const GemmArgs& a) {
    const uint32_t stages = (counted(a, kCountK, a.K) + kStage - 1) / kStage;
    return (stages + a.splits - 1) / a.splits;
  }
  static constexpr bool wave_sync(int ph) { return ph == 1; }
  // Workgroups go round the eight dies; each die takes a run of consecutive tiles, which walk through bands of four tiles of m, so
  // that the operands' rows that its workgroups read at a time are few.  Tiles beyond the counted rows are not in the order.
  HCNN_HD static bool skip(const GemmArgs& a, unsigned bid) {
    if (a.count_of != kCountM) return false;
    const uint64_t tiles = (uint64_t)((counted(a, kCountM, a.M) + BM - 1) / BM) * ((a.N + BN - 1) / BN) * a.splits;
    return bid >= tiles;
  }
  HCNN_HD static void place(const GemmArgs& a, unsigned bid, Regs& r) {
    r.M = counted(a, kCountM, a.M);
    const uint32_t tm = (r.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN, all = tm * tn * a.splits;
    const uint32_t die = bid % 8, each = all / 8, rest = all % 8;
    uint32_t at = die * each + (die < rest ? die : rest) + bid / 8;
    r.split = at / (tm * tn);
    at -= r.split * (tm * tn);
    constexpr uint32_t kBand = 4;
    const uint32_t band = at / (kBand * tn), high = tm - band * kBand < kBand ? tm - band * kBand : kBand;
    at -= band * kBand * tn;
    r.m0 = (band * kBand + at % high) * BM;
    r.n0 = at / high * BN;
    const bool kept = a.kept && (a.kept_always || wave_uniform(*a.count) < (a.count_of == kCountM ? a.M : a.K));
    r.a = static_cast<const T*>(kept && a.count_of == kCountM ? a.kept : a.a);
    r.b = static_cast<const T*>(kept && a.count_of == kCountK ? a.kept : a.b);
    r.lda = kept && a.count_of == kCountM ? a.ld_kept : a.lda;
    r.ldb = kept && a.count_of == kCountK ? a.ld_kept : a.ldb;
    r.a_extent = kept && a.count_of == kCountM ? a.M * a.ld_kept : a.a_extent;
    r.b_extent = kept && a.count_of == kCountK ? a.K * a.ld_kept : a.b_extent;
    const uint32_t K = counted(a, kCountK, a.K), run = loop_count(a) * kStage;
    r.k_begin = r.split * run;
    r.k_end = K < r.k_begin + run ? K : r.k_begin + run;
  }
  HCNN_HD static void fetch(const GemmArgs& a, uint32_t k0, int tid, Regs& r) {
    A::load(r.a, r.lda, r.a_extent, r.M, r.k_end, r.m0, k0, tid, r.ra);
    B::load(r.b, r.ldb, r.b_extent, a.N, r.k_end, r.n0, k0, tid, r.rb);
  }
  HCNN_HD static void keep(char* lds, int tid, const Regs& r) {
    A::store(lds, tid, r.ra);
    B::store(lds + A::kLdsBytes, tid, r.rb);
  }
  // The stage at k0 to LDS, past the registers where it may be read whole: then in kDirect pieces that the caller spreads out
  static constexpr int kDirect = A::kEach + B::kEach;
  static constexpr int kCopyDeep = FM * FN >= 32 ? 1 : 4;      // (the largest tile has no registers to spare)
  struct Bring {
    const T *pa, *pb;
    char* lds;
    bool whole;
    HCNN_HD Bring(const GemmArgs& a, uint32_t k0, char* to, bool wanted, int tid, const Regs& r) : lds(to), whole(false) {
      if (!wanted) return;
      whole = A::direct_stage(r.lda, r.a_extent, r.M, r.k_end, k0) && B::direct_stage(r.ldb, r.b_extent, a.N, r.k_end, k0);
      pa = A::direct_base(r.a, r.lda, r.m0, k0);
      pb = B::direct_base(r.b, r.ldb, r.n0, k0);
      if (whole) return;
      A::template copy<kCopyDeep>(r.a, r.lda, r.a_extent, r.M, r.k_end, r.m0, k0, lds, tid);
      B::template copy<kCopyDeep>(r.b, r.ldb, r.b_extent, a.N, r.k_end, r.n0, k0, lds + A::kLdsBytes, tid);
    }
    HCNN_HD void piece(int i, int tid, const Regs& r) const {
      if (i < A::kEach) A::direct(pa, lds, tid, i, r.oa);
      else B::direct(pb, lds + A::kLdsBytes, tid, i - A::kEach, r.ob);
    }
    HCNN_HD void all(int tid, const Regs& r) const {
      if (!whole) return;
#pragma unroll
      for (int i = 0; i < kDirect; ++i) piece(i, tid, r);
    }
  };
  HCNN_HD static void begin(const GemmArgs& a, unsigned bid, int tid, uint32_t* lds, Regs& r) {
    place(a, bid, r);
    if constexpr (DIRECT) {
      A::direct_offsets(r.lda, r.M, r.m0, tid, r.oa);
      B::direct_offsets(r.ldb, a.N, r.n0, tid, r.ob);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) r.acc[i][j][e] = 0.0f;
    char* l = reinterpret_cast<char*>(lds);
    if constexpr (DIRECT) {
      Bring(a, r.k_begin, l, true, tid, r).all(tid, r);
      Bring(a, r.k_begin + kStage, l + kBuffer, r.k_begin + kStage < r.k_end, tid, r).all(tid, r);
      direct_done();
    } else {
      fetch(a, r.k_begin, tid, r);
      keep(l, tid, r);
      fetch(a, r.k_begin + kStage, tid, r);
    }
  }
  HCNN_HD static void begin_next(const GemmArgs&, unsigned, int tid, uint32_t* lds, Regs& r) {
#pragma unroll
    for (int i = 0; i < FM; ++i) read_a(reinterpret_cast<char*>(lds), 0, i, tid, r);
#pragma unroll
    for (int j = 0; j < FN; ++j) read_b(reinterpret_cast<char*>(lds), 0, j, tid, r);
  }
  HCNN_HD static uint32_t m_wave(int tid) { return (uint32_t)tid / 64 / WN * (FM * 16); }
  HCNN_HD static uint32_t n_wave(int tid) { return (uint32_t)tid / 64 % WN * (FN * 16); }
  // place of a's i-th operand of step s
  static constexpr int a_place(int s, int i) { return s && i >= FM - kAhead ? i + kAhead : i; }
#if defined(__HIP_DEVICE_COMPILE__)
  __device__ __forceinline__ static void read_a(const char* lds, int s, int i, int tid, Regs& r) {
    r.step.a[a_place(s, i)] = A::read(lds, m_wave(tid), i, s, tid % 64);
  }
  __device__ __forceinline__ static void read_b(const char* lds, int s, int j, int tid, Regs& r) {
    r.step.b[s][j] = B::read(lds + A::kLdsBytes, n_wave(tid), j, s, tid % 64);
  }
  __device__ __forceinline__ static void products(int s, int i, Regs& r) {
#pragma unroll
    for (int j = 0; j < FN; ++j) mma<T>(r.acc[i][j], r.step.b[s][j], r.step.a[a_place(s, i)]);
  }
#else
  // (the checker keeps the numbers that a lane's four sums of each 16 x 16 take)
  HCNN_HD static void read_a(const char* lds, int s, int i, int tid, Regs& r) {
    for (uint32_t k = 0; k < kStep; ++k) r.step.a[a_place(s, i)][k] = A::at(lds, m_wave(tid) + i * 16 + tid % 16, s * kStep + k);
  }
  HCNN_HD static void read_b(const char* lds, int s, int j, int tid, Regs& r) {
    for (uint32_t e = 0; e < 4; ++e)
      for (uint32_t k = 0; k < kStep; ++k) r.step.b[s][j * 4 + e][k] = B::at(lds + A::kLdsBytes, n_wave(tid) + B::row_of(j, tid % 64 / 16 * 4 + e), s * kStep + k);
  }
  HCNN_HD static void products(int s, int i, Regs& r) {
    for (int j = 0; j < FN; ++j)
      for (uint32_t e = 0; e < 4; ++e)
        for (uint32_t k = 0; k < kStep; ++k) r.acc[i][j][e] += r.step.a[a_place(s, i)][k] * r.step.b[s][j * 4 + e][k];
  }
#endif
  // The products of step s, and the operands of the step after it from `next`
  template <class Each>
  HCNN_HD static void multiply(const char* next, int s, int tid, Regs& r, Each&& each) {
#pragma unroll
    for (int j = 0; j < FN; ++j) read_b(next, 1 - s, j, tid, r);
#pragma unroll
    for (int i = FM - kAhead; i < FM; ++i) read_a(next, 1 - s, i, tid, r);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      products(s, i, r);
      if (i < FM - kAhead) read_a(next, 1 - s, i, tid, r);
      each(i);
      sched_fence();
    }
  }

  template <int PH>
  HCNN_HD static void phase(const GemmArgs& a, unsigned, int tid, uint32_t* lds_words, Regs& r) {
    char* lds = reinterpret_cast<char*>(lds_words);
    const uint32_t wave = (uint32_t)tid / 64, lane = (uint32_t)tid % 64;
    const uint32_t m_lane = wave / WN * (FM * 16) + lane % 16, n_wave0 = wave % WN * (FN * 16);   // in the tile
    if constexpr (PH < 2) {
      char *here = lds + r.iter % 2 * kBuffer, *next = lds + (r.iter + 1) % 2 * kBuffer;
      const uint32_t k0 = r.k_begin + r.iter * kStage;
      if constexpr (PH == 0) {
        if (k0 < r.k_end) multiply(here, 0, tid, r, [](int) {});
        if constexpr (DIRECT) direct_done();
        else if (k0 + kStage < r.k_end) keep(next, tid, r);
      } else if constexpr (DIRECT) {
        const Bring bring(a, k0 + 2 * kStage, here, k0 + 2 * kStage < r.k_end, tid, r);
        if (k0 < r.k_end)
          multiply(next, 1, tid, r, [&](int i) {
            // (each behind some products: in front of them all, the matrix unit waited for their issue)
            if (bring.whole) {
              constexpr int kGroup = (kDirect + FM - 1) / FM;
#pragma unroll
              for (int d = 0; d < kGroup; ++d)
                if (i * kGroup + d < kDirect) bring.piece(i * kGroup + d, tid, r);
            }
          });
      } else {
        if (k0 + 2 * kStage < r.k_end) fetch(a, k0 + 2 * kStage, tid, r);
        if (k0 < r.k_end) multiply(next, 1, tid, r, [](int) {});
      }
    } else if constexpr (EPI != kEpiStats) {
      // a lane has W numbers side by side of FM rows, 4 FN / W times; R rows at a time (two: their residuals come together)
      constexpr int W = kGroup, R = FM % 2 == 0 ? 2 : 1;
#pragma unroll
      for (int j0 = 0; j0 < FN; j0 += W / 4) {
        const uint32_t n = r.n0 + n_wave0 + B::row_of(j0, lane / 16 * 4);
        if (n >= a.N) continue;
        const uint32_t left = a.N - n;
        float bias[W] = {};
        if (EPI == kEpiOut && a.bias) load_row(static_cast<const T*>(a.bias) + n, left, bias);
#pragma unroll
        for (int i0 = 0; i0 < FM; i0 += R) {
          uint32_t m[R];
          float v[R][W];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            m[i] = r.m0 + m_lane + (i0 + i) * 16;
            if (m[i] >= r.M) m[i] = ~0u;
#pragma unroll
            for (int e = 0; e < W; ++e) v[i][e] = r.acc[i0 + i][j0 + e / 4][e % 4];
          }
          if constexpr (EPI == kEpiDelta) {
            // the gradient of the row's loss for its scores, times delta_scale: an operand of the two products after this, so that
            // it is rounded to their type here
#pragma unroll
            for (int i = 0; i < R; ++i) {
              if (m[i] == ~0u) continue;
              const float lse = a.lse[m[i]];
              const uint32_t t = a.target[m[i]] - a.n_offset;
#pragma unroll
              for (uint32_t e = 0; e < W; ++e) v[i][e] = (exp_of(v[i][e] - lse) - (n + e == t ? 1.0f : 0.0f)) * a.delta_scale;
              store_row(static_cast<T*>(a.out) + (size_t)m[i] * a.ld_out + n, left, v[i]);
            }
          } else {
            // (rows of sums have room for whole quads)
            const uint32_t quads = (left + 3) / 4 * 4;
            if (a.addend && r.split == 0) {
#pragma unroll
              for (int i = 0; i < R; ++i) {
                if (m[i] == ~0u) continue;
                float old[W];
                load_row(a.addend + (size_t)m[i] * a.ld_sums + n, quads, old);
#pragma unroll
                for (int e = 0; e < W; ++e) v[i][e] += old[e];
              }
            }
            if constexpr (EPI == kEpiOut) finish<T>(a, m, n, bias, v);
            else {
#pragma unroll
              for (int i = 0; i < R; ++i)
                if (m[i] != ~0u) store_row(a.sums + ((size_t)r.split * a.M + m[i]) * a.ld_sums + n, quads, v[i]);
            }
          }
        }
      }
    } else if constexpr (EPI == kEpiStats) {
      float* part = reinterpret_cast<float*>(lds);                 // [2][WN * 4][BM]
      if constexpr (PH == 2) {
        // each lane's largest score of a row and the exponentials relative to it; the class's own score has one owner
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const uint32_t m = r.m0 + m_lane + i * 16;
          const uint32_t t = m < r.M ? a.target[m] : 0xffffffffu;
          float top = -INFINITY, sum = 0.0f;
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (r.n0 + n_wave0 + B::row_of(j, lane / 16 * 4 + e) < a.N) top = fmaxf(top, r.acc[i][j][e]);
          // (scores of -infinity only: relative to 0, so that they add nothing, where the difference of two infinities is no number)
          const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t n = r.n0 + n_wave0 + B::row_of(j, lane / 16 * 4 + e);
              if (n < a.N) sum += exp_of(r.acc[i][j][e] - from);
              if (n == t) a.target_score[m] = r.acc[i][j][e];
            }
          const uint32_t at = (wave % WN * 4 + lane / 16) * BM + m_lane + i * 16;
          part[at] = top;
          part[WN * 4 * BM + at] = sum;
        }
      } else if (tid < BM && r.m0 + tid < r.M) {
        float top = -INFINITY, sum = 0.0f;
        for (int w = 0; w < WN * 4; ++w) top = fmaxf(top, part[w * BM + tid]);
        for (int w = 0; w < WN * 4; ++w) {
          const float s = part[(WN * 4 + w) * BM + tid];
          if (s != 0.0f) sum += s * exp_of(part[w * BM + tid] - top);
        }
        float* to = a.stats + (size_t)(r.n0 / BN) * 2 * a.ld_stats + r.m0 + tid;
        to[0] = top;
        to[a.ld_stats] = sum;
      }
    }
  }
};

// Joins the parts of k: four outputs of a row for SIDE threads, which share the parts.  (50 x 125 outputs of 63 parts: 9.1 us with one
// thread each, in 7 workgroups; few outputs need the parts side by side: 4.1.)
template <class T, int SIDE>
struct GemmJoin {
  static constexpr int kThreads = 256, kQuads = kThreads / SIDE;
  static constexpr int kPhases = 2;
  static constexpr size_t kLdsBytes = SIDE > 1 ? kThreads * 16 : 0;
  struct Regs { float v[1][4]; };
  static size_t grid(const GemmArgs& a) { return ((size_t)a.M * ((a.N + 3) / 4) + kQuads - 1) / kQuads; }
  template <int PH>
  HCNN_HD static void phase(const GemmArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs& r) {
    float* lds = reinterpret_cast<float*>(lds_words);              // [4][SIDE][kQuads]
    const uint32_t quads = (a.N + 3) / 4, side = (uint32_t)tid / kQuads;
    const size_t at = (size_t)bid * kQuads + tid % kQuads;
    const size_t m = at / quads;
    const uint32_t n = (uint32_t)(at - m * quads) * 4;
    const uint32_t M = a.count_of == kCountM && *a.count < a.M ? *a.count : a.M;
    if constexpr (PH == 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) r.v[0][e] = 0.0f;
      if (m < M) {
#pragma unroll 4
        for (uint32_t s = side; s < a.splits; s += SIDE) {
          float x[4];
          load_row(a.sums + ((size_t)s * a.M + m) * a.ld_sums + n, x);
#pragma unroll
          for (int e = 0; e < 4; ++e) r.v[0][e] += x[e];
        }
      }
      if (SIDE > 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[e * kThreads + tid] = r.v[0][e];
    } else if (m < M && side == 0) {
      if (SIDE > 1)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int l = 1; l < SIDE; ++l) r.v[0][e] += lds[e * kThreads + l * kQuads + tid];
      float bias[4] = {};
      if (a.bias) load_row(static_cast<const T*>(a.bias) + n, a.N - n, bias);
      const uint32_t at_m[1] = {(uint32_t)m};
      finish<T>(a, at_m, n, bias, r.v);
    }
  }
};

// A matrix of 16-bit numbers with rows that start on 16 bytes and end in zeros: eight numbers per thread.
struct PackArgs {
  const void* from;
  size_t ld_from;
  void* to;
  size_t ld_to;               // a multiple of 8
  uint32_t rows, cols;
  size_t pieces;              // rows * ld_to / 8
  size_t threads;             // of the launch
};
struct PackRows {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const PackArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    typedef GemmOperand<Half, kAlongK, 16, 64> Op;
    const size_t each = a.ld_to / 8;
    for (size_t at = (size_t)bid * kThreads + tid; at < a.pieces; at += a.threads) {
      const size_t row = at / each;
      const uint32_t c = (uint32_t)(at - row * each) * 8;
      const uint32_t left = c < a.cols ? a.cols - c : 0;
      U4 v{};
      if (left) v = Op::first(Op::piece(static_cast<const Half*>(a.from), row * a.ld_from + c, (a.rows - 1) * a.ld_from + a.cols), left);
      *reinterpret_cast<U4*>(static_cast<Half*>(a.to) + row * a.ld_to + c) = v;
    }
  }
};

// ---------------------------------------------------------------- gradient of the activation and of the bias
// dz = dy * act'(z) (written where z and a place for it are there: rounded to T, the operand type of the two products that take it) and, per block of
// rows, the columns' sums of it in 32 bits.  A workgroup takes `rows_each` rows and kCols columns: lanes along the row, four numbers each.
// binary16 does not hold the products of two of its numbers: 300 x 200 x 2 is infinite there, 1e-4 x 1e-4 nothing.  Where the slope is any
// number (kRoom), dz is held once for each product, times a power of two for each row of dx or of dw (room_of the largest finite number of that row
// or column of dz), which goes back out of the product's sums; ActTops finds the largest ones before.  What it costs, us of the whole call with silu,
// bfloat16 / binary16: 8192 x 4096 -> 4096 485 / 580, 1024 x 1024 -> 1024 41.5 / 63, 16384 x 125 -> 50 29 / 43.
enum { kNoRoom = 0, kRoom = 1 };
struct ActGradArgs {
  const void *dy, *z;
  void* dz;
  void* dz_cols;              // kRoom: dz times the columns' powers of two (dz: the rows'); either may be null
  uint32_t *row_top, *col_top;   // kRoom: bits of the largest magnitudes, 0 before ActTops; either may be null
  float* part;                // [row blocks][ld_part], null: no sums
  size_t ld_dy, ld_z, ld_dz, ld_part;
  uint32_t M, N, rows_each, col_blocks;
  int act;
};
template <class T, int LANES, int ROOM>
struct ActGrad {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 2;
  static constexpr uint32_t kCols = LANES * 4, kLines = kThreads / LANES;
  static constexpr size_t kLdsBytes = kThreads * 16;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const ActGradArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    float* lds = reinterpret_cast<float*>(lds_words);              // [kLines][kCols]
    const uint32_t cb = bid % a.col_blocks, rb = bid / a.col_blocks;
    const uint32_t lane = (uint32_t)tid % LANES, line = (uint32_t)tid / LANES;
    const uint32_t n = cb * kCols + lane * 4;
    if constexpr (PH == 0) {
      const uint32_t m0 = rb * a.rows_each, m1 = a.M - m0 < a.rows_each ? a.M : m0 + a.rows_each;
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (n < a.N) {
        const uint32_t left = a.N - n;
        float room[4] = {};
        if constexpr (ROOM == kRoom)
          if (a.dz_cols)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) room[e] = e < left ? room_of(a.col_top[n + e]) : 0.0f;
#pragma unroll 4
        for (uint32_t m = m0 + line; m < m1; m += kLines) {
          float v[4];
          load_row(static_cast<const T*>(a.dy) + m * a.ld_dy + n, left, v);
          if (a.z) {
            float z[4];
            load_row(static_cast<const T*>(a.z) + m * a.ld_z + n, left, z);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= slope_of(z[e], a.act);
            if constexpr (ROOM == kRoom) {
              float t[4];
              if (a.dz) {
                const float of_row = room_of(a.row_top[m]);
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = v[e] * of_row;
                store_row(static_cast<T*>(a.dz) + m * a.ld_dz + n, left, t);
              }
              if (a.dz_cols) {
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = v[e] * room[e];
                store_row(static_cast<T*>(a.dz_cols) + m * a.ld_dz + n, left, t);
              }
            } else if (a.dz) {
              store_row(static_cast<T*>(a.dz) + m * a.ld_dz + n, left, v);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += v[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) lds[line * kCols + lane * 4 + e] = sum[e];
    } else if (a.part) {
      for (uint32_t c = tid; c < kCols; c += kThreads) {
        float s = 0.0f;
        for (uint32_t l = 0; l < kLines; ++l) s += lds[l * kCols + c];
        if (cb * kCols + c < a.N) a.part[(size_t)rb * a.ld_part + cb * kCols + c] = s;
      }
    }
  }
};
// Largest finite magnitudes of dz in each row and column, in ActGrad's shape.  A largest number does not depend on the order of the atomics.
template <class T, int LANES>
struct ActTops {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 2;
  static constexpr uint32_t kCols = LANES * 4, kLines = kThreads / LANES;
  static constexpr size_t kLdsBytes = kThreads * 16;
  struct Regs {};
  HCNN_HD static uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
  // The largest of a line's lanes for four rows, kLines apart: two exchanges leave a lane with one row's largest of four lanes, the others
  // make it that of the line, and four lanes hand it over (7 exchanges of 64 lanes, 24 for each row by itself).
  HCNN_HD static void row_tops(uint32_t* to, uint32_t rows, uint32_t lane, const uint32_t (&v)[4]) {   // to: the first row's; rows: that exist of it and those behind it
#if defined(__HIP_DEVICE_COMPILE__)
    const bool odd = lane & 1, high = lane & 2;
    const uint32_t a0 = larger(odd ? v[2] : v[0], (uint32_t)__shfl_xor((int)(odd ? v[0] : v[2]), 1));
    const uint32_t a1 = larger(odd ? v[3] : v[1], (uint32_t)__shfl_xor((int)(odd ? v[1] : v[3]), 1));
    uint32_t b = larger(high ? a1 : a0, (uint32_t)__shfl_xor((int)(high ? a0 : a1), 2));
#pragma unroll
    for (int d = 4; d < LANES; d *= 2) b = larger(b, (uint32_t)__shfl_xor((int)b, d));
    const uint32_t at = (odd ? 2 : 0) + (high ? 1 : 0);
    if (lane < 4 && at * kLines < rows) atomic_max32(to + at * kLines, b);
#else
    for (uint32_t i = 0; i < 4; ++i)
      if (i * kLines < rows) atomic_max32(to + i * kLines, v[i]);
#endif
  }
  template <int PH>
  HCNN_HD static void phase(const ActGradArgs& a, unsigned bid, int tid, uint32_t* lds, Regs&) {
    const uint32_t cb = bid % a.col_blocks, rb = bid / a.col_blocks;
    const uint32_t lane = (uint32_t)tid % LANES, line = (uint32_t)tid / LANES;
    const uint32_t n = cb * kCols + lane * 4;
    if constexpr (PH == 0) {
      const uint32_t m0 = rb * a.rows_each, m1 = a.M - m0 < a.rows_each ? a.M : m0 + a.rows_each;
      uint32_t top[4] = {};
      // four rows at a time; what lies beyond the rows or columns is another look at the last of them
      const uint32_t at = n < a.N ? n : (a.N - 1) / 4 * 4;
      for (uint32_t mi = m0 + line; mi < m1; mi += 4 * kLines) {
        float v[4][4], z[4][4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
          const uint32_t m = mi + i * kLines < m1 ? mi + i * kLines : m1 - 1;
          load_row(static_cast<const T*>(a.dy) + m * a.ld_dy + at, a.N - at, v[i]);
          load_row(static_cast<const T*>(a.z) + m * a.ld_z + at, a.N - at, z[i]);
        }
        uint32_t of_row[4] = {};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            uint32_t b = float_bits(v[i][e] * slope_of(z[i][e], a.act)) & 0x7fffffffu;
            if (b >= 0x7f800000u) b = 0;
            top[e] = larger(top[e], b);
            of_row[i] = larger(of_row[i], b);
          }
        if (a.row_top) row_tops(a.row_top + mi, m1 - mi, lane, of_row);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) lds[line * kCols + lane * 4 + e] = top[e];
    } else if (a.col_top) {
      for (uint32_t c = tid; c < kCols; c += kThreads) {
        uint32_t t = 0;
        for (uint32_t l = 0; l < kLines; ++l) t = larger(t, lds[l * kCols + c]);
        if (cb * kCols + c < a.N) atomic_max32(a.col_top + cb * kCols + c, t);
      }
    }
  }
};
struct ZeroWordsArgs { uint32_t* to; size_t count; };
struct ZeroWords {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const ZeroWordsArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    const size_t at = (size_t)bid * kThreads + tid;
    if (at < a.count) a.to[at] = 0;
  }
};
struct ColumnSumArgs {
  const float* part;          // [blocks][ld_part]
  size_t ld_part;
  uint32_t blocks, N;
  void* out;
};
// Sums of the blocks' sums: a workgroup takes 16 columns, 16 threads each.
template <class T>
struct ColumnSum {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 2;
  static constexpr size_t kLdsBytes = kThreads * 4;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const ColumnSumArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    float* lds = reinterpret_cast<float*>(lds_words);
    const uint32_t n = bid * 16 + tid % 16;
    if constexpr (PH == 0) {
      float s = 0.0f;
      if (n < a.N)
        for (uint32_t b = tid / 16; b < a.blocks; b += 16) s += a.part[b * a.ld_part + n];
      lds[tid] = s;
    } else if (tid < 16 && n < a.N) {
      float s = 0.0f;
      for (int l = 0; l < 16; ++l) s += lds[l * 16 + tid];
      static_cast<T*>(a.out)[n] = Num<T>::narrow(s);
    }
  }
};

// ---------------------------------------------------------------- rows whose target is a class
struct KeepRowsArgs {
  const void* targets;        // int32 or int64
  int wide;
  int64_t ignore;
  uint32_t M, classes;
  uint32_t* rows;             // [M] rows that take part, in order
  uint32_t* target;           // [M] their classes
  uint32_t* count;            // rows that take part
  unsigned long long* bad;    // targets that are neither a class nor the ignored value
  float* loss;                // 0 here: the mean of no rows (may be null)
  float* alpha;               // scale / count
  float scale;
};
// One workgroup, 8192 rows at a time: thread t takes rows t, 1024 + t, ..., so that what it reads and writes lies side by side with the
// other lanes' (a run of rows per thread: 14.6 us for 8192 rows, this 11.8).  A row's place is the number of rows before it that
// take part: of those in its 64, by their bits in LDS, and of the 64s before.
struct KeepRows {
  static constexpr int kThreads = 1024, kEach = 8, kWaves = kThreads / 64;
  static constexpr int kLoopPhases = 4, kPhases = 5;
  static constexpr size_t kLdsBytes = kEach * kWaves * 12;
  struct Regs {
    uint32_t iter;
    uint32_t before;          // rows of earlier iterations that take part
    uint32_t target[kEach];   // ~0: takes no part
  };
  HCNN_HD static uint32_t loop_count(const KeepRowsArgs& a) { return (a.M + kThreads * kEach - 1) / (kThreads * kEach); }
  HCNN_HD static int64_t target(const KeepRowsArgs& a, uint32_t m) {
    return a.wide ? static_cast<const int64_t*>(a.targets)[m] : static_cast<const int32_t*>(a.targets)[m];
  }
  HCNN_HD static bool kept(const KeepRowsArgs& a, int64_t t) { return t != a.ignore && t >= 0 && t < (int64_t)a.classes; }
  HCNN_HD static uint32_t ones(uint32_t x) { return (uint32_t)__builtin_popcount(x); }
  HCNN_HD static void begin(const KeepRowsArgs&, unsigned, int, uint32_t*, Regs& r) { r.before = 0; }
  template <int PH>
  HCNN_HD static void phase(const KeepRowsArgs& a, unsigned, int tid, uint32_t* lds, Regs& r) {
    uint32_t* counts = lds + kEach * kWaves * 2;                   // [kEach][kWaves], behind the bits [kEach][kWaves][2]
    const uint32_t m0 = r.iter * (kThreads * kEach) + tid, wave = (uint32_t)tid / 64, lane = (uint32_t)tid % 64;
    if constexpr (PH == 0) {
      if (tid < kEach * kWaves * 2) lds[tid] = 0;
    } else if constexpr (PH == 1) {
      int64_t t[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const uint32_t m = m0 + i * kThreads;
        t[i] = target(a, m < a.M ? m : a.M - 1);
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const bool is = m0 + i * kThreads < a.M, keep = is && kept(a, t[i]);
        r.target[i] = keep ? (uint32_t)t[i] : ~0u;
        if (keep) lds_or(lds + (i * kWaves + wave) * 2 + lane / 32, 1u << lane % 32);
        else if (is && t[i] != a.ignore) atomic_inc64(a.bad);
      }
    } else if constexpr (PH == 2) {
      if (tid < kEach * kWaves) counts[tid] = ones(lds[tid * 2]) + ones(lds[tid * 2 + 1]);
    } else if constexpr (PH == 3) {
      uint32_t at = r.before, start[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          if (w == (int)wave) start[i] = at;
          at += counts[i * kWaves + w];
        }
      }
      r.before = at;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (r.target[i] == ~0u) continue;
        const uint32_t *bits = lds + (i * kWaves + wave) * 2, below = (1u << lane % 32) - 1;
        const uint32_t to = start[i] + (lane < 32 ? ones(bits[0] & below) : ones(bits[0]) + ones(bits[1] & below));
        a.rows[to] = m0 + i * kThreads;
        a.target[to] = r.target[i];
      }
    } else if (tid == 0) {
      *a.count = r.before;
      if (a.loss) *a.loss = 0.0f;
      *a.alpha = (float)((double)a.scale / (r.before ? r.before : 1));
    }
  }
};

// ---------------------------------------------------------------- softmax statistics of whole rows
struct RowStatsArgs {
  const float* stats;         // [tiles][2][ld_stats]
  size_t ld_stats;
  uint32_t tiles, M;
  const uint32_t* count;
  const uint32_t* rows;
  const float* target_score;
  float* lse;                 // [rows that take part]
  double* part;               // [workgroups] sums of the losses
  float *row_loss, *row_lse;  // [M] or null
};
// Loss of a row from its largest score, the sum of exponentials relative to it, and the class's score; what the row has to leave behind.
HCNN_HD float row_loss(const RowStatsArgs& a, uint32_t m, float top, float sum, float score, float* lse_out) {
  const float log_sum = logf(sum), lse = top + log_sum;
  const float l = (top - score) + log_sum;                      // (the difference of the two large numbers first)
  if (a.row_loss) a.row_loss[a.rows[m]] = l;
  if (a.row_lse) a.row_lse[a.rows[m]] = lse;
  *lse_out = lse;
  return l;
}
// 64 rows per workgroup, four threads each.  A part without a sum adds nothing: its scores are all -infinity, or there are none.
struct RowStats {
  static constexpr int kThreads = 256;
  static constexpr uint32_t kRows = 64;
  static constexpr int kPhases = 3;
  static constexpr size_t kLdsBytes = (2 * kThreads + 2 * kRows) * 4;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const RowStatsArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    float* lds = reinterpret_cast<float*>(lds_words);
    double* losses = reinterpret_cast<double*>(lds + 2 * kThreads);
    const uint32_t m = bid * kRows + tid % kRows, M = *a.count;
    if constexpr (PH == 0) {
      float top = -INFINITY, sum = 0.0f;
      if (m < M)
#pragma unroll 4
        for (uint32_t t = tid / kRows; t < a.tiles; t += 4) {
          const float* s = a.stats + (size_t)t * 2 * a.ld_stats + m;
          const float x = s[0], y = s[a.ld_stats], high = fmaxf(top, x);
          sum = (sum != 0.0f ? sum * exp_of(top - high) : 0.0f) + (y != 0.0f ? y * exp_of(x - high) : 0.0f);
          top = high;
        }
      lds[tid] = top;
      lds[kThreads + tid] = sum;
    } else if constexpr (PH == 1) {
      if (tid < (int)kRows) {
        double loss = 0.0;
        if (m < M) {
          float top = -INFINITY, sum = 0.0f;
          for (int i = 0; i < 4; ++i) top = fmaxf(top, lds[i * kRows + tid]);
          for (int i = 0; i < 4; ++i) {
            const float s = lds[kThreads + i * kRows + tid];
            if (s != 0.0f) sum += s * exp_of(lds[i * kRows + tid] - top);
          }
          loss = row_loss(a, m, top, sum, a.target_score[m], a.lse + m);
        }
        losses[tid] = loss;
      }
    } else if (tid == 0) {
      double s = 0.0;
#pragma unroll 8
      for (uint32_t i = 0; i < kRows; ++i) s += losses[i];
      a.part[bid] = s;
    }
  }
};
struct MeanLossArgs {
  const double* part;
  uint32_t parts;
  const uint32_t* count;
  float* loss;                // mean over the rows that take part, 0 where there are none
};
// (by a workgroup of its own: when the last one of the kernel before took it along, each one's fence at the device cost more)
struct MeanLoss {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 3;
  static constexpr size_t kLdsBytes = kThreads * 8;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const MeanLossArgs& a, unsigned, int tid, uint32_t* lds_words, Regs&) {
    double* lds = reinterpret_cast<double*>(lds_words);
    if constexpr (PH == 0) {
      double s = 0.0;
      for (uint32_t i = tid; i < a.parts; i += kThreads) s += a.part[i];
      lds[tid] = s;
    } else if constexpr (PH == 1) {
      if (tid < 16) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += lds[tid * 16 + i];
        lds[tid * 16] = s;
      }
    } else if (tid == 0) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 16; ++i) s += lds[i * 16];
      *a.loss = (float)(s / (*a.count ? *a.count : 1));
    }
  }
};
// out = a b^T with at most 16 rows of a or (NARROW) of b, both along k: bound by reading the other operand, once.  It is loaded straight to
// the registers that the products read (lane: row lane % 16, 16 bytes lane / 16 of a 64-byte step of k); no wave waits for another.
//   SHARE 8  a workgroup takes 16 of its rows, eight waves every eighth step of k each, kDeep steps asked for at a time; sums join in LDS
//   SHARE 1  a wave takes 4 x 16 rows and all of k (short rows: at most 1 KiB)
// GPU us: one row of 4096 x 4096 bfloat16 weights in tiles of 16 x 128, 16 parts of k and their join 5.4 + 4.5, this 8.1; 147456 rows of
// 25 numbers by 5 filters in tiles of 128 x 16 10.2, this 8.5.
// LOSS (NARROW): the scores of at most 16 classes end in the rows' losses and the gradients for the scores.
struct StripLossArgs { GemmArgs g; RowStatsArgs rows; };
template <bool LOSS> struct StripArgs { typedef GemmArgs type; };
template <> struct StripArgs<true> { typedef StripLossArgs type; };
template <class T, bool NARROW, int SHARE, bool LOSS>
struct Strip {
  typedef typename StripArgs<LOSS>::type Args;
  static constexpr int kWaves = SHARE == 8 ? 8 : 4, kThreads = kWaves * 64;
  static constexpr int R = SHARE == 8 ? 1 : 4, kDeep = SHARE == 8 ? 8 : 2;
  static constexpr uint32_t kRows = SHARE == 8 ? 16 : kWaves * R * 16;         // of the streamed operand in a workgroup
  static constexpr int kPhases = LOSS ? 3 : SHARE == 8 ? 2 : 1;
  static constexpr uint32_t kStep = GemmNum<T>::kStage / 2, kPer16 = GemmNum<T>::kPer16;
  static constexpr size_t kLdsBytes = (SHARE == 8 ? kWaves * 256 : LOSS ? kWaves * R * 256 : 0) * 4 + (LOSS ? kThreads * 8 : 0);
  typedef GemmOperand<T, kAlongK, 16, 64> Op;
  struct Regs {};
  HCNN_HD static const GemmArgs& gemm(const GemmArgs& a) { return a; }
  HCNN_HD static const GemmArgs& gemm(const StripLossArgs& a) { return a.g; }
  // 16 bytes at k of row x (the last one where there is none)
  HCNN_HD static U4 piece(const T* p, size_t ld, size_t extent, uint32_t X, uint32_t K, uint32_t x, uint32_t k) {
    const U4 v = Op::piece(p, (x < X ? x : X - 1) * ld + (k < K ? k : K - 1), extent);
    return Op::first(v, k < K ? K - k : 0);
  }
  template <int PH>
  HCNN_HD static void phase(const Args& args, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    const GemmArgs& a = gemm(args);
    float* lds = reinterpret_cast<float*>(lds_words);              // [wave][R][m][n]
    const uint32_t wave = (uint32_t)tid / 64, lane = (uint32_t)tid % 64, i = lane % 16, g = lane / 16;
    const uint32_t x0 = bid * kRows;                                // first streamed row
    uint32_t M = a.M;
    if constexpr (LOSS) M = wave_uniform(*a.count) < M ? wave_uniform(*a.count) : M;
    if constexpr (PH == 0) {
      const bool kept = LOSS && a.kept && (a.kept_always || M < a.M);
      const T *pa = static_cast<const T*>(kept ? a.kept : a.a), *pb = static_cast<const T*>(a.b);
      const size_t lda = kept ? a.ld_kept : a.lda, a_extent = kept ? a.M * a.ld_kept : a.a_extent;
      const T *ps = NARROW ? pa : pb, *po = NARROW ? pb : pa;
      const size_t lds_ = NARROW ? lda : a.ldb, ldo = NARROW ? a.ldb : lda;
      const size_t es = NARROW ? a_extent : a.b_extent, eo = NARROW ? a.b_extent : a_extent;
      const uint32_t XS = NARROW ? M : a.N, XO = NARROW ? a.N : M;
      if (x0 < XS) {
        const uint32_t row = x0 + (SHARE == 8 ? 0 : wave * (R * 16)) + i;
        hcnn_float4 acc[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[r][e] = 0.0f;
#if defined(__HIP_DEVICE_COMPILE__)
        const uint32_t mine = SHARE == 8 ? wave_uniform(wave) : 0, whole = a.K / kStep;        // the wave's first step; steps that are whole
        const T* at[R];
#pragma unroll
        for (int r = 0; r < R; ++r) at[r] = ps + (row + r * 16 < XS ? row + r * 16 : XS - 1) * lds_ + g * kPer16;
        const T* other = po + (i < XO ? i : XO - 1) * ldo + g * kPer16;
        auto add = [&](const U4 (&fs)[R], const U4& fo) {
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const hcnn_word4 s4{fs[r].x, fs[r].y, fs[r].z, fs[r].w}, o4{fo.x, fo.y, fo.z, fo.w};
            mma<T>(acc[r], NARROW ? o4 : s4, NARROW ? s4 : o4);
          }
        };
        // the step that is not whole, asked for before the others are waited for
        const bool rest = whole * kStep < a.K && whole % SHARE == mine;
        U4 rs[R], ro{};
        if (rest) {
          const uint32_t k = whole * kStep + g * kPer16;
#pragma unroll
          for (int r = 0; r < R; ++r) rs[r] = piece(ps, lds_, es, XS, a.K, row + r * 16, k);
          ro = piece(po, ldo, eo, XO, a.K, i, k);
        }
        for (uint32_t s = mine; s < whole; s += SHARE * kDeep) {
          U4 fs[kDeep][R], fo[kDeep];
#pragma unroll
          for (int d = 0; d < kDeep; ++d) {
            const uint32_t step = s + d * SHARE;
            if (step < whole) {
#pragma unroll
              for (int r = 0; r < R; ++r) fs[d][r] = ld16(reinterpret_cast<const char*>(at[r] + step * kStep));
              fo[d] = ld16(reinterpret_cast<const char*>(other + step * kStep));
            } else {
#pragma unroll
              for (int r = 0; r < R; ++r) fs[d][r] = U4{};
              fo[d] = U4{};
            }
          }
#pragma unroll
          for (int d = 0; d < kDeep; ++d) add(fs[d], fo[d]);
        }
        if (rest) add(rs, ro);
#else
        for (int r = 0; r < R; ++r)
          for (uint32_t k0 = SHARE == 8 ? wave * kStep : 0; k0 < a.K; k0 += SHARE * kStep)
            for (uint32_t p = 0; p < 4; ++p)
              for (uint32_t e = 0; e < 4; ++e) {
                // (the lane's m: row i of a, its n: rows 4 g + e of b)
                const uint32_t ra = (NARROW ? row + r * 16 : i), rb = NARROW ? g * 4 + e : x0 + g * 4 + e, k = k0 + p * kPer16;
                T x[kPer16], y[kPer16];
                const U4 fa = piece(pa, lda, a_extent, M, a.K, ra, k), fb = piece(pb, a.ldb, a.b_extent, a.N, a.K, rb, k);
                __builtin_memcpy(x, &fa, 16);
                __builtin_memcpy(y, &fb, 16);
                for (uint32_t l = 0; l < kPer16; ++l) acc[r][e] += Num<T>::widen(x[l]) * Num<T>::widen(y[l]);
              }
        (void)ps; (void)po; (void)lds_; (void)ldo; (void)es; (void)eo; (void)XO;
#endif
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float v[1][4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[0][e] = acc[r][e];
          if constexpr (SHARE == 8 || LOSS) {
            __builtin_memcpy(lds + ((wave * R + r) * 16 + i) * 16 + g * 4, v, 16);
          } else {
            const uint32_t m[1] = {row + r * 16}, n = g * 4;
            if (m[0] < M && n < a.N) end(a, m, n, v);
          }
        }
      }
    } else if constexpr (!LOSS) {
      if (tid < 64) {
        const uint32_t m[1] = {(NARROW ? x0 : 0) + (uint32_t)tid / 4}, n = (NARROW ? 0 : x0) + tid % 4 * 4;
        if (m[0] >= M || n >= a.N) return;
        float v[1][4] = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[0][e] += lds[w * 256 + tid * 4 + e];
        end(a, m, n, v);
      }
    } else {
      double* losses = reinterpret_cast<double*>(lds + (SHARE == 8 ? kWaves : kWaves * R) * 256);
      const RowStatsArgs& rows = args.rows;
      const uint32_t m = x0 + tid;
      if constexpr (PH == 1) {
        double loss = 0.0;
        if (tid < (int)kRows && m < M) {
          float v[16], top = -INFINITY, sum = 0.0f, score = 0.0f;
          const uint32_t t = a.target[m];
#pragma unroll
          for (uint32_t n = 0; n < 16; ++n) {
            v[n] = 0.0f;
#pragma unroll
            for (int w = 0; w < SHARE; ++w) v[n] += lds[(SHARE == 8 ? w * 256 : 0) + tid * 16 + n];
            if (n < a.N) top = fmaxf(top, v[n]);
            if (n == t) score = v[n];
          }
#pragma unroll
          for (uint32_t n = 0; n < 16; ++n) {
            v[n] = exp_of(v[n] - top);
            if (n < a.N) sum += v[n];
          }
          float lse;
          loss = row_loss(rows, m, top, sum, score, &lse);
          if (a.out) {
            const float part = 1.0f / sum;
            T* to = static_cast<T*>(a.out) + (size_t)m * a.ld_out;
#pragma unroll
            for (uint32_t n = 0; n < 16; ++n)
              if (n < a.N) to[n] = Num<T>::narrow((v[n] * part - (n == t ? 1.0f : 0.0f)) * a.delta_scale);
          }
        }
        losses[tid] = loss;
      } else if (tid == 0) {
        double s = 0.0;
#pragma unroll 8
        for (uint32_t l = 0; l < (kRows < (uint32_t)kThreads ? kRows : kThreads); ++l) s += losses[l];
        rows.part[bid] = s;
      }
    }
  }
  HCNN_HD static void end(const GemmArgs& a, const uint32_t (&m)[1], uint32_t n, float (&v)[1][4]) {
    float bias[4] = {};
    if (a.bias) load_row(static_cast<const T*>(a.bias) + n, a.N - n, bias);
    finish<T>(a, m, n, bias, v);
  }
};

// Rows that do not take part: zeros in the gradient, and in the losses and statistics asked for.  Rows that do: a copy of theirs in x one
// behind the other, where they are not all rows or the copy is wanted in any case.  64 threads per row.
struct SortRowsArgs {
  KeepRowsArgs keep;
  void* dx;                   // null: none
  size_t ld_dx;               // bytes
  size_t row_bytes;
  float *row_loss, *row_lse;
  const void* x;
  size_t ld_x;                // bytes
  void* kept;
  size_t ld_kept;             // bytes, a multiple of 16
  uint32_t always;
  uint32_t rows;              // that the launch takes at a time
};
struct SortRows {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const SortRowsArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    const uint32_t n = *a.keep.count;
    if (n == a.keep.M && !a.always) return;
    for (uint32_t m = bid * 4 + tid / 64; m < a.keep.M; m += a.rows) row(a, m, n, tid % 64);
  }
  HCNN_HD static void row(const SortRowsArgs& a, uint32_t m, uint32_t n, uint32_t lane) {
    const size_t whole = a.row_bytes / 16 * 16;
    if (!KeepRows::kept(a.keep, KeepRows::target(a.keep, m))) {
      if (lane == 0 && a.row_loss) a.row_loss[m] = 0.0f;
      if (lane == 0 && a.row_lse) a.row_lse[m] = 0.0f;
      if (a.dx) {
        char* row = static_cast<char*>(a.dx) + m * a.ld_dx;
        const U4 zero{};
        for (size_t b = (size_t)lane * 16; b < whole; b += 1024) st16(row + b, zero);
        for (size_t b = whole + (size_t)lane * 2; b < a.row_bytes; b += 128) *reinterpret_cast<uint16_t*>(row + b) = 0;
      }
    }
    if (m >= n) return;
    const char* from = static_cast<const char*>(a.x) + a.keep.rows[m] * a.ld_x;
    char* to = static_cast<char*>(a.kept) + m * a.ld_kept;
#pragma unroll 4
    for (size_t b = (size_t)lane * 16; b < whole; b += 1024) st16(to + b, ld16(from + b));
    for (size_t b = whole + (size_t)lane * 2; b < a.row_bytes; b += 128) *reinterpret_cast<uint16_t*>(to + b) = *reinterpret_cast<const uint16_t*>(from + b);
    for (size_t b = a.row_bytes + (size_t)lane * 2; b < a.ld_kept; b += 128) *reinterpret_cast<uint16_t*>(to + b) = 0;
  }
};

// ---------------------------------------------------------------- norm of many gradients
// A list of tensors travels in the launch's arguments; a workgroup takes runs of kRun numbers, `first` tells whose they are.
constexpr uint32_t kNormTensors = 96;
constexpr uint32_t kNormRun = 16384;
struct NormArgs {
  const void* in[kNormTensors];
  void* out[kNormTensors];
  uint64_t size[kNormTensors];
  uint32_t first[kNormTensors + 1];        // first run of each tensor; the last entry: number of runs
  uint8_t type[kNormTensors];              // 0: 32 bits, 1: binary16, 2: bfloat16
  uint32_t tensors;
  double* part;                            // sums of squares of the whole list, a number per workgroup
  uint32_t part_first;                     // of this launch
  const double* factor;
  double max_norm, eps;                    // ClipSmall
  float* norm;
};
struct NormRun { const char* in; char* out; uint32_t n; int type; };
HCNN_HD NormRun norm_run(const NormArgs& a, uint32_t run) {
  uint32_t lo = 0, hi = a.tensors;                                // first[lo] <= run < first[hi]
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.first[mid] <= run) lo = mid; else hi = mid;
  }
  NormRun r;
  r.type = a.type[lo];
  const uint64_t at = (uint64_t)(run - a.first[lo]) * kNormRun, left = a.size[lo] - at;
  const uint32_t bytes = r.type == 0 ? 4 : 2;
  r.in = static_cast<const char*>(a.in[lo]) + at * bytes;
  r.out = a.out[lo] ? static_cast<char*>(a.out[lo]) + at * bytes : nullptr;
  r.n = left < kNormRun ? (uint32_t)left : kNormRun;
  return r;
}
// Squares are summed in 64 bits: no square of a 32-bit number leaves their range, and the sum's order does not show in a 32-bit norm.
template <class T>
HCNN_HD double sum_squares(const T* p, uint32_t n, int tid, int threads) {
  constexpr uint32_t kPer16 = 16 / sizeof(T);
  double s = 0.0;
  const uint32_t whole = n / kPer16;
#pragma unroll 4
  for (uint32_t i = tid; i < whole; i += threads) {
    const U4 w = ld16(reinterpret_cast<const char*>(p + (size_t)i * kPer16));
    T t[kPer16];
    __builtin_memcpy(t, &w, 16);
#pragma unroll
    for (uint32_t e = 0; e < kPer16; ++e) { const double x = Num<T>::widen(t[e]); s += x * x; }
  }
  for (uint32_t i = whole * kPer16 + tid; i < n; i += threads) { const double x = Num<T>::widen(p[i]); s += x * x; }
  return s;
}
HCNN_HD double sum_any(const NormRun& r, int tid, int threads) {
  return r.type == 0 ? sum_squares(reinterpret_cast<const float*>(r.in), r.n, tid, threads)
       : r.type == 1 ? sum_squares(reinterpret_cast<const Half*>(r.in), r.n, tid, threads)
                     : sum_squares(reinterpret_cast<const Bfloat*>(r.in), r.n, tid, threads);
}
// The norm, and the factor that goes with it: a norm that is no number makes it none
HCNN_HD double norm_factor(double squares, double max_norm, double eps, float* norm_out) {
  const double norm = sqrt(squares), c = max_norm / (norm + eps);
  *norm_out = (float)norm;
  return c < 1.0 || c != c ? c : 1.0;
}
struct SumSquares {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 3;
  static constexpr size_t kLdsBytes = kThreads * 8;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const NormArgs& a, unsigned bid, int tid, uint32_t* lds_words, Regs&) {
    double* lds = reinterpret_cast<double*>(lds_words);
    if constexpr (PH == 0) {
      const NormRun r = norm_run(a, bid);
      lds[tid] = sum_any(r, tid, kThreads);
    } else if constexpr (PH == 1) {
      if (tid < 16) {
        double s = 0.0;
        for (int i = 0; i < 16; ++i) s += lds[tid * 16 + i];
        lds[tid * 16] = s;
      }
    } else if (tid == 0) {
      double s = 0.0;
      for (int i = 0; i < 16; ++i) s += lds[i * 16];
      a.part[a.part_first + bid] = s;
    }
  }
};
struct NormTotalArgs {
  const double* part;
  uint32_t parts;
  double max_norm, eps;
  float* norm;
  double* factor;
};
struct NormTotal {
  static constexpr int kThreads = 1024;
  static constexpr int kPhases = 3;
  static constexpr size_t kLdsBytes = kThreads * 8;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const NormTotalArgs& a, unsigned, int tid, uint32_t* lds_words, Regs&) {
    double* lds = reinterpret_cast<double*>(lds_words);
    if constexpr (PH == 0) {
      double s = 0.0;
      for (uint32_t i = tid; i < a.parts; i += kThreads) s += a.part[i];
      lds[tid] = s;
    } else if constexpr (PH == 1) {
      if (tid < 32) {
        double s = 0.0;
        for (int i = 0; i < 32; ++i) s += lds[tid * 32 + i];
        lds[tid * 32] = s;
      }
    } else if (tid == 0) {
      double s = 0.0;
      for (int i = 0; i < 32; ++i) s += lds[i * 32];
      *a.factor = norm_factor(s, a.max_norm, a.eps, a.norm);
    }
  }
};
template <class T, class C>
HCNN_HD void scale_run(const T* p, T* to, uint32_t n, C c, int tid, int threads) {
  constexpr uint32_t kPer16 = 16 / sizeof(T);
  const uint32_t whole = n / kPer16;
#pragma unroll 4
  for (uint32_t i = tid; i < whole; i += threads) {
    U4 w = ld16(reinterpret_cast<const char*>(p + (size_t)i * kPer16));
    T t[kPer16];
    __builtin_memcpy(t, &w, 16);
#pragma unroll
    for (uint32_t e = 0; e < kPer16; ++e) t[e] = Num<T>::narrow((float)(Num<T>::widen(t[e]) * c));
    __builtin_memcpy(&w, t, 16);
    st16(reinterpret_cast<char*>(to + (size_t)i * kPer16), w);
  }
  for (uint32_t i = whole * kPer16 + tid; i < n; i += threads) to[i] = Num<T>::narrow((float)(Num<T>::widen(p[i]) * c));
}
template <class C>
HCNN_HD void scale_by(const NormRun& r, C c, int tid, int threads) {
  if (r.type == 0) scale_run(reinterpret_cast<const float*>(r.in), reinterpret_cast<float*>(r.out), r.n, c, tid, threads);
  else if (r.type == 1) scale_run(reinterpret_cast<const Half*>(r.in), reinterpret_cast<Half*>(r.out), r.n, c, tid, threads);
  else scale_run(reinterpret_cast<const Bfloat*>(r.in), reinterpret_cast<Bfloat*>(r.out), r.n, c, tid, threads);
}
// (a factor near or below the smallest normal 32-bit number has few bits there, or none, where its products with large numbers have all)
HCNN_HD void scale_any(const NormRun& r, double c, int tid, int threads) {
  if (c < 7.888609052210118e-31) scale_by(r, c, tid, threads);      // 2^-100
  else scale_by(r, (float)c, tid, threads);
}
struct ScaleGrads {
  static constexpr int kThreads = 256;
  static constexpr int kPhases = 1;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const NormArgs& a, unsigned bid, int tid, uint32_t*, Regs&) {
    const double c = *a.factor;
    const NormRun r = norm_run(a, a.first[a.tensors] - 1 - bid);      // the last ones first: the sum has just read them
    if ((float)c == 1.0f && r.in == r.out) return;                         // nothing to scale, nowhere to copy
    scale_any(r, c, tid, kThreads);
  }
};
// The whole of it for a list of few numbers: one workgroup, one launch.
struct ClipSmall {
  static constexpr int kThreads = 1024;
  static constexpr int kPhases = 4;
  static constexpr size_t kLdsBytes = kThreads * 8 + 16;
  struct Regs {};
  template <int PH>
  HCNN_HD static void phase(const NormArgs& a, unsigned, int tid, uint32_t* lds_words, Regs&) {
    double* lds = reinterpret_cast<double*>(lds_words);
    double* factor = lds + kThreads;
    if constexpr (PH == 0) {
      double s = 0.0;
      for (uint32_t i = 0; i < a.first[a.tensors]; ++i) s += sum_any(norm_run(a, i), tid, kThreads);
      lds[tid] = s;
    } else if constexpr (PH == 1) {
      if (tid < 32) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += lds[tid * 32 + i];
        lds[tid * 32] = s;
      }
    } else if constexpr (PH == 2) {
      if (tid == 0) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += lds[i * 32];
        *factor = norm_factor(s, a.max_norm, a.eps, a.norm);
      }
    } else {
      for (uint32_t i = 0; i < a.first[a.tensors]; ++i) {
        const NormRun r = norm_run(a, i);
        if ((float)*factor != 1.0f || r.in != r.out) scale_any(r, *factor, tid, kThreads);
      }
    }
  }
};

}  // namespace hcnn
