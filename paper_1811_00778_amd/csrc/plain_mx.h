// Products of microscaled matrices: y = act(x w^T + bias) + residual, w of four-bit numbers, x of four or eight bits.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows by 16 rows over 128 numbers, four blocks of 32, and scales every block's sum by the two
// blocks' powers of two.  Lane l holds of its row l mod 16, with g = l / 16: of four-bit numbers the 16 bytes of block g, of eight-bit ones bytes 16 g .. 16 g + 15 of
// the first and of the last 64; and of its row the byte of block g in one of four bytes of a register.  w is the first operand: a lane's four sums are of w's rows
// 4 g .. 4 g + 3 and x's row l mod 16.  F products side by side take rows F i + j (i: row of the instruction, j: product), so that a lane's sums of
// all of them are 4 F columns side by side, and the scales of four products one 32-bit word.
//
// What the instruction sums: measured with single numbers, the products of eight consecutive four-by-eight-bit pairs are cut to multiples of 2^-13 of the power of two
// in the largest of them (four-bit pairs lie within that: exact), and the groups' sums join in 32 bits.  The cut is 2^-9 of the eight-bit rounding of the largest
// number itself: it stands for outputs of 16 bits.  Outputs of 32 bits take x in two halves (Split), numbers from 4 on and numbers below, whose products lie within 13 bits: exact, at half the rate.
#pragma once
#include "plain_rows.h"

namespace hcnn {

struct MxArgs {
  GemmArgs g;                  // M, N, the ending, the sums
  const uint8_t *x, *x_scales, *w, *w_scales;
  size_t x_bytes, w_bytes;     // of a row
  size_t x_pitch, w_pitch;     // bytes from a block's row scales to the next block's: multiples of 64, so that whole 64 rows can be read
  uint32_t steps;              // of 128 numbers
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
template <int F, bool SPLIT, int JW, int JX>
__device__ __forceinline__ void mx_mma(hcnn_float4& acc, const MxFrag<kMx4>& w, const MxFrag<F>& x, uint32_t sw, uint32_t sx) {
  const hcnn_int8 wv = w.words(), xv = x.words();
  if constexpr (F == kMx4) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc, 4, 4, JW, (int)sw, JX, (int)sx);
  } else if constexpr (!SPLIT) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc, 4, 0, JW, (int)sw, JX, (int)sx);
  } else {
    hcnn_int8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // bytes whose magnitude is 0x48 (4) or more: the carry into the sign's place
      const uint32_t b = (uint32_t)xv[i], up = ((b & 0x7f7f7f7fu) + 0x38383838u) & 0x80808080u, mask = (up >> 7) * 255u;
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

// The simple form: a workgroup computes 16 MF rows by 16 NF columns, its waves share the steps; operands come straight from memory to the registers that the
// products read, kDeep steps asked for at a time, and no wave waits for another before the sums join in LDS.
template <class T, int F, int MF, int NF>
struct MxStrip {
  static constexpr int kWaves = MF * NF == 16 ? 4 : 8, kThreads = kWaves * 64, kDeep = MF * NF == 16 ? 2 : 4;
  static constexpr uint32_t kRows = MF * 16, kCols = NF * 16;
  static constexpr int kPhases = 2;
  static constexpr size_t kLdsBytes = (size_t)kWaves * kRows * kCols * 4;
  static constexpr bool kSplit = F == kMx8 && sizeof(T) == 4;
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
              mx_mma<F, kSplit, n, m>(acc[m][n], w[d][n], x[d][m], bw[d], bx[d]);
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

}  // namespace hcnn
