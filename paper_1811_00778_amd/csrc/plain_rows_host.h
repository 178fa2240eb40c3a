// Host side of the operators along rows and of the microscaled products: choice of the kernels' shapes and their order.
#pragma once
#include "plain_host.h"
#include "plain_mx.h"

namespace plain_host {

inline Chunks chunks_of(size_t rows, size_t per_row, int threads, int each) {
  Chunks c;
  c.all = (uint64_t)rows * per_row;
  c.per_row = fast_div((uint32_t)per_row);
  c.groups = (uint32_t)std::min<uint64_t>((c.all + threads * each - 1) / (threads * each), most_workgroups(threads));
  return c;
}

template <class T>
int dropout(hcnn_plain* h, size_t rows, size_t n, const void* x, size_t ldx, const void* residual, size_t ld_residual, double p, uint64_t seed, uint32_t stream,
            void* y, size_t ldy) {
  typedef Dropout<T, false> Plain;
  const double threshold = std::nearbyint(p * 4294967296.0);
  DropoutArgs a{};
  a.chunks = chunks_of(rows, blocks(n, Plain::W), Plain::kThreads, Plain::EACH);
  a.x = x; a.ldx = ldx; a.residual = residual; a.ld_residual = ld_residual; a.y = y; a.ldy = ldy;
  a.n = (uint32_t)n;
  a.none = threshold >= 4294967296.0;
  a.threshold = a.none ? 0xffffffffu : (uint32_t)threshold;
  a.scale = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f;
  a.seed = seed; a.stream = stream;
  return residual ? launch<Dropout<T, true>>(h->stream, a.chunks.groups, 0, a) : launch<Plain>(h->stream, a.chunks.groups, 0, a);
}

// ---------------------------------------------------------------- norm
// Threads that share a row, and numbers that each of them holds (0: any length, read twice)
struct RowShape { int lanes, el; };
inline RowShape row_shape(size_t n) {
  for (int lanes : {8, 64, 256, 1024})
    for (int el : {8, 16})
      if (n <= (size_t)lanes * el) return RowShape{lanes, el};
  return RowShape{1024, 0};
}
#define PLAIN_ROW_SHAPE(s, CALL)                                     \
  do {                                                               \
    if (s.lanes == 8) return s.el == 8 ? CALL(8, 8) : CALL(8, 16);   \
    if (s.lanes == 64) return s.el == 8 ? CALL(64, 8) : CALL(64, 16); \
    if (s.lanes == 256) return s.el == 8 ? CALL(256, 8) : CALL(256, 16); \
    return s.el == 8 ? CALL(1024, 8) : s.el == 16 ? CALL(1024, 16) : CALL(1024, 0); \
  } while (0)

template <class K>
int norm_rows_launch(hcnn_plain* h, NormRowsArgs a) {
  const size_t most = most_workgroups(K::kThreads) * K::kLines;       // rows of a launch
  for (size_t row = 0; row < a.rows; row += most) {
    a.first = (uint32_t)row;
    const int e = launch<K>(h->stream, blocks(std::min(most, a.rows - row), K::kLines), K::kLdsBytes, a);
    if (e) return e;
  }
  return 0;
}
template <class T, int F>
int norm_rows(hcnn_plain* h, const NormRowsArgs& a) {
  const RowShape s = row_shape(F == kMxNone ? a.n : up(a.n, 128));
#define PLAIN_CALL(L, E) norm_rows_launch<NormRows<T, L, E, F>>(h, a)
  PLAIN_ROW_SHAPE(s, PLAIN_CALL);
#undef PLAIN_CALL
}
template <class T>
int rms_norm(hcnn_plain* h, size_t rows, size_t n, const void* x, size_t ldx, const void* residual, size_t ld_residual, const void* weight, double eps, void* hid,
             size_t ldh, void* y, size_t ldy, const MxOut& to) {
  NormRowsArgs a{};
  a.x = x; a.ldx = ldx; a.residual = residual; a.ld_residual = ld_residual; a.weight = weight;
  a.rows = (uint32_t)rows; a.n = (uint32_t)n; a.per = 1.0 / (double)n; a.eps = eps;
  a.h = hid; a.ldh = ldh; a.y = y; a.ldy = ldy; a.to = to;
  return to.codes ? norm_rows<T, kMx8>(h, a) : norm_rows<T, kMxNone>(h, a);
}

// Rows of a workgroup, and workgroups, of the norm's gradient: as many as the compute units hold at a time, by the kernels' registers
struct RowShare { uint32_t each; size_t groups; };
inline RowShare norm_share(const hcnn_plain* h, size_t rows, const RowShape& s, bool wide) {
  const size_t most = (size_t)h->compute_units * (s.lanes == 1024 ? 1 : s.el == 16 ? (wide ? 2 : 3) : wide ? 4 : 5);
  const size_t each = up(std::max<size_t>(blocks(rows, most), 1), s.lanes < 256 ? 256 / s.lanes : 1);
  return RowShare{(uint32_t)each, blocks(rows, each)};
}
template <class K>
int norm_grad_launch(hcnn_plain* h, const NormGradArgs& a, size_t groups) { return launch<K>(h->stream, groups, K::kLdsBytes, a); }
template <class T>
int norm_grad_rows(hcnn_plain* h, const NormGradArgs& a, const RowShape& s, size_t groups) {
#define PLAIN_CALL(L, E) norm_grad_launch<NormGrad<T, L, E>>(h, a, groups)
  PLAIN_ROW_SHAPE(s, PLAIN_CALL);
#undef PLAIN_CALL
}
template <class T>
int rms_norm_grad(hcnn_plain* h, size_t rows, size_t n, const void* dy, size_t ld_dy, const void* hid, size_t ldh, const void* weight, const void* dh, size_t ld_dh,
                  double eps, void* dx, size_t ld_dx, void* dw) {
  const RowShape s = row_shape(n);
  const RowShare share = norm_share(h, rows, s, sizeof(T) == 4);
  // rows of any length: their columns' sums in a pass of their own, about eight workgroups for each compute unit
  const size_t col_blocks = blocks(n, NormColumns<T>::kCols);
  const uint32_t col_rows = (uint32_t)std::max<size_t>(16, blocks(rows, std::max<size_t>(1, (size_t)h->compute_units * 8 / col_blocks)));
  const size_t parts = s.el ? share.groups : blocks(rows, col_rows);
  Arena ar;
  NormGradArgs a{};
  a.ld_part = up(n, 4);
  const size_t o_part = ar.take(dw ? parts * a.ld_part * 4 : 0), o_inverse = ar.take(dw && !s.el ? rows * 8 : 0);
  int e = reserve(h, ar.bytes);
  if (e) return e;
  a.dy = dy; a.ld_dy = ld_dy; a.h = hid; a.ldh = ldh; a.weight = weight; a.dh = dh; a.ld_dh = ld_dh;
  a.rows = (uint32_t)rows; a.n = (uint32_t)n; a.rows_each = share.each; a.per = 1.0 / (double)n; a.eps = eps;
  a.dx = dx; a.ld_dx = ld_dx;
  a.part = dw ? at<float>(h, o_part) : nullptr;
  a.inverse = dw && !s.el ? at<double>(h, o_inverse) : nullptr;
  if (rows) {
    if ((e = norm_grad_rows<T>(h, a, s, share.groups))) return e;
    if (dw && !s.el) {
      a.rows_each = col_rows;
      if ((e = launch<NormColumns<T>>(h->stream, col_blocks * parts, 0, a))) return e;
    }
  }
  if (dw) {
    // (a launch has fewer than 2^32 threads: 32 columns for each workgroup)
    const size_t most = most_workgroups(QuadSums<T>::kThreads) * 32;
    for (size_t c = 0; c < n; c += most) {
      const size_t some = std::min(most, n - c);
      const ColumnSumArgs cs{at<float>(h, o_part) + c, a.ld_part, (uint32_t)(rows ? parts : 0), (uint32_t)some, static_cast<char*>(dw) + c * sizeof(T)};
      if ((e = launch<QuadSums<T>>(h->stream, blocks(some, 32), QuadSums<T>::kLdsBytes, cs))) return e;
    }
  }
  return 0;
}

// ---------------------------------------------------------------- microscaled formats
inline size_t mx_row_bytes(int format, size_t n) { return up(n, 128) / 8 * (size_t)format; }
template <class T>
int quantize(hcnn_plain* h, int format, size_t rows, size_t n, const void* x, size_t ldx, const MxOut& to, void* values, size_t ld_values) {
  typedef Quantize<T, kMx4> Four;
  QuantizeArgs a{};
  a.tiles.all = (uint64_t)blocks(rows, Four::kRows) * blocks(n, 128);
  a.tiles.per_row = fast_div((uint32_t)blocks(n, 128));
  a.tiles.groups = (uint32_t)std::min<uint64_t>((a.tiles.all + Four::EACH - 1) / Four::EACH, most_workgroups(Four::kThreads));
  a.x = x; a.ldx = ldx; a.rows = (uint32_t)rows; a.n = (uint32_t)n; a.to = to; a.values = values; a.ld_values = ld_values;
  return format == kMx4 ? launch<Four>(h->stream, a.tiles.groups, 0, a) : launch<Quantize<T, kMx8>>(h->stream, a.tiles.groups, 0, a);
}

struct MxCall {
  int format, act;
  size_t M, K, N;
  const uint8_t *x, *x_scales; size_t x_pitch;
  const uint8_t *w, *w_scales; size_t w_pitch;
  const void *bias, *residual; size_t ld_residual;
  void* y; size_t ldy;
};
// Shape of the product, by an estimate of its time in us: `load` workgroups for each compute unit, a step's time with few workgroups and for each of several on a
// unit, what a workgroup's beginning and ending add, parts of k written and joined.  Strips (kMxStrip) of 16 MF x 16 NF outputs, tiles of 128 and 256.  Fitted to
// graphs of 20 calls, us estimated / measured with four and with eight bits (whose steps take two instructions a product, for results of 16 and of 32 bits alike):
// 1 x 4096 -> 4096 strips of 16 x 16 5 / 4.4, 5 / 5.0; 64 x 4096 -> 4096 of 64 x 16 8 / 8.3, 14 / 13.1; 256 x 4096 -> 4096 of 64 x 64 14 / 13.8, 23 / 22.9; 1024 x 4096 -> 4096
// tiles of 128 19 / 18.6, 40 / 43; 4096 x 4096 -> 4096 of 256 39 / 38.9, 90 / 91.  Of 37 sizes from 1 x 4096 -> 4096 to 8192 x 4096 -> 8192 with eight bits, in both types of results,
// the choice is the fastest shape or within 6 % of it, but for 128 x 4096 -> 4096 (17 %: eight parts where six are faster).
enum { kMxStrip11, kMxStrip14, kMxStrip41, kMxStrip44, kMxTile128, kMxTile256, kMxShapes };
struct MxShape { int kind; uint32_t splits; };
inline MxShape mx_shape(const hcnn_plain* h, const MxCall& c) {
  constexpr uint32_t kRows[] = {16, 16, 64, 64, 128, 256}, kCols[] = {16, 64, 16, 64, 128, 256};
  constexpr double kBegin[] = {2.9, 3.3, 3.2, 6.0, 4.5, 7.0}, kMore[] = {0.3, 1.0, 0.8, 2.2, 2.3, 9.0};     // a launch; each further workgroup of a unit
  constexpr double kStep[2][kMxShapes] = {{0.05, 0.145, 0.14, 0.25, 0.37, 1.0}, {0.06, 0.16, 0.22, 0.42, 1.1, 2.6}};
  constexpr double kLoad[2][kMxShapes] = {{0.07, 0.2, 0.15, 0.17, 0.29, 0.84}, {0.08, 0.22, 0.33, 0.53, 0.85, 2.5}};
  // offsets within a tile and a step in 32 bits
  const bool tiles = 256 * mx_row_bytes(c.format, c.K) < ((size_t)1 << 32) && 4 * std::max(c.x_pitch, c.w_pitch) < ((size_t)1 << 32) && c.K && c.M > 16 && c.N > 16;
  const int f = c.format == kMx4 ? 0 : 1;
  const size_t steps = blocks(c.K, 128);
#ifdef HCNN_HOSTEMU
  if (emu_tile >= 0 && tiles) return emu_tile == kTile256 ? MxShape{kMxTile256, emu_parts} : emu_tile == kTile128 ? MxShape{kMxTile128, emu_parts} : MxShape{kMxStrip44, 1};
#endif
  MxShape best{kMxStrip44, 1};
  double least = 1e300;
  for (int k = 0; k < kMxShapes; ++k) {
    if ((kRows[k] == 16 && c.M > 16) || (k >= kMxTile128 && !tiles)) continue;
    const double all = (double)blocks(c.M, kRows[k]) * (double)blocks(c.N, kCols[k]);
    for (uint32_t s = 1; s == 1 || (k >= kMxTile128 && s <= 8 && s * 4 <= steps); ++s) {
      const double load = std::ceil(all * s / h->compute_units);
      double us = kBegin[k] + kMore[k] * (load - 1) + std::max(kStep[f][k], kLoad[f][k] * load) * (double)blocks(steps, s);
      if (s > 1) us += 3.0 + (double)s * (double)c.M * (double)c.N * 8 / 4.2e6;
      if (us < least) {
        least = us;
        best = MxShape{k, s};
      }
    }
  }
  return best;
}
template <class T, int F, int BM, int BN, int WM, int WN>
int mx_tile(hcnn_plain* h, MxArgs& a) {
  typedef MxTile<T, F, BM, BN, WM, WN, kEpiOut> One;
  typedef MxTile<T, F, BM, BN, WM, WN, kEpiSums> Parts;
  const size_t grid = One::grid(a.g);
  if (grid > most_workgroups(One::kThreads)) return HCNN_ERR_ARG;
#ifdef HCNN_HOSTEMU
  emu_taken |= (uint64_t)1 << (a.g.splits == 1 ? 0 : 1) << (BM == 256 ? 0 : 2) << (F == kMx4 ? 0 : 4);
#endif
  if (a.g.splits == 1) return launch<One>(h->stream, grid, One::kLdsBytes, a);
  a.g.ld_sums = up(a.g.N, 8);
  const int e = reserve(h, (size_t)a.g.splits * a.g.M * a.g.ld_sums * 4);
  if (e) return e;
  a.g.sums = at<float>(h, 0);
  const int f = launch<Parts>(h->stream, grid, Parts::kLdsBytes, a);
  return f ? f : launch<GemmJoin<T, 1>>(h->stream, GemmJoin<T, 1>::grid(a.g), 0, a.g);
}
template <class T, int F>
int linear_mx_of(hcnn_plain* h, const MxCall& c) {
  MxArgs a{};
  a.g.M = (uint32_t)c.M; a.g.N = (uint32_t)c.N; a.g.act = c.act; a.g.splits = 1;
  a.g.bias = c.bias; a.g.residual = c.residual; a.g.ld_residual = c.ld_residual; a.g.out = c.y; a.g.ld_out = c.ldy;
  a.x = c.x; a.x_scales = c.x_scales; a.x_pitch = c.x_pitch; a.x_bytes = mx_row_bytes(F, c.K);
  a.w = c.w; a.w_scales = c.w_scales; a.w_pitch = c.w_pitch; a.w_bytes = mx_row_bytes(kMx4, c.K);
  a.steps = (uint32_t)blocks(c.K, 128);
  const MxShape s = mx_shape(h, c);
  auto strip = [&](auto kernel) {
    typedef decltype(kernel) S;
    const size_t grid = S::grid(a.g), most = most_workgroups(S::kThreads);
    int e = 0;
    for (a.first = 0; a.first < grid && !e; a.first += most) e = launch<S>(h->stream, std::min(most, grid - a.first), S::kLdsBytes, a);
    return e;
  };
  if (s.kind >= kMxTile128) {
    a.part = (uint32_t)up(blocks(a.steps, s.splits), 2);
    a.g.splits = (uint32_t)blocks(a.steps, a.part);
  }
  switch (s.kind) {
    case kMxStrip11: return strip(MxStrip<T, F, 1, 1>{});
    case kMxStrip14: return strip(MxStrip<T, F, 1, 4>{});
    case kMxStrip41: return strip(MxStrip<T, F, 4, 1>{});
    case kMxStrip44: return strip(MxStrip<T, F, 4, 4>{});
    case kMxTile128: return mx_tile<T, F, 128, 128, 2, 2>(h, a);
    // (of eight bits, whose x every wave parts in two: the waves that share a row's x are two in place of four, 8192 x 4096 -> 16384 781 -> 690 us)
    default: return mx_tile<T, F, 256, 256, F == kMx8 ? 4 : 2, F == kMx8 ? 2 : 4>(h, a);
  }
}
template <class T>
int linear_mx(hcnn_plain* h, const MxCall& c) { return c.format == kMx4 ? linear_mx_of<T, kMx4>(h, c) : linear_mx_of<T, kMx8>(h, c); }

}  // namespace plain_host

// What a number type's translation unit defines
#define PLAIN_ROWS_TYPE(PREFIX, T)                                                                                                            \
  namespace plain_host {                                                                                                                      \
  PREFIX template int dropout<T>(hcnn_plain*, size_t, size_t, const void*, size_t, const void*, size_t, double, uint64_t, uint32_t, void*, size_t); \
  PREFIX template int rms_norm<T>(hcnn_plain*, size_t, size_t, const void*, size_t, const void*, size_t, const void*, double, void*, size_t, void*, size_t, const MxOut&); \
  PREFIX template int rms_norm_grad<T>(hcnn_plain*, size_t, size_t, const void*, size_t, const void*, size_t, const void*, const void*, size_t, double, void*, size_t, void*); \
  PREFIX template int quantize<T>(hcnn_plain*, int, size_t, size_t, const void*, size_t, const MxOut&, void*, size_t);                         \
  PREFIX template int linear_mx<T>(hcnn_plain*, const MxCall&);                                                                               \
  }
