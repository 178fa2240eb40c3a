// Host side of the plain network's training: choice of the kernels' shapes, their order, work memory.  Templates over the number
// type, instantiated in a translation unit for each.
#pragma once
#include "../../include/hcnn.h"

#include <algorithm>
#include <cmath>
#include <new>

#include "plain_kernels.h"

using namespace hcnn;

struct hcnn_plain {
  struct Block { char* p; Block* next; };
  hcnn_stream_t stream = nullptr;
  char* work = nullptr;                       // grows to the largest call's need
  size_t work_bytes = 0;
  bool recorded = false;                      // `work` is in the launches of a recorded graph
  Block* kept = nullptr;                      // outgrown blocks that are
  unsigned long long* d_bad = nullptr;
  uint32_t compute_units = 256;
};

namespace plain_host {

constexpr size_t kMaxSize = 0x7fffffff;
constexpr size_t kDeltaBytes = (size_t)512 << 20;      // scores' gradients held at a time by hcnn_cross_entropy_grad

inline size_t up(size_t x, size_t to) { return (x + to - 1) / to * to; }
inline size_t blocks(size_t x, size_t each) { return (x + each - 1) / each; }
inline size_t type_bytes(int dtype) { return dtype == HCNN_F32 ? 4 : 2; }
inline bool bad_type(int dtype) { return dtype != HCNN_F32 && dtype != HCNN_F16 && dtype != HCNN_BF16; }
inline bool misaligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % type_bytes(dtype) != 0; }

// Work memory of one call, cut into arrays: sizes first, then addresses.
struct Arena {
  size_t bytes = 0;
  size_t take(size_t n) {
    const size_t at = bytes;
    bytes += up(n, 256);
    return at;
  }
};
// A recorded graph reads and writes the block that its calls had: such a block is outgrown, but not freed before the handle.
inline int reserve(hcnn_plain* h, size_t bytes) {
  const bool recording = stream_recording(h->stream);
  if (bytes > h->work_bytes) {
    const bool keep = h->work && (h->recorded || recording);      // (while it is recorded, the stream cannot be waited for)
    hcnn_plain::Block* old = keep ? new (std::nothrow) hcnn_plain::Block{h->work, h->kept} : nullptr;
    if (keep && !old) return HCNN_ERR_ARG;
    if (h->work && !keep) {
      const int e = stream_sync(h->stream);
      if (e) return e;
      dev_free(h->work);
      h->work = nullptr;
      h->work_bytes = 0;
    }
    void* p = nullptr;
    const int e = dev_malloc(&p, bytes);
    if (e) {
      delete old;
      return e;
    }
    if (keep) h->kept = old;
    h->work = static_cast<char*>(p);
    h->work_bytes = bytes;
    h->recorded = false;
  }
  if (recording) h->recorded = true;
  return 0;
}
template <class V> V* at(hcnn_plain* h, size_t offset) { return reinterpret_cast<V*>(h->work + offset); }

// ---------------------------------------------------------------- tiles
enum { kTile256, kTile128, kTile64, kTall, kFlat };
struct Shape { int tile; uint32_t bm, bn, splits; bool direct; };
constexpr uint32_t kTileRows[] = {256, 128, 64, 128, 16}, kTileCols[] = {256, 128, 64, 16, 128};

// Tile and parts of k by an estimate of the time in us: `load` workgroups for each compute unit, `held` of them at a time; a stage takes
// what the unit's matrix instructions and LDS need for it (kFull, per workgroup) or a load's way (kAlone), whichever is more; a
// workgroup's beginning and ending kEnds; parts of k are written and joined.  (kFull is that of operands along k.  In 32 bits with both
// across k a stage of 64 x 64 took 0.7, not 0.5: dw of 8192 x 2048 -> 256 91 us in 512 workgroups where the estimate has 68.)
template <class T>
Shape choose(const hcnn_plain* h, size_t M, size_t N, size_t K, bool may_split, bool direct) {
  constexpr bool wide = sizeof(T) == 4;
  constexpr double kFull[] = {1.5, wide ? 1.9 : 0.55, wide ? 0.5 : 0.2, wide ? 0.3 : 0.12, wide ? 0.3 : 0.12};
  constexpr double kHeld[] = {1, 2, 4, 4, 4}, kEnds[] = {10, 6, 4, 4, 4}, kAlone = 0.7;
  const double units = h->compute_units;
  const size_t stages = std::max<size_t>(1, blocks(K, GemmNum<T>::kStage));
#ifdef HCNN_HOSTEMU
  if (emu_tile >= 0 && (emu_tile != kTile256 || (!wide && direct)))
    return Shape{emu_tile, kTileRows[emu_tile], kTileCols[emu_tile], may_split ? (uint32_t)std::max<size_t>(1, std::min<size_t>(emu_parts, stages / 2)) : 1, direct};
#endif
  Shape best{kTile64, 64, 64, 1, direct};
  double least = 1e300;
  for (int t = kTile256; t <= kFlat; ++t) {
    if (t == kTile256 && (wide || !direct)) continue;
    const size_t tiles = std::max<size_t>(1, blocks(M, kTileRows[t]) * blocks(N, kTileCols[t]));
    for (size_t s = 1; s == 1 || (may_split && s * 2 <= stages && s <= 64); s += s < 8 ? 1 : s / 4) {
      const double load = std::ceil((double)(tiles * s) / units), turns = std::ceil(load / kHeld[t]);
      const double stage = std::max(kAlone * turns, load * kFull[t]) * (direct ? 1.0 : 1.6);
      double us = (double)blocks(stages, s) * stage + turns * kEnds[t];
      if (s > 1) us += 5.0 + (double)(2 * s * M * N * 4) / 3e6;
      if (us < least) {
        least = us;
        best = Shape{t, kTileRows[t], kTileCols[t], (uint32_t)s, direct};
      }
    }
  }
  return best;
}
inline size_t sums_bytes(const Shape& s, size_t M, size_t N) { return s.splits > 1 ? s.splits * M * up(N, 8) * 4 : 0; }

template <class G>
int start(hcnn_plain* h, const GemmArgs& a, size_t grid) { return launch<G>(h->stream, grid, G::kLdsBytes, a); }

// An operand as the caller has it, or a copy of it in the work memory whose rows all start on 16 bytes, as whole stages' way to LDS
// past the registers needs them (also: offsets within a stage in 32 bits).
struct Input {
  const void* p;
  size_t ld, rows, cols;
  bool packed = false;
  size_t offset = 0;
  size_t extent() const { return rows && cols ? packed ? rows * ld : (rows - 1) * ld + cols : 0; }
};
template <class T>
bool direct_input(const Input& x) {
  const bool aligned = x.packed || (reinterpret_cast<uintptr_t>(x.p) % 16 == 0 && x.ld * sizeof(T) % 16 == 0);
  return aligned && 257 * x.ld * sizeof(T) < ((size_t)1 << 32);
}
// Copies pay from some size of the products that take the operand on: `work` = M N K of all of them against a launch and the bytes read
// and written.  Measured with and without copies of both operands, bfloat16 products of odd sizes M = N = K, us: 1001 20.4 / 15.0,
// 2001 54.6 / 50.0, 2501 70.0 / 70.8, 4001 157 / 225; 8192 x 517 x 1000 34.5 / 24.4, 256 x 4001 x 4001 43.5 / 35.7.  32-bit
// products are bound by the matrix unit either way.
constexpr double kPackWork = 0.6e-15, kPackByte = 2e-13, kPackLaunch = 4e-6;       // seconds
inline bool copy_pays(const Input& x, double work) {
#ifdef HCNN_HOSTEMU
  if (emu_copies) return true;
#endif
  return work * kPackWork >= kPackLaunch + 4.0 * (double)x.rows * (double)x.cols * kPackByte;
}
template <class T>
void plan_pack(Input& x, Arena& a, double work) {
  if (sizeof(T) != 2 || direct_input<T>(x) || x.rows == 0 || x.cols == 0) return;
  if (!copy_pays(x, work)) return;
  x.packed = true;
  x.ld = up(x.cols, GemmNum<T>::kStage);                // whole stages along the row, zeros at its end
  x.offset = a.take(x.rows * x.ld * sizeof(T));
}
template <class T>
int pack(hcnn_plain* h, Input& x, const void* from, size_t ld_from) {
  if (!x.packed) return 0;
#ifdef HCNN_HOSTEMU
  ++emu_copied;
#endif
  const size_t pieces = x.rows * (x.ld / 8), grid = std::min(blocks(pieces, PackRows::kThreads), most_workgroups(PackRows::kThreads));
  const PackArgs p{from, ld_from, at<void>(h, x.offset), x.ld, (uint32_t)x.rows, (uint32_t)x.cols, pieces, grid * PackRows::kThreads};
  x.p = p.to;
  return launch<PackRows>(h->stream, grid, 0, p);
}
template <class T, int LA, int LB, int EPI>
int gemm(hcnn_plain* h, const GemmArgs& a, const Shape& s) {
  const size_t grid = blocks(a.M, s.bm) * blocks(a.N, s.bn) * s.splits;
  if (grid > kMaxSize) return HCNN_ERR_ARG;
#ifdef HCNN_HOSTEMU
  emu_taken |= (uint64_t)1 << (EPI * 16 + s.tile * 2 + s.direct);
#endif
#define PLAIN_TILE(BM, BN, WM, WN) \
  return s.direct ? start<Gemm<T, LA, LB, BM, BN, WM, WN, EPI, true>>(h, a, grid) : start<Gemm<T, LA, LB, BM, BN, WM, WN, EPI, false>>(h, a, grid)
  switch (s.tile) {
    case kTile256:
      if constexpr (sizeof(T) == 2)
        if (s.direct) return start<Gemm<T, LA, LB, 256, 256, 2, 4, EPI, true>>(h, a, grid);
      return HCNN_ERR_ARG;
    case kTile128: PLAIN_TILE(128, 128, 2, 2);
    case kTile64: PLAIN_TILE(64, 64, 2, 2);
    case kTall: PLAIN_TILE(128, 16, 4, 1);
    default: PLAIN_TILE(16, 128, 1, 4);
  }
#undef PLAIN_TILE
}
// The product with the linear layer's ending, in parts of k where the shape says so (their sums at `sums`).
template <class T, int LA, int LB>
int product(hcnn_plain* h, GemmArgs a, const Shape& s, float* sums) {
  if (a.M == 0 || a.N == 0) return 0;
  a.splits = s.splits;
  if (s.splits == 1) return gemm<T, LA, LB, kEpiOut>(h, a, s);
  a.sums = sums;
  a.ld_sums = up(a.N, 8);
  const int e = gemm<T, LA, LB, kEpiSums>(h, a, s);
  if (e) return e;
  // the parts side by side where there are fewer outputs than a workgroup of quads for each compute unit
  const bool few = (size_t)a.M * blocks(a.N, 4) < (size_t)h->compute_units * 256 && s.splits >= 8;
  if (few) return launch<GemmJoin<T, 8>>(h->stream, GemmJoin<T, 8>::grid(a), GemmJoin<T, 8>::kLdsBytes, a);
  return launch<GemmJoin<T, 1>>(h->stream, GemmJoin<T, 1>::grid(a), 0, a);
}

inline GemmArgs operands(const Input& a, const Input& b) {
  GemmArgs g{};
  g.a = a.p; g.lda = a.ld; g.a_extent = a.extent();
  g.b = b.p; g.ldb = b.ld; g.b_extent = b.extent();
  g.splits = 1;
  return g;
}

constexpr size_t kShortRow = 1024;       // bytes up to which a wave takes whole rows (Strip)
template <class T, bool NARROW, int SHARE>
int strip(hcnn_plain* h, const GemmArgs& g, size_t streamed) {
  typedef Strip<T, NARROW, SHARE, false> S;
  return launch<S>(h->stream, blocks(streamed, S::kRows), S::kLdsBytes, g);
}

// ---------------------------------------------------------------- linear layer
template <class T>
int linear(hcnn_plain* h, int act, size_t M, size_t K, size_t N, const void* x, size_t ldx, const void* w, size_t ldw, const void* bias,
           const void* residual, size_t ld_residual, void* y, size_t ldy, void* z, size_t ldz) {
  if (K && (M <= 16 || N <= 16)) {
    GemmArgs g = operands(Input{x, ldx, M, K}, Input{w, ldw, N, K});
    g.M = (uint32_t)M; g.N = (uint32_t)N; g.K = (uint32_t)K;
    g.act = act; g.bias = bias; g.residual = residual; g.ld_residual = ld_residual;
    g.out = y; g.ld_out = ldy; g.z = z; g.ld_z = ldz;
    if (M <= 16) return strip<T, false, 8>(h, g, N);
    return K * sizeof(T) <= kShortRow ? strip<T, true, 1>(h, g, M) : strip<T, true, 8>(h, g, M);
  }
  Arena ar;
  Input ix{x, ldx, M, K}, iw{w, ldw, N, K};
  const double work = (double)M * (double)N * (double)K;
  plan_pack<T>(ix, ar, work);
  plan_pack<T>(iw, ar, work);
  const Shape s = choose<T>(h, M, N, K, true, direct_input<T>(ix) && direct_input<T>(iw));
  const size_t o_sums = ar.take(sums_bytes(s, M, N));
  int e = reserve(h, ar.bytes);
  if (e || (e = pack<T>(h, ix, x, ldx)) || (e = pack<T>(h, iw, w, ldw))) return e;
  GemmArgs g = operands(ix, iw);
  g.M = (uint32_t)M; g.N = (uint32_t)N; g.K = (uint32_t)(ix.packed && iw.packed ? ix.ld : K);
  g.act = act; g.bias = bias; g.residual = residual; g.ld_residual = ld_residual;
  g.out = y; g.ld_out = ldy; g.z = z; g.ld_z = ldz;
  return product<T, kAlongK, kAlongK>(h, g, s, at<float>(h, o_sums));
}

enum { kSizeOnly, kTops, kGradients };
template <class T, int LANES>
int act_grad_lanes(hcnn_plain* h, const ActGradArgs& a, size_t grid, int what) {
  if constexpr (std::is_same_v<T, Half>) {
    if (what == kTops) return launch<ActTops<T, LANES>>(h->stream, grid, ActTops<T, LANES>::kLdsBytes, a);
    if (a.row_top || a.col_top) return launch<ActGrad<T, LANES, kRoom>>(h->stream, grid, ActGrad<T, LANES, kRoom>::kLdsBytes, a);
  }
  return launch<ActGrad<T, LANES, kNoRoom>>(h->stream, grid, ActGrad<T, LANES, kNoRoom>::kLdsBytes, a);
}
template <class T>
int act_grad(hcnn_plain* h, ActGradArgs a, size_t* row_blocks, int what) {
  // at least 64 rows a workgroup, and no more workgroups than eight for each compute unit
  const int lanes = a.N <= 16 ? 4 : a.N <= 64 ? 16 : 64;
  a.col_blocks = (uint32_t)std::max<size_t>(1, blocks(a.N, lanes * 4));
  const size_t most = std::max<size_t>(1, (size_t)h->compute_units * 8 / a.col_blocks);
  a.rows_each = (uint32_t)std::max<size_t>(64, up(blocks(a.M, most), 64));
  *row_blocks = blocks(a.M, a.rows_each);
  if (what == kSizeOnly) return 0;
  const size_t grid = *row_blocks * a.col_blocks;
  switch (lanes) {
    case 4: return act_grad_lanes<T, 4>(h, a, grid, what);
    case 16: return act_grad_lanes<T, 16>(h, a, grid, what);
    default: return act_grad_lanes<T, 64>(h, a, grid, what);
  }
}

template <class T>
int linear_grad(hcnn_plain* h, int act, size_t M, size_t K, size_t N, const void* dy, size_t ld_dy, const void* x, size_t ldx, const void* w,
                size_t ldw, const void* z, size_t ldz, void* dx, size_t ld_dx, void* dw, size_t ld_dw, void* db) {
  const double work = (double)M * (double)N * (double)K;
  ActGradArgs ag{};
  ag.dy = dy; ag.ld_dy = ld_dy; ag.M = (uint32_t)M; ag.N = (uint32_t)N; ag.act = act;
  if (act != kActNone) { ag.z = z; ag.ld_z = ldz; }
  ag.ld_part = up(N, 4);
  size_t row_blocks = 0;
  act_grad<T>(h, ag, &row_blocks, kSizeOnly);
  // dz in binary16 of a slope that is any number: times powers of two of its rows (for dx) and of its columns (for dw), see ActGrad
  const bool room = std::is_same_v<T, Half> && act != kActNone && act != kActRelu;
  Arena ar;
  Input ix{x, ldx, M, K}, iw{w, ldw, N, K}, idz{dy, ld_dy, M, N};
  if (act != kActNone) {                                   // dz: aligned rows in the work memory
    idz.packed = true;
    idz.ld = up(N, 16 / sizeof(T));
    if (dx || (dw && !room)) idz.offset = ar.take(M * idz.ld * sizeof(T));
  } else {
    plan_pack<T>(idz, ar, work * ((dx != nullptr) + (dw != nullptr)));
  }
  Input idw = idz;                                         // dw's
  if (room && dw) idw.offset = ar.take(M * idz.ld * sizeof(T));
  const size_t o_tops = ar.take(room ? (M + N) * 4 : 0);
  if (dw) plan_pack<T>(ix, ar, work);
  if (dx) plan_pack<T>(iw, ar, work);
  const bool direct = direct_input<T>(idz);
  const Shape sx = choose<T>(h, M, K, N, true, direct && direct_input<T>(iw)), sw = choose<T>(h, N, K, M, true, direct && direct_input<T>(ix));
  const size_t o_part = ar.take(db ? row_blocks * ag.ld_part * 4 : 0);
  const size_t o_sums = ar.take(std::max(dx ? sums_bytes(sx, M, K) : 0, dw ? sums_bytes(sw, N, K) : 0));
  int e = reserve(h, ar.bytes);
  if (e || (e = pack<T>(h, ix, x, ldx)) || (e = pack<T>(h, iw, w, ldw))) return e;
  if (act == kActNone) {
    if ((e = pack<T>(h, idz, dy, ld_dy))) return e;
    idw.p = idz.p;
  } else {
    idz.p = at<void>(h, idz.offset);
    idw.p = at<void>(h, idw.offset);
    ag.dz = dx || (dw && !room) ? at<void>(h, idz.offset) : nullptr;     // (db alone takes no dz)
    ag.ld_dz = idz.ld;
  }
  if (M && N && room && (dx || dw)) {
    uint32_t* tops = at<uint32_t>(h, o_tops);
    ag.row_top = dx ? tops : nullptr;
    ag.col_top = dw ? tops + M : nullptr;
    ag.dz_cols = dw ? at<void>(h, idw.offset) : nullptr;
    if ((e = launch<ZeroWords>(h->stream, blocks(M + N, ZeroWords::kThreads), 0, ZeroWordsArgs{tops, M + N}))) return e;
    if ((e = act_grad<T>(h, ag, &row_blocks, kTops))) return e;
  }
  if (M && N && (act != kActNone || db)) {
    if (db) ag.part = at<float>(h, o_part);
    if ((e = act_grad<T>(h, ag, &row_blocks, kGradients))) return e;
  }
  if (db && N) {
    const ColumnSumArgs cs{at<float>(h, o_part), ag.ld_part, (uint32_t)(M ? row_blocks : 0), (uint32_t)N, db};
    if ((e = launch<ColumnSum<T>>(h->stream, blocks(N, 16), ColumnSum<T>::kLdsBytes, cs))) return e;
  }
  if (dx) {
    GemmArgs g = operands(idz, iw);
    g.M = (uint32_t)M; g.N = (uint32_t)K; g.K = (uint32_t)N;
    g.top = ag.row_top;
    g.out = dx; g.ld_out = ld_dx;
    if ((e = product<T, kAlongK, kAcrossK>(h, g, sx, at<float>(h, o_sums)))) return e;
  }
  if (dw) {
    GemmArgs g = operands(idw, ix);
    g.M = (uint32_t)N; g.N = (uint32_t)K; g.K = (uint32_t)M;
    g.top = ag.col_top;
    g.out = dw; g.ld_out = ld_dw;
    if ((e = product<T, kAcrossK, kAcrossK>(h, g, sw, at<float>(h, o_sums)))) return e;
  }
  return 0;
}

// ---------------------------------------------------------------- softmax cross entropy
struct LossCall {
  size_t M, K, V;
  const void* x; size_t ldx;
  const void* w; size_t ldw;
  const void* targets; int target_bytes; int64_t ignore;
  float *row_loss, *row_lse, *loss;
  float scale;
  void* dx; size_t ld_dx;
  void* dw; size_t ld_dw;
};

// A 16-bit float with 5 bits of exponent holds nothing below 2^-24: the scores' gradients, at most 1 in magnitude, are held 2^15
// times as large there.  The factor goes back out of the sums.
template <class T> constexpr float delta_scale() { return std::is_same_v<T, Half> ? 32768.0f : 1.0f; }

template <class T, int SHARE>
int strip_loss(hcnn_plain* h, const GemmArgs& g, const RowStatsArgs& rows) {
  typedef Strip<T, true, SHARE, true> S;
  return launch<S>(h->stream, blocks(g.M, S::kRows), S::kLdsBytes, StripLossArgs{g, rows});
}

template <class T>
int cross_entropy(hcnn_plain* h, const LossCall& c, bool grad) {
  const size_t M = c.M, K = c.K, V = c.V;
  Arena a;
  Input ix{c.x, c.ldx, M, K}, iw{c.w, c.ldw, V, K};
  const double work = (double)M * (double)V * (double)K * (grad ? 3 : 1);
  plan_pack<T>(ix, a, work);
  plan_pack<T>(iw, a, work);
  // the rows that take part, one behind the other: used where they are not all rows, or where x is copied anyway
  Input ikept{c.x, ix.packed ? ix.ld : up(K, 16 / sizeof(T)), M, K, true, ix.offset};
  if (!ix.packed) ikept.offset = a.take(M * ikept.ld * sizeof(T));
  // columns of a piece: whole tiles, all columns where they fit
  const size_t fit = kDeltaBytes / (std::max<size_t>(M, 1) * sizeof(T)) / 256 * 256;
  const size_t piece = grad ? std::min(V, std::max<size_t>(fit, 256)) : 0;
  const size_t pieces = grad ? blocks(V, piece) : 0, ld_delta = up(piece, 16 / sizeof(T));
  const bool direct_x = direct_input<T>(ix) && direct_input<T>(ikept), direct_w = direct_input<T>(iw);
  const Shape ss = choose<T>(h, M, V, K, false, direct_x && direct_w);
  Input idelta{nullptr, ld_delta, M, piece, true, a.take(grad ? M * ld_delta * sizeof(T) : 0)};
  const bool direct_d = direct_input<T>(idelta);
  const Shape sx = choose<T>(h, M, K, piece, pieces == 1, direct_d && direct_w), sw = choose<T>(h, piece, K, M, true, direct_d && direct_x);
  const bool narrow = V <= 16 && K;                             // scores, losses and the scores' gradients in one kernel
  const size_t tiles = narrow ? 0 : blocks(V, ss.bn), ld_stats = up(M, 64), row_wgs = blocks(M, 16);
  const size_t o_count = a.take(4), o_alpha = a.take(4), o_rows = a.take(M * 4), o_target = a.take(M * 4), o_score = a.take(M * 4), o_lse = a.take(M * 4);
  const size_t o_stats = a.take(tiles * 2 * ld_stats * 4), o_part = a.take(row_wgs * 8);
  const size_t o_dx = a.take(pieces > 1 && c.dx ? M * up(K, 8) * 4 : 0);
  const size_t o_sums = a.take(grad ? std::max(c.dx ? sums_bytes(sx, M, K) : 0, c.dw ? sums_bytes(sw, piece, K) : 0) : 0);
  int e = reserve(h, a.bytes);
  if (e || (e = pack<T>(h, iw, c.w, c.ldw))) return e;
  idelta.p = at<void>(h, idelta.offset);
  uint32_t *count = at<uint32_t>(h, o_count), *rows = at<uint32_t>(h, o_rows), *target = at<uint32_t>(h, o_target);
  float *alpha = at<float>(h, o_alpha), *score = at<float>(h, o_score), *lse = at<float>(h, o_lse);

  KeepRowsArgs kr{c.targets, c.target_bytes == 8, c.ignore, (uint32_t)M, (uint32_t)V, rows, target, count, h->d_bad, c.loss, alpha, c.scale / delta_scale<T>()};
  if ((e = launch<KeepRows>(h->stream, 1, KeepRows::kLdsBytes, kr))) return e;
  if (M) {
    const size_t grid = std::min(blocks(M, 4), most_workgroups(SortRows::kThreads));
    const SortRowsArgs sr{kr, K ? c.dx : nullptr, c.ld_dx * sizeof(T), K * sizeof(T), c.row_loss, c.row_lse,
                          c.x, c.ldx * sizeof(T), at<void>(h, ikept.offset), ikept.ld * sizeof(T), ix.packed, (uint32_t)grid * 4};
    if ((e = launch<SortRows>(h->stream, grid, 0, sr))) return e;
  }
  if (ix.packed) ix.p = at<void>(h, ikept.offset);
  GemmArgs g = operands(ix, iw);
  g.M = (uint32_t)M; g.N = (uint32_t)V; g.K = (uint32_t)(ix.packed && iw.packed ? ix.ld : K);
  g.count = count; g.count_of = kCountM; g.kept = at<void>(h, ikept.offset); g.ld_kept = ikept.ld; g.kept_always = ix.packed;
  g.stats = at<float>(h, o_stats); g.ld_stats = ld_stats; g.target = target; g.target_score = score; g.lse = lse;
  g.delta_scale = delta_scale<T>();
  const RowStatsArgs rs{g.stats, ld_stats, (uint32_t)tiles, (uint32_t)M, count, rows, score, lse, at<double>(h, o_part), c.row_loss, c.row_lse};
  if (M && narrow) {
    if (grad) { g.out = at<void>(h, idelta.offset); g.ld_out = ld_delta; }
    if ((e = K * sizeof(T) <= kShortRow ? strip_loss<T, 1>(h, g, rs) : strip_loss<T, 8>(h, g, rs))) return e;
  } else if (M) {
    if ((e = gemm<T, kAlongK, kAlongK, kEpiStats>(h, g, ss))) return e;
    if ((e = launch<RowStats>(h->stream, blocks(M, RowStats::kRows), RowStats::kLdsBytes, rs))) return e;
  }
  if (M && c.loss) {
    const size_t groups = blocks(M, !narrow ? RowStats::kRows : K * sizeof(T) <= kShortRow ? Strip<T, true, 1, true>::kRows : Strip<T, true, 8, true>::kRows);
    const MeanLossArgs ml{at<double>(h, o_part), (uint32_t)groups, count, c.loss};
    if ((e = launch<MeanLoss>(h->stream, 1, MeanLoss::kLdsBytes, ml))) return e;
  }

  for (size_t p = 0; p < pieces; ++p) {
    const size_t v0 = p * piece, n = std::min(piece, V - v0);
    Input wp{static_cast<const char*>(iw.p) + v0 * iw.ld * sizeof(T), iw.ld, n, K, iw.packed};
    idelta.cols = n;
    if (M && !narrow) {
      GemmArgs d = g;
      d.b = wp.p; d.b_extent = wp.extent();
      d.N = (uint32_t)n; d.n_offset = (uint32_t)v0;
      d.out = at<void>(h, idelta.offset); d.ld_out = ld_delta;
      if ((e = gemm<T, kAlongK, kAlongK, kEpiDelta>(h, d, choose<T>(h, M, n, K, false, direct_x && direct_w)))) return e;
    }
    if (c.dx && M && K) {
      GemmArgs d = operands(idelta, wp);
      d.M = (uint32_t)M; d.N = (uint32_t)K; d.K = (uint32_t)n;
      d.count = count; d.count_of = kCountM;
      if (p) { d.addend = at<float>(h, o_dx); d.ld_sums = up(K, 8); }
      if (p + 1 < pieces) {
        d.sums = at<float>(h, o_dx); d.ld_sums = up(K, 8);
        if ((e = gemm<T, kAlongK, kAcrossK, kEpiSums>(h, d, sx))) return e;
      } else {
        d.rows = rows; d.alpha = alpha;
        d.out = c.dx; d.ld_out = c.ld_dx;
        if ((e = product<T, kAlongK, kAcrossK>(h, d, sx, at<float>(h, o_sums)))) return e;
      }
    }
    if (c.dw && K) {
      GemmArgs d = operands(idelta, ix);
      d.M = (uint32_t)n; d.N = (uint32_t)K; d.K = (uint32_t)M;
      d.count = count; d.count_of = kCountK; d.kept = at<void>(h, ikept.offset); d.ld_kept = ikept.ld; d.kept_always = ix.packed; d.alpha = alpha;
      d.out = static_cast<char*>(c.dw) + v0 * c.ld_dw * sizeof(T); d.ld_out = c.ld_dw;
      if ((e = product<T, kAcrossK, kAcrossK>(h, d, sw, at<float>(h, o_sums)))) return e;
    }
  }
  return 0;
}

}  // namespace plain_host

// What a number type's translation unit defines
#define PLAIN_TYPE(PREFIX, T)                                                                                                             \
  namespace plain_host {                                                                                                                 \
  PREFIX template int linear<T>(hcnn_plain*, int, size_t, size_t, size_t, const void*, size_t, const void*, size_t, const void*, const void*, \
                                size_t, void*, size_t, void*, size_t);                                                                   \
  PREFIX template int linear_grad<T>(hcnn_plain*, int, size_t, size_t, size_t, const void*, size_t, const void*, size_t, const void*, size_t, \
                                     const void*, size_t, void*, size_t, void*, size_t, void*);                                          \
  PREFIX template int cross_entropy<T>(hcnn_plain*, const LossCall&, bool);                                                              \
  }
