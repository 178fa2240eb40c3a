// C ABI of the plain (unencrypted) network's training: argument checks and the calls behind them.  The device build has a
// translation unit of its own for each number type; the CPU checker is built from hcnn.cpp, which includes this file there.
#include "plain_host.h"

#ifndef HCNN_HOSTEMU
PLAIN_TYPE(extern, float)
PLAIN_TYPE(extern, Half)
PLAIN_TYPE(extern, Bfloat)
#endif

namespace plain_host {

constexpr size_t kClipSmall = 32768;

// The call of the operator for its number type.
#define PLAIN_BY_TYPE(dtype, fn, ...) \
  (dtype == HCNN_F32 ? fn<float>(__VA_ARGS__) : dtype == HCNN_F16 ? fn<Half>(__VA_ARGS__) : fn<Bfloat>(__VA_ARGS__))

int loss_checked(hcnn_plain* h, int dtype, const LossCall& c, bool grad) {
  if (bad_type(dtype)) return HCNN_ERR_ARG;
  if (c.M > kMaxSize || c.K > kMaxSize || c.V == 0 || c.V > kMaxSize || (c.target_bytes != 4 && c.target_bytes != 8)) return HCNN_ERR_ARG;
  if ((c.M && !c.targets) || (c.M && c.K && !c.x) || (c.K && !c.w)) return HCNN_ERR_NULL;
  if (misaligned(c.x, dtype) || misaligned(c.w, dtype) || misaligned(c.dx, dtype) || misaligned(c.dw, dtype)) return HCNN_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(c.targets) % c.target_bytes || misaligned(c.row_loss, HCNN_F32) || misaligned(c.row_lse, HCNN_F32) ||
      misaligned(c.loss, HCNN_F32))
    return HCNN_ERR_ALIGN;
  if ((c.dx && c.ld_dx < c.K) || (c.dw && c.ld_dw < c.K)) return HCNN_ERR_ARG;
  return PLAIN_BY_TYPE(dtype, cross_entropy, h, c, grad);
}

}  // namespace plain_host

using namespace plain_host;

extern "C" {

int hcnn_plain_create(hcnn_plain** out, void* hip_stream) {
  if (!out) return HCNN_ERR_NULL;
  *out = nullptr;
  if (max_lds_bytes() < 128 * 1024) return HCNN_ERR_NODEVICE;
  hcnn_plain* h = new (std::nothrow) hcnn_plain();
  if (!h) return HCNN_ERR_ARG;
  h->stream = (hcnn_stream_t)hip_stream;
  h->compute_units = compute_unit_count();
  void* p = nullptr;
  int e = dev_malloc(&p, sizeof(unsigned long long));
  if (!e) {
    h->d_bad = static_cast<unsigned long long*>(p);
    e = dev_memset(p, 0, sizeof(unsigned long long), h->stream);
  }
  if (e) {
    hcnn_plain_destroy(h);
    return e;
  }
  *out = h;
  return HCNN_OK;
}

int hcnn_plain_destroy(hcnn_plain* h) {
  if (!h) return HCNN_ERR_NULL;
  stream_sync(h->stream);
  if (h->work) dev_free(h->work);
  while (hcnn_plain::Block* b = h->kept) {
    h->kept = b->next;
    dev_free(b->p);
    delete b;
  }
  if (h->d_bad) dev_free(h->d_bad);
  delete h;
  return HCNN_OK;
}

int hcnn_plain_set_stream(hcnn_plain* h, void* hip_stream) {
  if (!h) return HCNN_ERR_NULL;
  const int e = stream_sync(h->stream);
  if (e) return e;
  h->stream = (hcnn_stream_t)hip_stream;
  return HCNN_OK;
}

int hcnn_plain_get_stat(hcnn_plain* h, int which, uint64_t* out) {
  if (!h || !out) return HCNN_ERR_NULL;
  if (which == HCNN_STAT_SCRATCH_BYTES) {
    *out = h->work_bytes;
    return HCNN_OK;
  }
  if (which != HCNN_STAT_BAD_INPUT) return HCNN_ERR_ARG;
  unsigned long long v = 0;
  const int e = copy_d2h(&v, h->d_bad, sizeof(v), h->stream);
  if (e) return e;
  *out = v;
  return HCNN_OK;
}

int hcnn_linear(hcnn_plain* h, int dtype, int activation, size_t rows, size_t n_in, size_t n_out, const void* x, size_t x_stride, const void* w,
                size_t w_stride, const void* bias, const void* residual, size_t residual_stride, void* y, size_t y_stride, void* z, size_t z_stride) {
  if (!h) return HCNN_ERR_NULL;
  if (bad_type(dtype) || activation < 0 || activation >= kActCount) return HCNN_ERR_ARG;
  if (rows > kMaxSize || n_in > kMaxSize || n_out > kMaxSize) return HCNN_ERR_ARG;
  if (rows == 0 || n_out == 0) return HCNN_OK;
  if ((n_in && (!x || !w)) || !y) return HCNN_ERR_NULL;
  for (const void* p : {x, w, bias, residual, (const void*)y, (const void*)z})
    if (misaligned(p, dtype)) return HCNN_ERR_ALIGN;
  if (y_stride < n_out || (z && z_stride < n_out)) return HCNN_ERR_ARG;
  return PLAIN_BY_TYPE(dtype, linear, h, activation, rows, n_in, n_out, x, x_stride, w, w_stride, bias, residual, residual_stride, y, y_stride, z, z_stride);
}

int hcnn_linear_grad(hcnn_plain* h, int dtype, int activation, size_t rows, size_t n_in, size_t n_out, const void* dy, size_t dy_stride, const void* x,
                     size_t x_stride, const void* w, size_t w_stride, const void* z, size_t z_stride, void* dx, size_t dx_stride, void* dw,
                     size_t dw_stride, void* db) {
  if (!h) return HCNN_ERR_NULL;
  if (bad_type(dtype) || activation < 0 || activation >= kActCount) return HCNN_ERR_ARG;
  if (rows > kMaxSize || n_in > kMaxSize || n_out > kMaxSize) return HCNN_ERR_ARG;
  const bool any = rows && n_out;
  if (any && (!dy || (activation != kActNone && !z) || (dx && n_in && !w) || (dw && n_in && !x))) return HCNN_ERR_NULL;
  for (const void* p : {dy, x, w, z, (const void*)dx, (const void*)dw, (const void*)db})
    if (misaligned(p, dtype)) return HCNN_ERR_ALIGN;
  if ((dx && dx_stride < n_in) || (dw && dw_stride < n_in)) return HCNN_ERR_ARG;
  return PLAIN_BY_TYPE(dtype, linear_grad, h, activation, rows, n_in, n_out, dy, dy_stride, x, x_stride, w, w_stride, z, z_stride, dx, dx_stride, dw, dw_stride, db);
}

int hcnn_cross_entropy(hcnn_plain* h, int dtype, size_t rows, size_t n_in, size_t n_classes, const void* x, size_t x_stride, const void* w, size_t w_stride,
                       const void* targets, int target_bytes, int64_t ignore, float* row_loss, float* row_lse, float* loss) {
  if (!h) return HCNN_ERR_NULL;
  const LossCall c{rows, n_in, n_classes, x, x_stride, w, w_stride, targets, target_bytes, ignore, row_loss, row_lse, loss, 1.0f, nullptr, 0, nullptr, 0};
  return loss_checked(h, dtype, c, false);
}

int hcnn_cross_entropy_grad(hcnn_plain* h, int dtype, size_t rows, size_t n_in, size_t n_classes, const void* x, size_t x_stride, const void* w,
                            size_t w_stride, const void* targets, int target_bytes, int64_t ignore, float scale, float* row_loss, float* loss, void* dx,
                            size_t dx_stride, void* dw, size_t dw_stride) {
  if (!h) return HCNN_ERR_NULL;
  const LossCall c{rows, n_in, n_classes, x, x_stride, w, w_stride, targets, target_bytes, ignore, row_loss, nullptr, loss, scale, dx, dx_stride, dw, dw_stride};
  return loss_checked(h, dtype, c, true);
}

int hcnn_clip_grad_norm(hcnn_plain* h, size_t n_tensors, const void* const* grads_host, const size_t* counts_host, const int* dtypes_host,
                        void* const* outs_host, double max_norm, double eps, float* norm) {
  if (!h || !norm) return HCNN_ERR_NULL;
  if (n_tensors && (!grads_host || !counts_host || !dtypes_host)) return HCNN_ERR_NULL;
  if (!(max_norm >= 0.0) || !(eps >= 0.0) || misaligned(norm, HCNN_F32)) return HCNN_ERR_ARG;
  size_t runs = 0, filled = 0, numbers = 0;
  for (size_t i = 0; i < n_tensors; ++i) {
    if (bad_type(dtypes_host[i])) return HCNN_ERR_ARG;
    if (counts_host[i] == 0) continue;
    if (!grads_host[i] || (outs_host && !outs_host[i])) return HCNN_ERR_NULL;
    if (misaligned(grads_host[i], dtypes_host[i]) || (outs_host && misaligned(outs_host[i], dtypes_host[i]))) return HCNN_ERR_ALIGN;
    runs += blocks(counts_host[i], kNormRun);
    numbers += counts_host[i];
    ++filled;
  }
  if (runs > kMaxSize) return HCNN_ERR_ARG;
  Arena a;
  const size_t o_part = a.take(runs * 8), o_factor = a.take(8);
  int e = reserve(h, a.bytes);
  if (e) return e;
  NormArgs n{};
  n.part = at<double>(h, o_part);
  n.factor = at<double>(h, o_factor);
  n.max_norm = max_norm;
  n.eps = eps;
  n.norm = norm;
  auto add = [&](size_t i) {
    n.in[n.tensors] = grads_host[i];
    n.out[n.tensors] = outs_host ? outs_host[i] : const_cast<void*>(grads_host[i]);
    n.size[n.tensors] = counts_host[i];
    n.type[n.tensors] = (uint8_t)dtypes_host[i];
    n.first[n.tensors + 1] = n.first[n.tensors] + (uint32_t)blocks(counts_host[i], kNormRun);
    ++n.tensors;
  };
  // the list in launches of kNormTensors: up for the sums, down for the scaling, whose first reads then find what the sums read last
  auto each_list = [&](bool down, auto&& body) {
    const size_t lists = blocks(filled, kNormTensors);
    for (size_t l = 0; l < lists && !e; ++l) {
      const size_t list = down ? lists - 1 - l : l;
      size_t seen = 0;
      n.tensors = 0;
      for (size_t i = 0; i < n_tensors && n.tensors < kNormTensors; ++i)
        if (counts_host[i] && seen++ / kNormTensors == list) add(i);
      e = body();
      if (!down) n.part_first += n.first[n.tensors];
    }
  };
  // one workgroup takes up to 32768 numbers in one launch (14375 numbers of three tensors: 12.5 us a call, in three launches 21.8)
  if (numbers <= kClipSmall && filled <= kNormTensors) {
    for (size_t i = 0; i < n_tensors; ++i)
      if (counts_host[i]) add(i);
    return launch<ClipSmall>(h->stream, 1, ClipSmall::kLdsBytes, n);
  }
  each_list(false, [&] { return launch<SumSquares>(h->stream, n.first[n.tensors], SumSquares::kLdsBytes, n); });
  if (e) return e;
  const NormTotalArgs t{at<double>(h, o_part), (uint32_t)runs, max_norm, eps, norm, at<double>(h, o_factor)};
  if ((e = launch<NormTotal>(h->stream, 1, NormTotal::kLdsBytes, t))) return e;
  each_list(true, [&] { return launch<ScaleGrads>(h->stream, n.first[n.tensors], 0, n); });
  return e;
}

#ifdef HCNN_HOSTEMU
// What the checker's tests force and ask (see platform.h)
void hcnn_emu_shape(int tile, uint32_t parts, int copies) {
  emu_tile = tile;
  emu_parts = parts;
  emu_copies = copies != 0;
  emu_taken = emu_copied = 0;
}
void hcnn_emu_threads(uint64_t most) { emu_threads = most; }
void hcnn_emu_taken(uint64_t* taken, uint64_t* copied) {
  *taken = emu_taken;
  *copied = emu_copied;
}
// Tile (low byte) and parts of k that a product of these sizes takes on the handle's device; does an unaligned operand of a product get copied?
uint32_t hcnn_emu_choice(hcnn_plain* h, int dtype, size_t M, size_t N, size_t K, int may_split, int direct) {
  const Shape s = PLAIN_BY_TYPE(dtype, choose, h, M, N, K, may_split != 0, direct != 0);
  return (uint32_t)s.tile | s.splits << 8;
}
int hcnn_emu_copies(size_t rows, size_t cols, double work) { return copy_pays(Input{nullptr, cols, rows, cols}, work); }
#endif

}  // extern "C"
