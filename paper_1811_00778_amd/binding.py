"""Python binding of libhcnn.so: same names as include/hcnn.h, torch tensors on the GPU as buffers.

PyTorch supplies device memory and the HIP stream only; every step of the path
runs in the library's kernels.  There is no CPU fallback: loading fails loudly
when the HIP library has not been built.
"""
import ctypes
import os

import torch

from . import _capi
from ._ops import OpsMixin
from ._plain_ops import PlainOpsMixin

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libhcnn.so")
_lib = None


def lib() -> ctypes.CDLL:
    """The HIP library (built beforehand with `python -m paper_1811_00778_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError("libhcnn.so is not built: run `python -m paper_1811_00778_amd.build` "
                              "(or __graft_entry__.build()) first; there is no fallback path")
        _lib = _capi.declare(ctypes.CDLL(_LIB_PATH))
    return _lib


def gen_primes(n: int, count: int):
    """The `count` largest primes below 2^30 congruent to 1 mod 2n (hcnn_gen_primes)."""
    return _capi.gen_primes(lib(), n, count)


def choose_moduli(n: int, k: int, t: int):
    """(q primes, auxiliary primes): the first k primes of the rule and the minimal auxiliary basis after them."""
    cand = gen_primes(n, k + min(_capi.MAX_LIMBS, k + 8))
    q, rest = cand[:k], cand[k:]
    k_aux = _capi.min_aux_count(lib(), n, q, t, rest)
    return q, rest[:k_aux]


_DT = {"u32": torch.int32, "i32": torch.int32, "u64": torch.int64}


class Context(OpsMixin):
    """An hcnn_ctx bound to the current torch device and stream.

    uint32 residues are carried in torch.int32 tensors (same 32 bits; torch has no
    arithmetic on uint32, and none is needed here); the 64-bit plaintext words of a
    plaintext modulus above 2^32 in torch.int64 tensors."""

    def __init__(self, n, q_primes, p_primes, t, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        stream = torch.cuda.current_stream(self.device).cuda_stream
        self._stream = stream
        self.raw = _capi.RawContext(lib(), n, q_primes, p_primes, t, stream)

    def use_stream(self, stream=None):
        """Launch on `stream` (a torch.cuda.Stream; default: torch's current stream) from now on
        (hcnn_set_stream; the library waits for the work it has enqueued on the old stream first).  After one
        warm-up call per operation and size, the hot-path calls allocate nothing and enqueue kernels only, so they
        can be recorded into a HIP graph on the stream given here.

        Rule: the context's stream must be torch's current stream whenever an operation is called.  Output
        tensors come from torch's allocator, which hands a freed block out again to later work on the stream it
        was allocated on; if the library launched on another stream, that work could overwrite a buffer the
        library's kernels still use.  Every call checks this and raises instead."""
        stream = torch.cuda.current_stream(self.device) if stream is None else stream
        self.raw.call("hcnn_set_stream", ctypes.c_void_p(stream.cuda_stream))
        self._stream = stream.cuda_stream

    def _pre_call(self):
        if torch.cuda.current_stream(self.device).cuda_stream != self._stream:
            raise RuntimeError("the context is bound to another HIP stream than torch's current one: call "
                               "use_stream() inside the `with torch.cuda.stream(...)` block (and again after it)")

    def _ptr(self, x):
        return ctypes.c_void_p(x.data_ptr())

    def _empty(self, shape, dtype_name):
        return torch.empty(shape, dtype=_DT[dtype_name], device=self.device)

    def _check(self, x, dtype_name):
        if not isinstance(x, torch.Tensor) or x.dtype != _DT[dtype_name] or not x.is_contiguous() \
                or x.device != self.device:
            raise TypeError("expected a contiguous %s tensor on %s" % (_DT[dtype_name], self.device))

    # host <-> device convenience (numpy uint32/int32 arrays)
    def to_device(self, array):
        import numpy as np
        a = np.ascontiguousarray(array)
        if a.dtype == np.uint32:
            a = a.view(np.int32)
        elif a.dtype == np.uint64:
            a = a.view(np.int64)            # 64-bit plaintext words of a wide plaintext modulus
        elif a.dtype not in (np.int32, np.int64):
            raise TypeError("uint32, int32 or uint64 expected")
        return torch.from_numpy(a).to(self.device)

    def to_host_u32(self, tensor):
        import numpy as np
        torch.cuda.current_stream(self.device).synchronize()
        a = tensor.cpu().numpy()
        return a.view(np.uint64) if a.dtype == np.int64 else a.view(np.uint32)


_PLAIN_DT = {torch.float32: _capi.F32, torch.float16: _capi.F16, torch.bfloat16: _capi.BF16}


class PlainContext(PlainOpsMixin):
    """An hcnn_plain bound to a torch device and stream: the training operators of the plain network (no ring, no keys).

    Tensors are torch.float32, torch.float16 or torch.bfloat16 on the device, matrices with any row stride.  Streams follow
    Context's rule: torch's current stream must be the one of the last use_stream (at first, of creation).  The calls of one
    PlainContext share its work memory: one thread at a time.  They are outside torch's autograd: results carry no graph, whether inputs require
    gradients or not; linear_grad and cross_entropy_grad are the backward passes."""

    def __init__(self, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        torch.cuda.set_device(self.device)
        self._index = self.device.index
        self._stream = torch.cuda.current_stream(self.device).cuda_stream
        self.raw = _capi.RawPlain(lib(), self._stream)

    def use_stream(self, stream=None):
        """Launch on `stream` (default: torch's current one) from now on; see Context.use_stream."""
        stream = torch.cuda.current_stream(self.device) if stream is None else stream
        self.raw.call("hcnn_plain_set_stream", ctypes.c_void_p(stream.cuda_stream))
        self._stream = stream.cuda_stream

    def _pre_call(self):
        # (the raw handle: a stream object's making takes a fifth of a small call)
        if torch._C._cuda_getCurrentRawStream(self._index) != self._stream:
            Context._pre_call(self)

    def _matrix(self, x, what):
        if not isinstance(x, torch.Tensor) or x.dtype not in _PLAIN_DT or x.get_device() != self._index or x.dim() != 2:
            raise TypeError("%s must be a 2-D float32, float16 or bfloat16 tensor on %s" % (what, self.device))
        rows, cols = x.shape
        stride, step = x.stride()
        if step != 1 and cols > 1 and rows:
            raise TypeError("the numbers of a row of %s must lie side by side" % what)
        return x.data_ptr(), rows, cols, stride, _PLAIN_DT[x.dtype]

    def _flat(self, x, what):
        if not isinstance(x, torch.Tensor) or x.dtype not in _PLAIN_DT or x.get_device() != self._index or not x.is_contiguous():
            raise TypeError("%s must be contiguous float32, float16 or bfloat16 tensors on %s" % (what, self.device))
        return x.data_ptr(), x.numel(), _PLAIN_DT[x.dtype]

    def _vector(self, x, what):
        got = self._flat(x, what)
        if x.dim() != 1:
            raise TypeError("%s must be 1-D" % what)
        return got

    def _targets(self, x, what):
        if not isinstance(x, torch.Tensor) or x.dtype not in (torch.int32, torch.int64) or x.get_device() != self._index \
                or x.dim() != 1 or not x.is_contiguous():
            raise TypeError("%s must be a contiguous 1-D int32 or int64 tensor on %s" % (what, self.device))
        return x.data_ptr(), x.numel(), x.element_size()

    def _new(self, shape, like):
        return torch.empty(shape, dtype=torch.float32 if like is None else like.dtype, device=self.device)

    @staticmethod
    def _address(x):
        return None if x is None else x.data_ptr()

    @staticmethod
    def _span(x):
        if x.numel() == 0:
            return 0, 0
        last = sum((n - 1) * s for n, s in zip(x.shape, x.stride()))
        return x.data_ptr(), x.data_ptr() + (last + 1) * x.element_size()
