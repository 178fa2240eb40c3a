"""Training entry points of include/hcnn.h as methods; array handling is supplied by a subclass.

A subclass provides
    _matrix(x, what)            (address, rows, columns, row stride in numbers, type code) of a 2-D array whose rows' numbers lie side by side
    _vector(x, what)            (address, length, type code) of a 1-D array without gaps
    _targets(x, what)           (address, length, bytes of a number) of a 1-D int32 or int64 array without gaps
    _new(shape, like)           new uninitialised array of the type and place of `like` (None: 32-bit floats)
    _span(x)                    (first byte, one past the last) of the array's memory
    _bytes(x, what)             (address, shape, strides) of a 2-D array of bytes
    _room(x)                    bytes from its first to the end of the memory it is a view of
    _new_bytes(rows, cols, of)  the first `of` columns of a new uninitialised 2-D array of bytes
    _new_of(shape, dtype)       (new uninitialised array of the type, the type's code)
Marshalling and checks only: no arithmetic of the method happens here.
"""
import ctypes as C

from . import _capi


class Microscaled:
    """A matrix of `columns` numbers a row in a microscaled format, "mx4" or "mx8" (hcnn_quantize_mx): codes [rows][bytes of a row], the rows' numbers with zeros up
    to whole 128, and scales [blocks of 32][rows], the exponents' bytes; in the memory of scales a block's bytes begin a multiple of 64 behind the last one's."""

    __slots__ = ("codes", "scales", "columns", "format")

    def __init__(self, codes, scales, columns, format):
        if format not in _capi.MX_BITS:
            raise ValueError("format must be one of %s, got %r" % (", ".join(_capi.MX_BITS), format))
        self.codes, self.scales, self.columns, self.format = codes, scales, int(columns), format

    @property
    def shape(self):
        return self.codes.shape[0], self.columns


class PlainOpsMixin:
    raw: _capi.RawPlain

    def close(self):
        self.raw.close()

    def _pre_call(self):
        """Hook run before every library call that enqueues work (the device binding checks the stream here)."""

    def _activation(self, name):
        if name not in _capi.ACTIVATIONS:
            raise ValueError("activation must be one of %s, got %r" % (", ".join(_capi.ACTIVATIONS), name))
        return _capi.ACTIVATIONS[name]

    def _like(self, x, shape, dtype, what, lead=None):
        """_matrix of x, which must have that shape and type."""
        got = self._matrix(x, what)
        if got[1:3] != shape:
            raise ValueError("%s must have shape %r, got %r" % (what, shape, got[1:3]))
        if got[4] != dtype:
            raise TypeError("%s must have the type of x" % what)
        return got

    def _output(self, x, shape, dtype, what, *inputs):
        """An output that the caller gave: shape, type, rows that do not overlap, no memory shared with the inputs.  (A single row has no
        next one: whatever its stride, the library is told its length.)"""
        got = self._like(x, shape, dtype, what)
        if got[1] > 1 and got[3] < got[2]:
            raise ValueError("the rows of %s must not overlap" % what)
        self._apart(x, what, *inputs)
        return got if got[1] > 1 else (*got[:3], max(got[2:4]), got[4])

    def _apart(self, x, what, *inputs):
        a0, a1 = self._span(x)
        for y in inputs:
            if y is None:
                continue
            b0, b1 = self._span(y)
            if a0 < b1 and b0 < a1 and not (y.ndim == 2 and self._other_columns(x, y)):
                raise ValueError("%s must not overlap an input" % what)

    def _other_columns(self, x, y):
        """Do the rows of two matrices of one type, whose memory interleaves, lie beside each other: other columns of one array?"""
        xp, x_rows, x_cols, x_pitch, dtype = self._matrix(x, "x")
        yp, y_rows, y_cols, y_pitch, _ = self._matrix(y, "y")
        if y_rows == 1:
            y_pitch = x_pitch
        if x_rows == 1:
            x_pitch = y_pitch
        if x_pitch != y_pitch or x_pitch <= 0:
            return False
        size = _capi.SIZES[dtype]
        behind = (yp - xp) % (x_pitch * size)                  # of a row of y, from the row of x in front of it
        return behind >= x_cols * size and behind + y_cols * size <= x_pitch * size

    # ---- layers
    def linear(self, x, w, bias=None, residual=None, activation="none", keep=False, out=None):
        """y = act(x w^T + bias) + residual (hcnn_linear).  x [rows][n_in], w [n_out][n_in], bias [n_out], residual
        [rows][n_out]; rows may have any stride (broadcast rows included).  With keep returns (y, z), z = x w^T + bias:
        what linear_grad takes.  out: where y goes (the residual's own memory allowed)."""
        xp, rows, n_in, ldx, dtype = self._matrix(x, "x")
        wp, n_out, w_in, ldw, w_dtype = self._matrix(w, "w")
        if w_in != n_in:
            raise ValueError("w must have shape (n_out, %d), got %r" % (n_in, (n_out, w_in)))
        if w_dtype != dtype:
            raise TypeError("w must have the type of x")
        bp = rp = None
        ldr = 0
        if bias is not None:
            bp = self._bias(bias, n_out, dtype)
        if residual is not None:
            rp, _, _, ldr, _ = self._like(residual, (rows, n_out), dtype, "residual")
        if out is None:
            y = self._new((rows, n_out), x)
            yp, ldy = self._address(y), n_out
        else:
            y = out
            yp, _, _, ldy, _ = self._output(y, (rows, n_out), dtype, "out", x, w, bias)
            if residual is not None and not (yp == rp and (ldy == ldr or rows == 1)):
                self._apart(y, "out", residual)
        zp, z = None, None
        if keep:
            z = self._new((rows, n_out), x)
            zp = self._address(z)
        self._pre_call()
        self.raw.call("hcnn_linear", dtype, self._activation(activation), rows, n_in, n_out, xp, ldx, wp, ldw, bp, rp, ldr, yp, ldy, zp, n_out)
        return (y, z) if keep else y

    def _bias(self, bias, n_out, dtype, what="bias"):
        bp, n, b_dtype = self._vector(bias, what)
        if n != n_out:
            raise ValueError("%s must have shape (%d,), got (%d,)" % (what, n_out, n))
        if b_dtype != dtype:
            raise TypeError("%s must have the type of x" % what)
        return bp

    def linear_grad(self, dy, x, w, z=None, activation="none", bias=False, need_dx=True, need_dw=True):
        """(dx, dw, db) of linear for dy [rows][n_out] (hcnn_linear_grad): dz = dy * act'(z), dx = dz w, dw = dz^T x, db = the
        columns' sums of dz (None unless bias).  z: what linear returned with keep, needed unless the activation is "none".
        need_dx, need_dw False: None in the place of that gradient.  The residual's gradient is dy."""
        xp, rows, n_in, ldx, dtype = self._matrix(x, "x")
        wp, n_out, w_in, ldw, w_dtype = self._matrix(w, "w")
        if w_in != n_in:
            raise ValueError("w must have shape (n_out, %d), got %r" % (n_in, (n_out, w_in)))
        if w_dtype != dtype:
            raise TypeError("w must have the type of x")
        dyp, _, _, ld_dy, _ = self._like(dy, (rows, n_out), dtype, "dy")
        act = self._activation(activation)
        zp, ldz = None, 0
        if act:
            if z is None:
                raise ValueError("z is required with activation %r" % activation)
            zp, _, _, ldz, _ = self._like(z, (rows, n_out), dtype, "z")
        dx = self._new((rows, n_in), x) if need_dx else None
        dw = self._new((n_out, n_in), x) if need_dw else None
        db = self._new((n_out,), x) if bias else None
        self._pre_call()
        self.raw.call("hcnn_linear_grad", dtype, act, rows, n_in, n_out, dyp, ld_dy, xp, ldx, wp, ldw, zp, ldz,
                      self._address(dx), n_in, self._address(dw), n_in, self._address(db))
        return dx, dw, db

    # ---- loss
    def _loss_inputs(self, x, w, targets):
        xp, rows, n_in, ldx, dtype = self._matrix(x, "x")
        wp, n_classes, w_in, ldw, w_dtype = self._matrix(w, "w")
        if w_in != n_in:
            raise ValueError("w must have shape (n_classes, %d), got %r" % (n_in, (n_classes, w_in)))
        if w_dtype != dtype:
            raise TypeError("w must have the type of x")
        if n_classes == 0:
            raise ValueError("w must have a row for each class")
        tp, n, size = self._targets(targets, "targets")
        if n != rows:
            raise ValueError("targets must have shape (%d,), got (%d,)" % (rows, n))
        return (dtype, rows, n_in, n_classes, xp, ldx, wp, ldw, tp, size)

    def cross_entropy(self, x, w, targets, ignore_index=-100, rows=False):
        """Mean softmax cross entropy of the scores x w^T (x [rows][n_in], w [n_classes][n_in], targets [rows] int32 or int64), as one
        32-bit float (hcnn_cross_entropy).  Rows whose target is ignore_index take no part and may hold anything; without any
        other row the loss is 0.  With rows=True returns (loss, each row's loss, each row's log sum of exponentials).  A target that is
        neither a class nor ignore_index is taken as ignored and counted in bad_inputs()."""
        args = self._loss_inputs(x, w, targets)
        loss = self._new((), None)
        row_loss = self._new((args[1],), None) if rows else None
        row_lse = self._new((args[1],), None) if rows else None
        self._pre_call()
        self.raw.call("hcnn_cross_entropy", *args, int(ignore_index), self._address(row_loss), self._address(row_lse), self._address(loss))
        return (loss, row_loss, row_lse) if rows else loss

    def cross_entropy_grad(self, x, w, targets, ignore_index=-100, scale=1.0, need_dx=True, need_dw=True):
        """(loss, dx, dw): cross_entropy's mean loss and the gradients of scale * loss (hcnn_cross_entropy_grad).  The scores are
        formed in pieces of the classes and never stored.  need_dx, need_dw False: None in the place of that gradient."""
        args = self._loss_inputs(x, w, targets)
        _, n_rows, n_in, n_classes = args[:4]
        loss = self._new((), None)
        dx = self._new((n_rows, n_in), x) if need_dx else None
        dw = self._new((n_classes, n_in), x) if need_dw else None
        self._pre_call()
        self.raw.call("hcnn_cross_entropy_grad", *args, int(ignore_index), float(scale), None, self._address(loss), self._address(dx), n_in,
                      self._address(dw), n_in)
        return loss, dx, dw

    # ---- between the layers
    def dropout(self, x, p, seed, stream=0, residual=None, out=None):
        """residual + (x / (1 - p) where it is kept, else 0) (hcnn_dropout).  What is kept is a function of (seed, stream, row, column) alone: no mask is
        stored, dropout_grad forms it again.  stream: below 2^32, another one for every layer and step that must not share a mask.  out: where the
        result goes (the memory of x or of the residual allowed)."""
        xp, rows, n, ldx, dtype = self._matrix(x, "x")
        p, seed, stream = float(p), int(seed), int(stream)
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie between 0 and 1")
        if not 0 <= seed < 1 << 64 or not 0 <= stream < 1 << 32:
            raise ValueError("seed must lie between 0 and 2^64 - 1, stream between 0 and 2^32 - 1")
        rp, ldr = None, 0
        if residual is not None:
            rp, _, _, ldr, _ = self._like(residual, (rows, n), dtype, "residual")
        if out is None:
            y = self._new((rows, n), x)
            yp, ldy = self._address(y), n
        else:
            y = out
            yp, _, _, ldy, _ = self._output(y, (rows, n), dtype, "out")
            for other, at, ld in ((x, xp, ldx), (residual, rp, ldr)):
                if other is not None and not (yp == at and (ldy == ld or rows == 1)):
                    self._apart(y, "out", other)
        self._pre_call()
        self.raw.call("hcnn_dropout", dtype, rows, n, xp, ldx, rp, ldr, p, seed, stream, yp, ldy)
        return y

    def dropout_grad(self, dy, p, seed, stream=0, out=None):
        """Gradient of dropout for x: dy / (1 - p) where x was kept, else 0.  The residual's is dy."""
        return self.dropout(dy, p, seed, stream, out=out)

    def rms_norm(self, x, weight=None, residual=None, eps=1e-6, keep=False, format=None):
        """s / sqrt(mean of s^2 over the row + eps) * weight, s = x + residual (hcnn_rms_norm).  x, residual [rows][n], weight [n]; rows may have any stride.
        With keep returns (y, s): what the next layers add to and rms_norm_grad takes.  format "mx8": y is a Microscaled matrix, what linear_mx takes."""
        xp, rows, n, ldx, dtype = self._matrix(x, "x")
        rp = wp = sp = yp = None
        ldr = pitch = 0
        if residual is not None:
            rp, _, _, ldr, _ = self._like(residual, (rows, n), dtype, "residual")
        if weight is not None:
            wp = self._bias(weight, n, dtype, "weight")
        if format not in (None, "mx8"):
            raise ValueError("format must be None or 'mx8', got %r" % (format,))
        self._eps(eps)
        s, codes, scales = None, None, None
        if keep:
            s = self._new((rows, n), x)
            sp = self._address(s)
        if format is None:
            y = self._new((rows, n), x)
            yp = self._address(y)
        else:
            y, codes, scales, pitch = self._new_microscaled(rows, n, format)
        self._pre_call()
        self.raw.call("hcnn_rms_norm", dtype, rows, n, xp, ldx, rp, ldr, wp, float(eps), sp, n, yp, n, codes, scales, pitch)
        return (y, s) if keep else y

    def rms_norm_grad(self, dy, s, weight=None, ds=None, eps=1e-6, need_dweight=True):
        """(dx, dweight) of rms_norm for dy [rows][n] at the sums s that it returned with keep (hcnn_rms_norm_grad); ds [rows][n]: the gradient that reaches
        s by other ways, added.  dx is the gradient for x and for the residual.  dweight is None without a weight or need_dweight."""
        sp, rows, n, lds, dtype = self._matrix(s, "s")
        dyp, _, _, ld_dy, _ = self._like(dy, (rows, n), dtype, "dy")
        wp = dsp = None
        ld_ds = 0
        if weight is not None:
            wp = self._bias(weight, n, dtype, "weight")
        if ds is not None:
            dsp, _, _, ld_ds, _ = self._like(ds, (rows, n), dtype, "ds")
        self._eps(eps)
        dx = self._new((rows, n), s)
        dw = self._new((n,), s) if weight is not None and need_dweight else None
        self._pre_call()
        self.raw.call("hcnn_rms_norm_grad", dtype, rows, n, dyp, ld_dy, sp, lds, wp, dsp, ld_ds, float(eps), self._address(dx), n, self._address(dw))
        return dx, dw

    @staticmethod
    def _eps(eps):
        if not 2.0 ** -126 <= eps <= 3e38:
            raise ValueError("eps must be a positive number that 32 bits hold")

    # ---- few bits
    def _new_microscaled(self, rows, n, format):
        """(new Microscaled matrix, its codes' address, its scales', their pitch)"""
        wide, pitch = -(-n // 128) * 128, -(-rows // 64) * 64
        row_bytes = wide // 8 * _capi.MX_BITS[format]
        codes, scales = self._new_bytes(rows, row_bytes, row_bytes), self._new_bytes(wide // 32, pitch, rows)
        return Microscaled(codes, scales, n, format), self._address(codes), self._address(scales), pitch

    def _microscaled(self, m, what):
        """(codes' address, rows, scales' address, their pitch) of a Microscaled matrix whose arrays are what its format says"""
        if not isinstance(m, Microscaled):
            raise TypeError("%s must be a Microscaled matrix" % what)
        if m.columns < 0:
            raise ValueError("%s must have columns" % what)
        wide = -(-m.columns // 128) * 128
        row_bytes = wide // 8 * _capi.MX_BITS[m.format]
        cp, (rows, got), strides = self._bytes(m.codes, what)
        if got != row_bytes or (rows and got and strides[1] != 1) or (rows > 1 and got and strides[0] != got):
            raise ValueError("the codes of %s must be a contiguous array of shape (rows, %d)" % (what, row_bytes))
        sp, shape, strides = self._bytes(m.scales, what)
        if shape != (wide // 32, rows):
            raise ValueError("the scales of %s must have shape %r, got %r" % (what, (wide // 32, rows), shape))
        if not rows or not wide:
            return cp, rows, sp, -(-rows // 64) * 64
        pitch = strides[0]
        if (rows > 1 and strides[1] != 1) or pitch % 64 or pitch < rows:
            raise ValueError("the scales of %s must be the first bytes of rows that lie a multiple of 64 bytes apart" % what)
        if pitch != rows and self._room(m.scales) < wide // 32 * pitch:
            raise ValueError("the memory of the scales of %s must reach to the end of their last row's %d bytes" % (what, pitch))
        if cp % 16 or sp % 16:
            raise ValueError("codes and scales of %s must start on 16 bytes" % what)
        return cp, rows, sp, pitch

    def quantize_mx(self, x, format="mx4", values=False):
        """x [rows][n] as a Microscaled matrix (hcnn_quantize_mx); with values returns (matrix, the numbers that it stands for, in the type of x)."""
        xp, rows, n, ldx, dtype = self._matrix(x, "x")
        if format not in _capi.MX_BITS:
            raise ValueError("format must be one of %s, got %r" % (", ".join(_capi.MX_BITS), format))
        m, cp, sp, pitch = self._new_microscaled(rows, n, format)
        v = self._new((rows, n), x) if values else None
        self._pre_call()
        self.raw.call("hcnn_quantize_mx", dtype, _capi.MX_BITS[format], rows, n, xp, ldx, cp, sp, pitch, self._address(v), n)
        return (m, v) if values else m

    def linear_mx(self, x, w, bias=None, residual=None, activation="none", dtype=None, out=None):
        """act(x w^T + bias) + residual of Microscaled matrices x [rows][n_in] ("mx4" or "mx8") and w [n_out][n_in] ("mx4") (hcnn_linear_mx).  The result, bias and
        residual are of one type: dtype, or that of out, residual or bias.  out: where the result goes (the residual's own memory allowed)."""
        xc, rows, xs, x_pitch = self._microscaled(x, "x")
        wc, n_out, ws, w_pitch = self._microscaled(w, "w")
        n_in = x.columns
        if w.format != "mx4":
            raise ValueError("w must be of the format 'mx4', got %r" % w.format)
        if w.columns != n_in:
            raise ValueError("w must have shape (n_out, %d), got %r" % (n_in, (n_out, w.columns)))
        if dtype is None:
            given = [a for a in (out, residual, bias) if a is not None]
            if not given:
                raise ValueError("dtype is required without out, residual and bias")
            dtype = given[0].dtype
        y, code = (out, None) if out is not None else self._new_of((rows, n_out), dtype)
        if out is not None:
            code = self._matrix(out, "out")[4]
            if out.dtype != dtype:
                raise TypeError("out must have the type dtype")
        bp = rp = None
        ldr = 0
        if bias is not None:
            bp = self._bias(bias, n_out, code)
        if residual is not None:
            rp, _, _, ldr, _ = self._like(residual, (rows, n_out), code, "residual")
        if out is None:
            yp, ldy = self._address(y), n_out
        else:
            yp, _, _, ldy, _ = self._output(y, (rows, n_out), code, "out", bias)
            spans = [self._span(y)] + [self._span(a) for a in (x.codes, x.scales, w.codes, w.scales)]
            if any(spans[0][0] < b and a < spans[0][1] for a, b in spans[1:]):
                raise ValueError("out must not overlap an input")
            if residual is not None and not (yp == rp and (ldy == ldr or rows == 1)):
                self._apart(y, "out", residual)
        self._pre_call()
        self.raw.call("hcnn_linear_mx", code, _capi.MX_BITS[x.format], self._activation(activation), rows, n_in, n_out, xc, xs, x_pitch, wc, ws, w_pitch,
                      bp, rp, ldr, yp, ldy)
        return y

    # ---- step
    def clip_grad_norm(self, grads, max_norm, out=None, eps=1e-6):
        """Euclidean norm over all numbers of the list `grads` (contiguous arrays of any shapes, types mixed), as one 32-bit float; every
        array is scaled by min(1, max_norm / (norm + eps)), in place or into the arrays of `out` (hcnn_clip_grad_norm).  What is written
        must not overlap anything else of the list: a tensor that shares its numbers with another is named once."""
        grads = list(grads)
        if not max_norm >= 0 or not eps >= 0:
            raise ValueError("max_norm and eps must not be negative")
        n = len(grads)
        flat = [self._flat(g, "grads") for g in grads]
        ptrs = (C.c_void_p * n)(*[f[0] for f in flat])
        counts = (C.c_size_t * n)(*[f[1] for f in flat])
        types = (C.c_int * n)(*[f[2] for f in flat])
        outs, to = None, flat
        if out is not None:
            out = list(out)
            to = [self._flat(g, "out") for g in out]
            if [t[1:] for t in to] != [f[1:] for f in flat]:
                raise ValueError("out must match grads in number, sizes and types")
            outs = (C.c_void_p * n)(*[t[0] for t in to])
        self._clip_apart(flat, to)
        norm = self._new((), None)
        self._pre_call()
        self.raw.call("hcnn_clip_grad_norm", n, ptrs, counts, types, outs, float(max_norm), float(eps), self._address(norm))
        return norm

    def _clip_apart(self, flat, to):
        """No result may overlap a gradient other than its own, which it may replace, nor another result."""
        spans = []                             # (first byte, one past the last, written)
        for f, t in zip(flat, to):
            if f[1]:
                n = f[1] * _capi.SIZES[f[2]]
                spans.append((f[0], f[0] + n, f[0] == t[0]))
                if f[0] != t[0]:
                    spans.append((t[0], t[0] + n, True))
        spans.sort()
        end = written = 0                      # the furthest byte so far, of all and of what is written
        for first, last, writes in spans:
            if first < (end if writes else written):
                raise ValueError("a tensor that is written must not overlap another one of the list")
            end = max(end, last)
            if writes:
                written = max(written, last)

    # ---- diagnostics
    def bad_inputs(self):
        return self.raw.stat(_capi.STAT_BAD_INPUT)

    def scratch_bytes(self):
        return self.raw.stat(_capi.STAT_SCRATCH_BYTES)
