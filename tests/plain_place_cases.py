"""The norm and its gradient in the memory of their inputs, through the C entry points, shared by the CPU checker's tests and the device's (test helper, not collected)."""
import numpy as np

import plain_cases as pc
from paper_1811_00778_amd import _capi

CODE = {"f32": _capi.F32, "f16": _capi.F16, "bf16": _capi.BF16}
# columns: rows in the registers of each shape's threads, and longer ones
SIZES = [(3, 5), (5, 77), (70, 150), (2, 1031), (3, 5000), (2, 16384), (2, 16400), (3, 17001)]


def _inputs(b, dtype, rows, n, count):
    rng = np.random.default_rng([rows, n, 31])
    return [pc.normal(rng, rows, n) for _ in range(count)], b.make(1 + 0.2 * pc.normal(rng, n), dtype)


def _call(b, name, dtype, rows, n, *rest):
    at = [a if a is None or isinstance(a, (int, float)) else b.ctx._address(a) for a in rest]
    b.ctx.raw.call(name, CODE[dtype], rows, n, *at)


def check_norm(b, dtype, rows, n):
    """the sum in the residual's or x's memory, y in the other's: what arrays of their own take"""
    (x, r), w = _inputs(b, dtype, rows, n, 2)
    new = lambda v: b.make(v, dtype)                                                    # noqa: E731
    want, s = b.ctx.rms_norm(new(x), w, new(r), keep=True)
    want, s = b.values(want), b.values(s)
    for to_sum, to_y in (("r", None), ("x", None), ("r", "x"), ("x", "r"), (None, "x"), (None, "r")):
        at = {"x": new(x), "r": new(r)}
        sums, y = (at[k] if k else new(np.zeros((rows, n))) for k in (to_sum, to_y))
        _call(b, "hcnn_rms_norm", dtype, rows, n, at["x"], n, at["r"], n, w, 1e-6, sums, n, y, n, None, None, 0)
        assert np.array_equal(b.values(y), want) and np.array_equal(b.values(sums), s), (to_sum, to_y)
    m = b.ctx.rms_norm(new(x), w, new(r), format="mx8")
    codes, scales = b.raw(m.codes).copy(), b.raw(m.scales).copy()
    for to_sum in ("x", "r"):
        at = {"x": new(x), "r": new(r)}
        got, cp, sp, pitch = b.ctx._new_microscaled(rows, n, "mx8")
        _call(b, "hcnn_rms_norm", dtype, rows, n, at["x"], n, at["r"], n, w, 1e-6, at[to_sum], n, None, 0, cp, sp, pitch)
        assert np.array_equal(b.values(at[to_sum]), s), to_sum
        assert np.array_equal(b.raw(got.codes), codes) and np.array_equal(b.raw(got.scales), scales), to_sum


def check_norm_grad(b, dtype, rows, n):
    """dx in the memory of ds"""
    (dy, s, ds), w = _inputs(b, dtype, rows, n, 3)
    dy, s = b.make(dy, dtype), b.make(s, dtype)
    dx, dw = (b.values(v) for v in b.ctx.rms_norm_grad(dy, s, w, b.make(ds, dtype)))
    place, got = b.make(ds, dtype), b.make(np.zeros(n), dtype)
    _call(b, "hcnn_rms_norm_grad", dtype, rows, n, dy, n, s, n, w, place, n, 1e-6, place, n, got)
    assert np.array_equal(b.values(place), dx) and np.array_equal(b.values(got), dw)
