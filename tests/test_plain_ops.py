"""The training operators on the CPU checker of the kernel sources: values against 64-bit definitions, gradients against
differences, refusals.  (The device's tests run the same cases at its sizes.)"""
import ctypes

import numpy as np
import pytest

import emu
import plain_cases as pc
from paper_1811_00778_amd import _capi
from paper_1811_00778_amd._plain_ops import PlainOpsMixin

_NP = {"f32": np.float32, "f16": np.float16, "bf16": np.uint16}
_CODE = {np.dtype(np.float32): _capi.F32, np.dtype(np.float16): _capi.F16, np.dtype(np.uint16): _capi.BF16}


def to_bf16(a):
    b = np.asarray(a, np.float32).view(np.uint32)
    r = ((b + 0x7fff + (b >> 16 & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(a), np.uint16(0x7fc0), r)


class EmuPlain(PlainOpsMixin):
    """numpy arrays; bfloat16 numbers as uint16"""

    def __init__(self):
        self.raw = _capi.RawPlain(emu.lib())

    def _matrix(self, x, what):
        if not isinstance(x, np.ndarray) or x.dtype not in _CODE or x.ndim != 2:
            raise TypeError("%s must be a 2-D array" % what)
        if x.size and x.shape[1] > 1 and x.strides[1] != x.itemsize:
            raise TypeError("the numbers of a row of %s must lie side by side" % what)
        return x.ctypes.data, x.shape[0], x.shape[1], x.strides[0] // x.itemsize, _CODE[x.dtype]

    def _flat(self, x, what):
        if not isinstance(x, np.ndarray) or x.dtype not in _CODE or not x.flags["C_CONTIGUOUS"]:
            raise TypeError("%s must be contiguous" % what)
        return x.ctypes.data, x.size, _CODE[x.dtype]

    def _vector(self, x, what):
        return self._flat(x, what)

    def _targets(self, x, what):
        if x.dtype not in (np.int32, np.int64) or x.ndim != 1:
            raise TypeError("%s must be a 1-D int32 or int64 array" % what)
        return x.ctypes.data, x.size, x.itemsize

    def _new(self, shape, like):
        a = np.empty(shape, np.float32 if like is None else like.dtype)
        a.reshape(-1).view(np.uint8).fill(0xff)                    # NaN in every type
        return a

    @staticmethod
    def _address(x):
        return None if x is None else x.ctypes.data

    @staticmethod
    def _span(x):
        if not x.size:
            return 0, 0
        return np.lib.array_utils.byte_bounds(x)


class Backend:
    def __init__(self):
        self.ctx = EmuPlain()

    def make(self, a, dtype, strides=None):
        """a in the type; with strides = (gap, shift) inside a larger array: rows `gap` numbers apart, `shift` numbers in, NaN around"""
        v = to_bf16(a) if dtype == "bf16" else np.asarray(a, np.float32).astype(_NP[dtype])
        if strides is None or v.ndim != 2:
            return np.ascontiguousarray(v)
        gap, shift = strides
        big = np.full(shift + v.shape[0] * (v.shape[1] + gap), 0x7fc0 if dtype == "bf16" else np.nan, v.dtype)
        view = np.lib.stride_tricks.as_strided(big[shift:], v.shape, ((v.shape[1] + gap) * v.itemsize, v.itemsize))
        view[...] = v
        return view

    def ints(self, a, dtype):
        return np.ascontiguousarray(a, dtype)

    def values(self, a):
        if a.dtype == np.uint16:
            a = (a.astype(np.uint32) << 16).view(np.float32)
        return a.astype(np.float64)


@pytest.fixture(scope="module", params=[1, 256], ids=["one-unit", "256-units"])
def b(request):
    """Handles made for a device of one compute unit (the largest tiles) and of 256 (the smallest, long sums in parts)."""
    with emu.device(emu.lib(), units=request.param):
        yield Backend()


@pytest.mark.parametrize("case", pc.LINEAR, ids=str)
def test_linear(b, case):
    pc.check_linear(b, *case)


@pytest.mark.parametrize("case", pc.GRAD, ids=str)
def test_linear_grad(b, case):
    pc.check_grad(b, *case)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strides_and_alignment(b, dtype):
    """rows further apart than their length, starts that are aligned to one number only; what lies between must not be seen"""
    pc.check_linear(b, dtype, 37, 41, 19, "silu", residual=True, keep=True, strides=(3, 1))
    pc.check_grad(b, dtype, 37, 41, 19, "square", bias=True, strides=(3, 1))
    pc.check_loss(b, dtype, 37, 41, 19, 0.3, strides=(3, 1))


def test_broadcast_rows(b):
    """one row for all: the gradient of a sum"""
    one = b.make(np.ones((1, 9)), "f32")
    pc.check_grad(b, "f32", 21, 12, 9, "none", bias=True, dy=np.broadcast_to(one, (21, 9)))


@pytest.mark.parametrize("case", pc.LOSS, ids=str)
def test_cross_entropy(b, case):
    pc.check_loss(b, *case)
    pc.check_loss(b, *case, wide=False, seed=1, junk=case[3] < 1000 and case[4] > 0)


def test_large_scores(b):
    """scores in the hundreds: their exponentials leave the range, their differences do not"""
    pc.check_loss(b, "f32", 40, 30, 50, 0.2, std=100.0)


def test_bad_targets_are_ignored_and_counted(b):
    x, w, t = pc.loss_inputs(b, "f32", 12, 5, 7)
    bad = t.copy()
    bad[[2, 5, 11]] = [7, -1, 2 ** 40]
    good = t.copy()
    good[[2, 5, 11]] = pc.IGNORE
    before = b.ctx.bad_inputs()
    got = b.ctx.cross_entropy_grad(x, w, bad)
    assert b.ctx.bad_inputs() == before + 3
    for u, v in zip(got, b.ctx.cross_entropy_grad(x, w, good)):
        assert np.array_equal(u, v)
    assert b.ctx.bad_inputs() == before + 3


@pytest.mark.parametrize("where", ["new", "place"])
@pytest.mark.parametrize("share", [0.3, 2.0])
def test_clip(b, where, share):
    pc.check_clip(b, ["f32"], [1], share, where)
    pc.check_clip(b, ["f32", "bf16", "f16"], [125, 16385, 3], share, where)
    pc.check_clip(b, ["bf16", "f16", "f32"] * 67, [(7 * i) % 40 for i in range(201)], share, where)
    pc.check_clip(b, ["f32", "f32"], [40, 50], share, where, std=1e25)          # squares beyond 32 bits
    pc.check_clip(b, ["f32", "f32"], [40, 50], share, where, std=1e-30)


def test_clip_of_nothing_and_of_what_is_not_finite(b):
    assert b.values(b.ctx.clip_grad_norm([], 1.0)) == 0.0
    assert b.values(b.ctx.clip_grad_norm([b.make(np.zeros(0), "f32")], 1.0)) == 0.0
    g = b.make(np.array([1.0, np.inf, 2.0]), "f32")
    assert b.values(b.ctx.clip_grad_norm([g], 1.0)) == np.inf
    assert g[0] == 0 and np.isnan(g[1])
    g = b.make(np.array([1.0, np.nan]), "f32")
    assert np.isnan(b.values(b.ctx.clip_grad_norm([g], 1.0)))
    assert np.isnan(g).all()


@pytest.mark.parametrize("name", ["none", "square", "gelu", "silu"])
def test_gradients_are_the_differences(b, name):
    """linear_grad against central differences of linear: d(sum(y * dy)) along random directions of x, w and the bias"""
    rng = np.random.default_rng(5)
    M, K, N, h = 9, 14, 6, 2.0 ** -6
    x, w, bias, dy = (rng.standard_normal(s) for s in ((M, K), (N, K), (N,), (M, N)))

    def value(x, w, bias):
        z = x @ w.T + bias
        return (pc.act(z, name)[0] * dy).sum()

    f = lambda a: b.make(a, "f32")  # noqa: E731
    y, z = b.ctx.linear(f(x), f(w), f(bias), activation=name, keep=True)
    dx, dw, db = (b.values(v) for v in b.ctx.linear_grad(f(dy), f(x), f(w), z, activation=name, bias=True))
    for _ in range(4):
        ux, uw, ub = (rng.standard_normal(a.shape) for a in (x, w, bias))
        ux, uw, ub = (u / np.linalg.norm(u) for u in (ux, uw, ub))
        slope = (dx * ux).sum() + (dw * uw).sum() + (db * ub).sum()
        # fourth-order differences: their error is h^4 / 30 times a fifth derivative, below 1e-9 x 1e3 here; 32-bit values leave 1e-4
        at = [value(x + s * h * ux, w + s * h * uw, bias + s * h * ub) for s in (-2, -1, 1, 2)]
        assert abs(slope - (at[0] - 8 * at[1] + 8 * at[2] - at[3]) / (12 * h)) < 2e-4 * (1 + np.abs(dx).max() + np.abs(dw).max())


def test_loss_gradient_is_the_difference(b):
    rng = np.random.default_rng(6)
    x, w, t = pc.loss_inputs(b, "f32", 15, 8, 11, 0.3)
    _, dx, dw = b.ctx.cross_entropy_grad(x, w, b.ints(t, np.int64))
    X, W, h = b.values(x), b.values(w), 2.0 ** -6
    for _ in range(4):
        ux, uw = rng.standard_normal(X.shape), rng.standard_normal(W.shape)
        ux, uw = ux / np.linalg.norm(ux), uw / np.linalg.norm(uw)
        at = [pc.loss_exact(X + s * h * ux, W + s * h * uw, t)[0] for s in (-2, -1, 1, 2)]
        assert abs((b.values(dx) * ux).sum() + (b.values(dw) * uw).sum() - (at[0] - 8 * at[1] + 8 * at[2] - at[3]) / (12 * h)) < 1e-5


def test_outputs_given_by_the_caller(b):
    rng = np.random.default_rng(7)
    x, w, r = (b.make(pc.normal(rng, *s), "f32") for s in ((9, 5), (4, 5), (9, 4)))
    want = b.ctx.linear(x, w, residual=r)
    got = b.ctx.linear(x, w, residual=r, out=r)                    # in the residual's place
    assert got is r and np.array_equal(r, want)
    wide = np.full((9, 7), 5.0, np.float32)
    b.ctx.linear(x, w, out=wide[:, 1:5])
    assert (wide[:, [0, 5, 6]] == 5).all() and np.array_equal(wide[:, 1:5], b.ctx.linear(x, w))


def test_refusals(b):
    f = lambda *s: b.make(np.ones(s), "f32")  # noqa: E731
    x, w, t = f(6, 5), f(4, 5), np.zeros(6, np.int64)
    for bad in (lambda: b.ctx.linear(x, f(4, 6)), lambda: b.ctx.linear(x, w, f(5)), lambda: b.ctx.linear(x, w, residual=f(6, 5)),
                lambda: b.ctx.linear(x, w, activation="tanh"), lambda: b.ctx.linear(x, w, out=f(5, 4)),
                lambda: b.ctx.linear(x, f(5, 5), out=x), lambda: b.ctx.linear(x, w, out=np.broadcast_to(f(1, 4), (6, 4))),
                lambda: b.ctx.linear_grad(f(6, 5), x, w), lambda: b.ctx.linear_grad(f(6, 4), x, w, activation="square"),
                lambda: b.ctx.linear_grad(f(6, 4), x, w, f(6, 3), activation="square"), lambda: b.ctx.cross_entropy(x, w, t[:5]),
                lambda: b.ctx.cross_entropy(x, f(0, 5), t), lambda: b.ctx.cross_entropy_grad(x, f(4, 3), t),
                lambda: b.ctx.clip_grad_norm([x], -1.0), lambda: b.ctx.clip_grad_norm([x], float("nan")),
                lambda: b.ctx.clip_grad_norm([x], 1.0, out=[w]), lambda: b.ctx.clip_grad_norm([x], 1.0, out=[]),
                lambda: b.ctx.clip_grad_norm([x[:4], x[4:]], 1.0, out=[x[2:], x[:2]])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: b.ctx.linear(x, b.make(np.ones((4, 5)), "f16")), lambda: b.ctx.linear(x.T, w), lambda: b.ctx.linear(x[0], w),
                lambda: b.ctx.cross_entropy(x, w, t.astype(np.int16)), lambda: b.ctx.clip_grad_norm([x.T], 1.0),
                lambda: b.ctx.linear(x, w, b.make(np.ones(4), "bf16"))):
        with pytest.raises(TypeError):
            bad()


def test_codes_of_the_c_entry_points():
    lib, err = emu.lib(), _capi.ERR
    raw = _capi.RawPlain(lib)
    h, p, z = raw.handle, ctypes.c_void_p(4096), ctypes.c_void_p(0)

    def lin(h=h, dtype=0, act=0, m=2, k=2, n=2, x=p, w=p, b=z, y=p, ldy=2, zz=z):
        return lib.hcnn_linear(h, dtype, act, m, k, n, x, 2, w, 2, b, z, 2, y, ldy, zz, 2)

    assert lin(h=None) == err["NULL"] and lin(x=z) == err["NULL"] and lin(y=z) == err["NULL"]
    assert lin(dtype=3) == err["ARG"] and lin(act=5) == err["ARG"] and lin(act=-1) == err["ARG"]
    assert lin(m=2 ** 31) == err["ARG"] and lin(ldy=1) == err["ARG"]
    assert lin(x=ctypes.c_void_p(4098)) == err["ALIGN"] and lin(dtype=1, w=ctypes.c_void_p(4097)) == err["ALIGN"]
    assert lin(m=0, x=z, w=z, y=z) == 0

    def grad(h=h, dtype=0, act=0, dy=p, x=p, w=p, zz=z, dx=p, dw=p, ld=2):
        return lib.hcnn_linear_grad(h, dtype, act, 2, 2, 2, dy, 2, x, 2, w, 2, zz, 2, dx, ld, dw, ld, z)

    assert grad(h=None) == err["NULL"] and grad(dy=z) == err["NULL"] and grad(act=1) == err["NULL"] and grad(x=z) == err["NULL"]
    assert grad(w=z) == err["NULL"] and grad(ld=1) == err["ARG"] and grad(dtype=-1) == err["ARG"]
    assert grad(dx=ctypes.c_void_p(4097)) == err["ALIGN"]

    def loss(h=h, v=2, x=p, w=p, t=p, size=8):
        return lib.hcnn_cross_entropy(h, 0, 2, 2, v, x, 2, w, 2, t, size, -100, z, z, p)

    assert loss(h=None) == err["NULL"] and loss(t=z) == err["NULL"] and loss(x=z) == err["NULL"] and loss(w=z) == err["NULL"]
    assert loss(v=0) == err["ARG"] and loss(size=2) == err["ARG"] and loss(t=ctypes.c_void_p(4100)) == err["ALIGN"]
    assert lib.hcnn_cross_entropy_grad(h, 0, 2, 2, 2, p, 2, p, 2, p, 8, -100, 1.0, z, p, p, 1, p, 2) == err["ARG"]

    one, types = (ctypes.c_size_t * 1)(4), (ctypes.c_int * 1)(0)
    ptrs, none = (ctypes.c_void_p * 1)(4096), (ctypes.c_void_p * 1)(None)
    clip = lib.hcnn_clip_grad_norm
    assert clip(None, 1, ptrs, one, types, None, 1.0, 0.0, p) == err["NULL"] and clip(h, 1, ptrs, one, types, None, 1.0, 0.0, None) == err["NULL"]
    assert clip(h, 1, none, one, types, None, 1.0, 0.0, p) == err["NULL"] and clip(h, 1, ptrs, one, types, none, 1.0, 0.0, p) == err["NULL"]
    assert clip(h, 1, ptrs, one, (ctypes.c_int * 1)(7), None, 1.0, 0.0, p) == err["ARG"]
    assert clip(h, 1, ptrs, one, types, None, -1.0, 0.0, p) == err["ARG"]
    assert clip(h, 1, (ctypes.c_void_p * 1)(4098), one, types, None, 1.0, 0.0, p) == err["ALIGN"]
    assert lib.hcnn_plain_create(None, None) == err["NULL"] and lib.hcnn_plain_destroy(None) == err["NULL"]
    assert lib.hcnn_plain_get_stat(h, 0, ctypes.byref(ctypes.c_uint64())) == err["ARG"]
