"""The operators between the plain network's layers on the CPU checker of the kernel sources: values against 64-bit definitions, gradients against differences,
masks, empty and long rows, refusals.  (The device's tests run the same cases at its sizes.)"""
import ctypes

import numpy as np
import pytest

import emu
import plain_cases as pc
import plain_rows_cases as rc
from paper_1811_00778_amd import _capi
from paper_1811_00778_amd._plain_ops import Microscaled
from test_plain_ops import _CODE, _NP, Backend, EmuPlain

TYPES = ["f32", "f16", "bf16"]


class EmuRows(EmuPlain):
    def _bytes(self, x, what):
        if not isinstance(x, np.ndarray) or x.dtype != np.uint8 or x.ndim != 2:
            raise TypeError("%s must be a 2-D array of bytes" % what)
        return x.ctypes.data, x.shape, x.strides

    @staticmethod
    def _room(x):
        base = x if x.base is None else x.base
        return base.nbytes - (x.ctypes.data - base.ctypes.data)

    def _new_bytes(self, rows, cols, of):
        return emu.aligned(np.full((rows, cols), 0xff, np.uint8))[:, :of]

    def _new_of(self, shape, dtype):
        a = np.empty(shape, dtype)
        a.reshape(-1).view(np.uint8).fill(0xff)
        return a, _CODE[a.dtype]


class RowsBackend(Backend):
    cuts = False                          # (the checker adds products as they are)

    def __init__(self):
        self.ctx = EmuRows()

    def type(self, dtype):
        return np.dtype(_NP[dtype])

    def raw(self, a):
        return a

    def microscaled(self, codes, scales, columns, form, pitch=None):
        rows = codes.shape[0]
        room = np.full((scales.shape[0], pitch or -(-rows // 64) * 64), 255, np.uint8)
        room[:, :rows] = scales
        return Microscaled(emu.aligned(codes), emu.aligned(room)[:, :rows], columns, form)


@pytest.fixture(scope="module", params=[1, 256], ids=["one-unit", "256-units"])
def b(request):
    with emu.device(emu.lib(), units=request.param):
        yield RowsBackend()


class few_threads:
    """Launches of at most so many threads while the block runs"""

    def __init__(self, most):
        self.set, self.most = emu.lib().hcnn_emu_threads, most
        self.set.argtypes, self.set.restype = [ctypes.c_uint64], None

    def __enter__(self):
        self.set(self.most)

    def __exit__(self, *_):
        self.set(0xffffffff)


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES, ids=str)
def test_dropout(b, dtype, size):
    rc.check_dropout(b, dtype, *size, 0.3, True)
    rc.check_dropout(b, dtype, *size, 0.9, False, seed=2 ** 64 - 1, stream=2 ** 32 - 1, strides=(5, 1), junk=True)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -33, 0.5, 1 - 2.0 ** -33, 1.0])
def test_dropout_at_the_ends(b, p):
    rc.check_dropout(b, "f32", 9, 30, p, True, junk=p > 0.4)
    x = b.make(np.ones((4, 9)), "bf16")
    if p == 0:
        assert np.array_equal(b.ctx.dropout(x, p, 3), x)


def test_dropout_counts_and_streams(b):
    """the share that is kept; masks of other seeds and streams have nothing in common with this one's"""
    one = b.make(np.ones((200, 500)), "f32")
    masks = [b.values(b.ctx.dropout(one, 0.25, s, t)) > 0 for s, t in ((1, 0), (2, 0), (1, 1), (1 << 32, 0))]
    for m in masks:                                                   # 1e5 draws: five standard deviations are 0.007
        assert abs(m.mean() - 0.75) < 0.007
    for m in masks[1:]:                                               # independent ones agree on 0.625 of the places
        assert abs((m == masks[0]).mean() - 0.625) < 0.008
    # rows and columns of a part of the matrix: the mask is that of the place, whatever the type
    part = b.values(b.ctx.dropout(b.make(np.ones((150, 321)), "f16"), 0.25, 1, 0)) > 0
    assert np.array_equal(part, masks[0][:150, :321])


@pytest.mark.parametrize("dtype", TYPES)
def test_dropout_in_place(b, dtype):
    x, r = pc.normal(np.random.default_rng(1), 13, 37), pc.normal(np.random.default_rng(2), 13, 37)
    want = b.ctx.dropout(b.make(x, dtype, (3, 1)), 0.4, 5, 6, residual=b.make(r, dtype, (3, 1)))
    for place in (0, 1):
        ins = [b.make(x, dtype, (3, 1)), b.make(r, dtype, (3, 1))]
        got = b.ctx.dropout(ins[0], 0.4, 5, 6, residual=ins[1], out=ins[place])
        assert got is ins[place] and np.array_equal(got, want)


# ---------------------------------------------------------------- norm
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES, ids=str)
def test_norm(b, dtype, size):
    rc.check_norm(b, dtype, *size, residual=True)
    rc.check_norm(b, dtype, *size, weight=False, strides=(3, 1))
    rc.check_norm_mx(b, dtype, *size)
    rc.check_norm_mx(b, dtype, *size, residual=True, weight=False, strides=(3, 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES, ids=str)
def test_norm_grad(b, dtype, size):
    rc.check_norm_grad(b, dtype, *size, ds=True)
    rc.check_norm_grad(b, dtype, *size, weight=False, strides=(3, 1))


@pytest.mark.parametrize("n", [16384, 16385, 17000])
def test_rows_longer_than_the_registers(b, n):
    for dtype in TYPES:
        rc.check_norm(b, dtype, 2, n, residual=True)
        rc.check_norm_grad(b, dtype, 3, n, ds=True)
    rc.check_norm_mx(b, "bf16", 2, n, residual=True)


def test_norm_of_many_rows(b):
    rc.check_norm_grad(b, "f32", 3000, 5)
    with few_threads(1024):                  # (more than one launch)
        rc.check_norm(b, "bf16", 300, 20, residual=True)
        rc.check_norm_mx(b, "bf16", 40, 140, residual=True)
        rc.check_norm_grad(b, "f16", 3, 100)
        rc.check_dropout(b, "f32", 70, 200, 0.5, True)
        rc.check_quantize(b, "bf16", "mx4", 40, 700)
        rc.check_linear(b, "bf16", "mx8", 3, 300, 200, "relu", bias=True)
        rc.check_linear(b, "f32", "mx4", 90, 140, 20)


def test_norm_of_large_and_small_numbers(b):
    """squares that 32 bits do not hold; rows of zeros"""
    for std in (1e25, 1e37, 1e-30):
        rc.check_norm(b, "f32", 4, 300, std=std, eps=1e-30)
        rc.check_norm(b, "bf16", 4, 300, std=std, eps=1e-30)
    rc.check_norm_grad(b, "f32", 4, 300, std=1e25)
    zeros = b.make(np.zeros((3, 40)), "f16")
    assert (b.values(b.ctx.rms_norm(zeros)) == 0).all()
    m = b.ctx.rms_norm(zeros, format="mx8")
    assert (b.raw(m.codes) == 0).all() and (b.raw(m.scales) == 127).all()
    dx, _ = b.ctx.rms_norm_grad(b.make(np.ones((3, 40)), "f16"), zeros, eps=1e-2)
    assert np.array_equal(b.values(dx), np.full((3, 40), 10.0))


def test_norm_of_what_is_not_finite(b):
    """an infinity or a NaN stays in its row"""
    x = pc.normal(np.random.default_rng(3), 4, 200)
    x[1, 7], x[2, 150] = np.inf, np.nan
    a = b.make(x, "f32")
    y = b.values(b.ctx.rms_norm(a))
    assert np.isfinite(y[[0, 3]]).all() and np.isnan(y[1, 7]) and (np.delete(y[1], 7) == 0).all() and np.isnan(y[2]).all()
    m = b.ctx.rms_norm(a, format="mx8")
    s = b.raw(m.scales)
    assert (s[0, 1] == 255) and (s[1:, 1] == 127).all() and (s[:7, 2] == 255).all() and (s[7, 2] == 127) and (s[:, [0, 3]] < 255).all()
    assert (unpack_row(b, m, 1)[:32] == 0).all()


def unpack_row(b, m, row):
    return rc.unpacked(b.raw(m.codes), m.format)[row]


def test_norm_of_no_rows(b):
    for rows, n in ((0, 5), (3, 0), (0, 0)):
        x, w = b.make(np.zeros((rows, n)), "bf16"), b.make(np.ones(n), "bf16")
        assert b.ctx.rms_norm(x, w).shape == (rows, n)
        assert b.ctx.rms_norm(x, w, format="mx8").shape == (rows, n)
        dx, dw = b.ctx.rms_norm_grad(x, x, w)
        assert dx.shape == (rows, n) and (b.values(dw) == 0).all() and dw.shape == (n,)
        assert b.ctx.dropout(x, 0.5, 1).shape == (rows, n)
        assert b.ctx.quantize_mx(x).shape == (rows, n)


def test_norm_gradient_is_the_difference(b):
    rng = np.random.default_rng(8)
    M, N, h, eps = 5, 23, 2.0 ** -6, 1e-3
    s, w, dy, ds = (b.make(rng.standard_normal(z), "f32") for z in ((M, N), (N,), (M, N), (M, N)))
    dx, dw = (b.values(v) for v in b.ctx.rms_norm_grad(dy, s, w, ds, eps=eps))
    S, W, DY, DS = (b.values(v) for v in (s, w, dy, ds))
    for _ in range(4):
        us, uw = rng.standard_normal(S.shape), rng.standard_normal(W.shape)
        us, uw = us / np.linalg.norm(us), uw / np.linalg.norm(uw)
        at = [(rc.norm_exact(S + t * h * us, W + t * h * uw, eps)[1] * DY).sum() + ((S + t * h * us) * DS).sum() for t in (-2, -1, 1, 2)]
        # (fourth-order differences: h^4 / 30 of a fifth derivative, below 1e-8 x 1e3; 32-bit gradients leave 1e-5)
        assert abs((dx * us).sum() + (dw * uw).sum() - (at[0] - 8 * at[1] + 8 * at[2] - at[3]) / (12 * h)) < 1e-4


def test_dropout_gradient_is_the_difference(b):
    """linear in x: the slope along any direction, over the whole step"""
    rng = np.random.default_rng(9)
    x, u, dy = (b.make(np.rint(rng.standard_normal((6, 30)) * 16) / 16, "f32") for _ in range(3))
    f = [b.values(b.ctx.dropout(b.make(b.values(x) + t * b.values(u), "f32"), 0.5, 4, 2, residual=x)) for t in (-1, 1)]
    slope = (b.values(b.ctx.dropout_grad(dy, 0.5, 4, 2)) * b.values(u)).sum()
    assert abs(((f[1] - f[0]) * b.values(dy)).sum() / 2 - slope) < 1e-12 * 180


# ---------------------------------------------------------------- microscaled formats
@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES, ids=str)
def test_quantize(b, dtype, form, size):
    rc.check_quantize(b, dtype, form, *size)
    rc.check_quantize(b, dtype, form, *size, strides=(3, 1))


def edge_numbers(form):
    """rows of 32: ties and neighbours of every number of the grid under a largest number that fixes the scale, and numbers that are cut to the largest"""
    grid = rc.GRID[form]
    mids = (grid[1:] + grid[:-1]) / 2
    v = np.concatenate([grid, mids, mids * (1 - 2.0 ** -7), mids * (1 + 2.0 ** -7)])
    v = np.concatenate([v, -v])
    v = np.pad(v, (0, -len(v) % 31))
    rows = np.concatenate([np.full((len(v) // 31, 1), 2.0 ** rc.TOP[form] * 1.984375), v.reshape(-1, 31)], 1)
    return np.concatenate([rows, rows * 2.0 ** -14, np.zeros((1, 32))])


@pytest.mark.parametrize("form", ["mx4", "mx8"])
def test_quantize_ties_and_ends(b, form):
    rows = edge_numbers(form)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows * 2.0 ** -120)            # the least scale and below
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows * 2.0 ** -140)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows * 2.0 ** (127 - rc.TOP[form]))
    rc.check_quantize(b, "bf16", form, *rows.shape, x=rows)
    rc.check_quantize(b, "f16", form, *rows.shape, x=rows * 2.0 ** -10)


def test_quantize_what_is_not_finite(b):
    x = pc.normal(np.random.default_rng(3), 3, 100)
    x[0, 40], x[2, 99] = -np.inf, np.nan
    rc.check_quantize(b, "bf16", "mx4", 3, 100, x=x)
    rc.check_quantize(b, "f32", "mx8", 3, 100, x=x)


@pytest.mark.parametrize("case", rc.LINEAR, ids=str)
def test_linear_mx(b, case):
    rc.check_linear(b, *case)


def test_linear_mx_wide_scales_and_nan(b):
    """blocks of very different size in one row; a block that stands for NaN makes its row or column NaN and nothing else"""
    rng = np.random.default_rng(4)
    X = pc.normal(rng, 20, 300) * np.exp2(rng.integers(-20, 20, size=(20, 10)).repeat(30, 1))
    rc.check_linear(b, "f32", "mx8", 20, 300, 40, X=X)
    rc.check_linear(b, "bf16", "mx4", 20, 300, 40, X=X)
    X[3, 77] = np.nan
    x, _ = rc.microscaled(b, X, "mx8")
    w, _ = rc.microscaled(b, pc.normal(rng, 40, 300), "mx4")
    y = b.values(b.ctx.linear_mx(x, w, dtype=b.type("f32")))
    assert np.isnan(y[3]).all() and np.isfinite(np.delete(y, 3, 0)).all()


def test_linear_mx_into_place(b):
    rng = np.random.default_rng(6)
    x, _ = rc.microscaled(b, pc.normal(rng, 30, 140), "mx8", pitch=192)
    w, _ = rc.microscaled(b, pc.normal(rng, 50, 140), "mx4")
    r = pc.normal(rng, 30, 50)
    want = b.ctx.linear_mx(x, w, residual=b.make(r, "bf16"), activation="relu")
    place = b.make(r, "bf16", (6, 1))
    assert b.ctx.linear_mx(x, w, residual=place, activation="relu", out=place) is place
    assert np.array_equal(b.values(place), b.values(want))


def test_an_answer_from_few_bits(b):
    """dropout, norm with the residual into eight bits, the product with four-bit weights: each step's result is what the next one takes"""
    rng = np.random.default_rng(7)
    x, r = b.make(pc.normal(rng, 18, 200), "bf16"), b.make(pc.normal(rng, 18, 200), "bf16")
    h = b.ctx.dropout(x, 0.2, 11, 1, residual=r)
    m, s = b.ctx.rms_norm(h, b.make(np.ones(200), "bf16"), residual=x, keep=True, format="mx8")
    w, W = b.ctx.quantize_mx(b.make(pc.normal(rng, 70, 200), "bf16"), "mx4", values=True)
    y = b.ctx.linear_mx(m, w, b.make(pc.normal(rng, 70), "f32"), activation="gelu")
    X = rc.decode(b.raw(m.codes), b.raw(m.scales), "mx8")[:, :200]
    _, want = rc.norm_exact(b.values(h) + b.values(x), 1.0, 1e-6)
    # eight bits: half a step of 2^-3 of a number, but numbers between 448 and 512 of their block's scale are cut to 448, by less than 64 / 512 of themselves
    assert np.abs(X - want).max() <= 2.0 ** -3 * np.abs(want).max() * (1 + 1e-6)
    assert np.array_equal(W, b.ctx.quantize_mx(W, "mx4", values=True)[1])                  # numbers of the format stay
    assert y.dtype == b.type("f32")


# ---------------------------------------------------------------- refusals
def test_refusals(b):
    c = b.ctx
    x, r = b.make(np.ones((6, 40)), "f32"), b.make(np.ones((6, 40)), "f32")
    half = b.make(np.ones((6, 40)), "f16")
    for p in (-0.1, 1.1, np.nan):
        with pytest.raises(ValueError):
            c.dropout(x, p, 1)
    for seed, stream in ((-1, 0), (1 << 64, 0), (1, -1), (1, 1 << 32)):
        with pytest.raises(ValueError):
            c.dropout(x, 0.5, seed, stream)
    with pytest.raises(ValueError):
        c.dropout(x, 0.5, 1, residual=b.make(np.ones((6, 41)), "f32"))
    with pytest.raises(TypeError):
        c.dropout(x, 0.5, 1, residual=half)
    flat = b.make(np.ones(600), "f32")
    with pytest.raises(ValueError):                                            # a place that overlaps its input by a row
        c.dropout(flat[40:280].reshape(6, 40), 0.5, 1, out=flat[:240].reshape(6, 40))
    for eps in (0.0, -1.0, 1e-40, np.nan, np.inf):
        with pytest.raises(ValueError):
            c.rms_norm(x, eps=eps)
        with pytest.raises(ValueError):
            c.rms_norm_grad(x, x, eps=eps)
    with pytest.raises(ValueError):
        c.rms_norm(x, format="mx4")
    with pytest.raises(ValueError):
        c.rms_norm(x, b.make(np.ones(41), "f32"))
    with pytest.raises(TypeError):
        c.rms_norm(x, b.make(np.ones(40), "f16"))
    with pytest.raises(TypeError):
        c.rms_norm_grad(half, x)
    with pytest.raises(ValueError):
        c.quantize_mx(x, "mx6")
    m, w = c.quantize_mx(x, "mx8"), c.quantize_mx(x, "mx4")
    with pytest.raises(ValueError):
        c.linear_mx(w, m, dtype=b.type("f32"))                                  # eight-bit weights
    with pytest.raises(ValueError):
        c.linear_mx(m, c.quantize_mx(b.make(np.ones((6, 41)), "f32")), dtype=b.type("f32"))
    with pytest.raises(ValueError):
        c.linear_mx(m, w)                                                       # no type
    with pytest.raises(TypeError):
        c.linear_mx(x, w, dtype=b.type("f32"))
    with pytest.raises(ValueError):
        c.linear_mx(Microscaled(m.codes, m.scales, 300, "mx8"), w, dtype=b.type("f32"))
    with pytest.raises(ValueError):
        c.linear_mx(Microscaled(m.codes[:4], m.scales, 40, "mx8"), w, dtype=b.type("f32"))
    with pytest.raises(ValueError):
        c.linear_mx(Microscaled(m.codes, emu.aligned(m.scales), 40, "mx8"), w, dtype=b.type("f32"))      # no room between the rows
    with pytest.raises(ValueError):
        Microscaled(m.codes, m.scales, 40, "mx5")


def test_refusals_of_the_library(b):
    lib, h = emu.lib(), b.ctx.raw.handle
    x = emu.aligned(np.zeros((64, 128), np.float32))
    p = x.ctypes.data
    bad, null, align = (_capi.ERR[k] for k in ("ARG", "NULL", "ALIGN"))
    assert lib.hcnn_dropout(h, 3, 1, 1, p, 1, None, 0, 0.5, 1, 1, p, 1) == bad
    assert lib.hcnn_dropout(h, 0, 1, 2, p, 2, None, 0, 0.5, 1, 1, p, 1) == bad
    assert lib.hcnn_dropout(h, 0, 1, 1, None, 1, None, 0, 0.5, 1, 1, p, 1) == null
    assert lib.hcnn_dropout(h, 0, 1, 1, p + 2, 1, None, 0, 0.5, 1, 1, p, 1) == align
    assert lib.hcnn_dropout(h, 0, 1, 1, p, 1, None, 0, float("nan"), 1, 1, p, 1) == bad
    assert lib.hcnn_dropout(None, 0, 1, 1, p, 1, None, 0, 0.5, 1, 1, p, 1) == null
    assert lib.hcnn_rms_norm(h, 0, 1, 4, p, 4, None, 0, None, 1e-6, None, 0, None, 4, None, None, 0) == null
    assert lib.hcnn_rms_norm(h, 0, 1, 4, p, 4, None, 0, None, 1e-6, None, 0, p, 4, p, p, 64) == bad
    assert lib.hcnn_rms_norm(h, 0, 1, 4, p, 4, None, 0, None, 1e-6, None, 0, None, 4, p, None, 64) == null
    assert lib.hcnn_rms_norm(h, 0, 65, 4, p, 4, None, 0, None, 1e-6, None, 0, None, 4, p, p, 64) == bad
    assert lib.hcnn_rms_norm(h, 0, 1, 4, p, 4, None, 0, None, 1e-6, None, 0, None, 4, p + 4, p, 64) == align
    assert lib.hcnn_rms_norm(h, 0, 1, 4, p, 4, None, 0, None, 0.0, None, 0, p, 4, None, None, 0) == bad
    assert lib.hcnn_rms_norm_grad(h, 0, 1, 4, p, 4, None, 4, None, None, 0, 1e-6, p, 4, None) == null
    assert lib.hcnn_rms_norm_grad(h, 0, 1, 4, p, 4, p, 4, None, None, 0, 1e-6, p, 3, None) == bad
    assert lib.hcnn_quantize_mx(h, 0, 5, 1, 4, p, 4, p, p, 64, None, 0) == bad
    assert lib.hcnn_quantize_mx(h, 0, 4, 1, 4, p, 4, p, p, 63, None, 0) == bad
    assert lib.hcnn_quantize_mx(h, 0, 4, 1, 4, p, 4, p, None, 64, None, 0) == null
    assert lib.hcnn_linear_mx(h, 0, 8, 9, 1, 4, 4, p, p, 64, p, p, 64, None, None, 0, p, 4) == bad
    assert lib.hcnn_linear_mx(h, 0, 8, 0, 1, 4, 4, p, p, 64, p, p, 64, None, None, 0, p, 3) == bad
    assert lib.hcnn_linear_mx(h, 0, 8, 0, 1, 4, 4, p, p, 64, p, p + 8, 64, None, None, 0, p, 4) == align
    assert lib.hcnn_linear_mx(h, 0, 8, 0, 1, 4, 65, p, p, 64, p, p, 64, None, None, 0, p, 65) == bad
    assert lib.hcnn_linear_mx(h, 0, 8, 0, 1, 4, 4, None, p, 64, p, p, 64, None, None, 0, p, 4) == null


# ---------------------------------------------------------------- the product's shapes
@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("tile,size", [(0, (300, 300, 270)), (0, (257, 130, 30)), (1, (140, 600, 150)), (1, (129, 1200, 129)), (1, (40, 120, 200))])
@pytest.mark.parametrize("parts", [1, 3])
def test_tiles_of_the_product(b, form, tile, size, parts):
    """every tile, one slot and several, a slot that is not whole, parts of k"""
    lib = emu.lib()
    lib.hcnn_emu_shape.argtypes, lib.hcnn_emu_shape.restype = [ctypes.c_int, ctypes.c_uint32, ctypes.c_int], None
    lib.hcnn_emu_taken.argtypes, lib.hcnn_emu_taken.restype = [ctypes.POINTER(ctypes.c_uint64)] * 2, None
    lib.hcnn_emu_shape(tile, parts, 0)
    try:
        rc.check_linear(b, "bf16", form, *size, "relu", bias=True, residual=True)
        rc.check_linear(b, "f32", form, *size, "none")
        bits, copied = ctypes.c_uint64(), ctypes.c_uint64()
        lib.hcnn_emu_taken(ctypes.byref(bits), ctypes.byref(copied))
        steps = -(-size[1] // 128)
        each = -(-(-(-steps // parts)) // 2) * 2
        assert bits.value == 1 << (0 if -(-steps // each) == 1 else 1) << (0 if tile == 0 else 2) << (0 if form == "mx4" else 4)
    finally:
        lib.hcnn_emu_shape(-1, 1, 0)


def test_shapes_of_the_product_by_the_rule():
    """every shape has sizes that take it on a device of 256 compute units"""
    lib = emu.lib()
    lib.hcnn_emu_mx_choice.argtypes, lib.hcnn_emu_mx_choice.restype = [ctypes.c_void_p, ctypes.c_int] + [ctypes.c_size_t] * 3, ctypes.c_uint32
    with emu.device(lib, units=256):
        ctx = EmuRows()
        got = {(form, size): lib.hcnn_emu_mx_choice(ctx.raw.handle, form, *size) for form in (4, 8)
               for size in ((1, 4096, 4096), (1, 4096, 16384), (64, 4096, 4096), (64, 4096, 16384), (1024, 4096, 4096), (8192, 8192, 256), (4096, 4096, 4096), (5000, 100, 3))}
    want = {(1, 4096, 4096): (0, 1), (1, 4096, 16384): (1, 1), (64, 4096, 4096): (2, 1), (64, 4096, 16384): (3, 1), (1024, 4096, 4096): (4, 1), (8192, 8192, 256): (4, 2),
            (4096, 4096, 4096): (5, 1), (5000, 100, 3): (2, 1)}
    for (form, size), choice in got.items():
        assert (choice & 255, choice >> 8) == want[size], (form, size, choice)
