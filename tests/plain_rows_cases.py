"""Cases of the operators between the plain network's layers -- dropout, root-mean-square norm, microscaled formats and their product -- shared by the CPU
checker's tests and the device's (test helper, not collected).

Everything expected is computed here in 64 bits from the values the arrays hold.  Bounds, checked number by number: u = half a unit of the last place of the
type for the rounding of a result, E = 2^-23 (two roundings of 32 bits) for every 32-bit operation in front of it.
"""
import numpy as np

import plain_cases as pc
from oracle import rng as orng

E, U, LEAST = pc.E, pc.U, pc.LEAST
TOP = {"mx4": 2, "mx8": 8}                  # exponent of the largest number
GRID = {"mx4": np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6]),
        "mx8": np.array([m * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127) for m in [c]])}


# ---------------------------------------------------------------- microscaled formats
def quantize(x, form):
    """(codes [rows][K], bytes [K / 32][rows], values [rows][K]) of a 64-bit matrix, K = columns up to whole 128: by search in the list of the format's numbers."""
    rows, n = x.shape
    K = -(-n // 128) * 128
    full = np.zeros((rows, K))
    full[:, :n] = x
    blocks = full.reshape(rows, K // 32, 32)
    top = np.abs(blocks).max(2, initial=0.0)
    bad = ~np.isfinite(top)
    with np.errstate(all="ignore"):
        e = np.where(top > 0, np.maximum(np.frexp(np.where(bad, 1.0, top))[1] - 1 - TOP[form], -127), 0)
    q = np.ldexp(np.where(bad[:, :, None], 0.0, blocks), -e[:, :, None])
    a = np.minimum(np.abs(q), GRID[form][-1])
    hi = np.clip(np.searchsorted(GRID[form], a), 1, len(GRID[form]) - 1)
    lo = hi - 1
    up, down = GRID[form][hi] - a, a - GRID[form][lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    values = np.where(bad[:, :, None], np.nan, np.ldexp(np.where(q < 0, -1, 1) * GRID[form][code], e[:, :, None]))
    sign = 8 if form == "mx4" else 128
    return (code + sign * np.signbit(q)).reshape(rows, K), np.where(bad, 255, e + 127).T, values.reshape(rows, K)


def packed(code, form):
    return code.astype(np.uint8) if form == "mx8" else (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)


def unpacked(codes, form):
    return codes.astype(int) if form == "mx8" else np.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1).astype(int)


def decode(codes, scales, form):
    """values [rows][K] of a matrix's bytes"""
    c = unpacked(codes, form)
    sign = 8 if form == "mx4" else 128
    grid = np.append(GRID[form], np.nan) if form == "mx8" else GRID[form]
    v = grid[c % sign] * np.where(c >= sign, -1, 1)
    e = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127)).T
    return (v.reshape(v.shape[0], -1, 32) * e[:, :, None]).reshape(v.shape)


def same_codes(got, want, form, what):
    """Equal but for the sign of zeros"""
    sign = 8 if form == "mx4" else 128
    got, want = np.where(got % sign == 0, 0, got), np.where(want % sign == 0, 0, want)
    assert np.array_equal(got, want), (what, np.argwhere(got != want)[:5].tolist())


def check_quantize(b, dtype, form, rows, n, x=None, seed=0, strides=None):
    rng = np.random.default_rng([seed, rows, n, 11])
    x = pc.normal(rng, rows, n) * np.exp2(rng.integers(-30 if dtype != "f16" else -6, 6, size=(rows, 1))) if x is None else x
    a = b.make(x, dtype, strides)
    m, values = b.ctx.quantize_mx(a, form, values=True)
    code, scale, want = quantize(b.values(a), form)
    assert m.shape == (rows, n) and m.format == form
    same_codes(unpacked(b.raw(m.codes), form), code, form, "codes")
    assert np.array_equal(b.raw(m.scales), scale), "scales"
    got, want = b.values(values), want[:, :n]
    # (values are numbers of the type: the codes' numbers have at most four bits, below the type's own least step they vanish)
    pc.within(np.nan_to_num(got), np.nan_to_num(want), LEAST[dtype] / 2 if dtype != "f32" else 2.0 ** -150, "values")
    assert np.array_equal(np.isnan(got), np.isnan(want))
    again = b.ctx.quantize_mx(a, form)
    assert np.array_equal(b.raw(again.codes), b.raw(m.codes)) and np.array_equal(b.raw(again.scales), b.raw(m.scales))


def microscaled(b, x, form, pitch=None):
    """A Microscaled matrix of the format's numbers nearest to x, made without the library, and its values.  What lies between the rows of scales is 255: NaN."""
    code, scale, values = quantize(x, form)
    return b.microscaled(packed(code, form), scale.astype(np.uint8), x.shape[1], form, pitch), values[:, :x.shape[1]]


def cut_of(X, W):
    """What the matrix unit may cut off the products of eight-bit numbers: each of eight neighbours to a multiple of 2^-13 of the power of two in the largest, seven of
    them (the largest product itself has six bits): 7 2^-13 of the largest product of every eight, added up.  [rows][n_out]  (Of large matrices: of the product of the
    largest numbers of every eight, which is not less.)"""
    K = X.shape[1]
    pad = -K % 8
    X, W = np.pad(np.abs(X), ((0, 0), (0, pad))), np.pad(np.abs(W), ((0, 0), (0, pad)))
    if X.shape[0] * W.shape[0] * K > 1 << 27:
        return X.reshape(len(X), -1, 8).max(2, initial=0.0) @ W.reshape(len(W), -1, 8).max(2, initial=0.0).T * 7 * 2.0 ** -13
    out = np.zeros((X.shape[0], W.shape[0]))
    for k in range(0, K + pad, 8):
        out += (X[:, None, k:k + 8] * W[None, :, k:k + 8]).max(2, initial=0.0)
    return out * 7 * 2.0 ** -13


def check_linear(b, dtype, form, M, K, N, name="none", bias=False, residual=False, seed=0, X=None, W=None, cut=None):
    rng = np.random.default_rng([seed, M, K, N, 12])
    X = pc.normal(rng, M, K) if X is None else X
    W = pc.normal(rng, N, K, std=max(K, 1) ** -0.5) if W is None else W
    x, X = microscaled(b, X, form)
    w, W = microscaled(b, W, "mx4")
    bi = b.make(pc.normal(rng, N), dtype) if bias else None
    r = b.make(pc.normal(rng, M, N), dtype) if residual else None
    y = b.ctx.linear_mx(x, w, bi, r, activation=name, dtype=b.type(dtype))
    Z = X @ W.T + (b.values(bi) if bias else 0)
    # 32-bit sums of K exact products, and the bias
    dz = (K + 4) * E * (np.abs(X) @ np.abs(W).T + (np.abs(b.values(bi)) if bias else 0))
    if form == "mx8" and dtype != "f32" and b.cuts:
        dz = dz + cut_of(X, W)
    Y, _ = pc.act(Z, name)
    R = b.values(r) if residual else 0
    steep = 2 * np.abs(Z) + dz if name == "square" else 1.2
    err = steep * dz + (pc.FN * (np.abs(Z) + 1e-30) * (2 + np.abs(Z)) if name in ("gelu", "silu") else 2 * E * np.abs(Y))
    pc.within(b.values(y), Y + R, U[dtype] * np.abs(Y + R) + err + 2 * E * np.abs(R) + LEAST[dtype], "y")
    return y


# ---------------------------------------------------------------- dropout
def kept(rows, n, p, seed, stream):
    words = orng.philox4x32_10((np.arange(-(-n // 4))[None, :], np.arange(rows)[:, None], stream, 4 << 24), (seed & 0xFFFFFFFF, seed >> 32))
    words = np.stack([np.broadcast_to(w, (rows, -(-n // 4))) for w in words], 2).reshape(rows, -1)[:, :n]
    return words.astype(np.uint64) >= np.uint64(round(p * 2 ** 32))


def check_dropout(b, dtype, rows, n, p, residual, seed=0x123456789ABCDEF0, stream=7, strides=None, junk=False):
    rng = np.random.default_rng([rows, n, 13])
    keep = kept(rows, n, p, seed, stream)
    x = pc.normal(rng, rows, n)
    if junk:                                # what is dropped must not be seen
        x[~keep] = np.resize([np.nan, np.inf, -np.inf], int((~keep).sum()))
    x = b.make(x, dtype, strides)
    r = b.make(pc.normal(rng, rows, n), dtype, strides) if residual else None
    X, R = np.where(keep, b.values(x), 0.0), b.values(r) if residual else 0.0
    S = X / (1 - p) if p < 1 else np.zeros_like(X)
    Y = S + R
    bound = U[dtype] * np.abs(Y) + 2 * E * (np.abs(S) + np.abs(Y)) + LEAST[dtype]
    pc.within(b.values(b.ctx.dropout(x, p, seed, stream, residual=r)), Y, bound, "y")
    got = b.ctx.dropout_grad(x, p, seed, stream)
    pc.within(b.values(got), S, U[dtype] * np.abs(S) + 2 * E * np.abs(S) + LEAST[dtype], "dx")
    assert (b.values(got)[~keep] == 0).all()


# ---------------------------------------------------------------- norm
def norm_inputs(b, dtype, rows, n, residual, weight, seed=0, strides=None, std=1.0):
    rng = np.random.default_rng([seed, rows, n, 14])
    x = b.make(pc.normal(rng, rows, n, std=std) * np.exp(rng.standard_normal((rows, 1))), dtype, strides)
    r = b.make(pc.normal(rng, rows, n, std=std), dtype, strides) if residual else None
    w = b.make(1 + 0.2 * pc.normal(rng, n), dtype) if weight else None
    return x, r, w


def norm_exact(S, W, eps):
    q = 1 / np.sqrt((S * S).mean(1, keepdims=True) + eps)
    return q, S * q * W


def check_norm(b, dtype, rows, n, residual=False, weight=True, eps=1e-6, seed=0, strides=None, std=1.0):
    x, r, w = norm_inputs(b, dtype, rows, n, residual, weight, seed, strides, std)
    y, s = b.ctx.rms_norm(x, w, r, eps=eps, keep=True)
    S = b.values(x) + (b.values(r) if residual else 0)
    W = b.values(w) if weight else np.ones(n)
    _, Y = norm_exact(S, W, eps)
    # the sum, the inverse root's two factors and the weight: five roundings of 32 bits, and the sums' own in the mean
    pc.within(b.values(y), Y, U[dtype] * np.abs(Y) + 4 * E * np.abs(Y) + LEAST[dtype], "y")
    pc.within(b.values(s), S, U[dtype] * np.abs(S) + E * np.abs(S) + LEAST[dtype], "s")
    assert np.array_equal(b.values(b.ctx.rms_norm(x, w, r, eps=eps)), b.values(y))


def check_norm_mx(b, dtype, rows, n, residual=False, weight=True, eps=1e-6, seed=0, strides=None):
    x, r, w = norm_inputs(b, dtype, rows, n, residual, weight, seed, strides)
    m, s = b.ctx.rms_norm(x, w, r, eps=eps, keep=True, format="mx8")
    S = b.values(x) + (b.values(r) if residual else 0)
    _, Y = norm_exact(S, b.values(w) if weight else np.ones(n), eps)
    # 64 bits up to the one rounding, but for a 32-bit sum with the residual: nearest for a number within that of the exact one
    near = 2 * E if residual else 1e-13
    got, scale = unpacked(b.raw(m.codes), "mx8"), b.raw(m.scales)
    got = np.where(got % 128 == 0, 0, got)
    fits_code, fits_scale = np.zeros(got.shape, bool), np.zeros(scale.shape, bool)
    for f in (1 - near, 1.0, 1 + near):
        code, byte, _ = quantize(Y * f, "mx8")
        fits_code |= got == np.where(code % 128 == 0, 0, code)
        fits_scale |= scale == byte
    assert fits_code.all() and fits_scale.all(), (np.argwhere(~fits_code)[:5], np.argwhere(~fits_scale)[:5])
    pc.within(b.values(s), S, U[dtype] * np.abs(S) + E * np.abs(S) + LEAST[dtype], "s")


def check_norm_grad(b, dtype, rows, n, ds=False, weight=True, eps=1e-6, seed=0, strides=None, std=1.0):
    s, d, w = norm_inputs(b, dtype, rows, n, ds, weight, seed, strides, std)
    rng = np.random.default_rng([seed, rows, n, 15])
    dy = b.make(pc.normal(rng, rows, n), dtype, strides)
    dx, dw = b.ctx.rms_norm_grad(dy, s, w, d, eps=eps)
    S, DY, W, D = b.values(s), b.values(dy), b.values(w) if weight else np.ones(n), b.values(d) if ds else 0.0
    q, u = norm_exact(S, 1.0, eps)
    g = DY * W
    mean, size = (g * u).mean(1, keepdims=True), np.abs(g * u).mean(1, keepdims=True)
    DX = q * (g - u * mean) + D
    err = q * (8 * E * (np.abs(g) + np.abs(u * mean)) + 4 * E * np.abs(u) * size) + E * (np.abs(D) + np.abs(DX))
    pc.within(b.values(dx), DX, U[dtype] * np.abs(DX) + err + LEAST[dtype], "dx")
    if weight:
        DW = (DY * u).sum(0)
        pc.within(b.values(dw), DW, U[dtype] * np.abs(DW) + (rows + 8) * E * np.abs(DY * u).sum(0) + LEAST[dtype], "dw")
        assert b.ctx.rms_norm_grad(dy, s, w, d, eps=eps, need_dweight=False)[1] is None
    else:
        assert dw is None


# rows, columns: one of each, less than an access, odd, a wave's worth and one more, several threads' shapes, blocks that are not whole
SIZES = [(1, 1), (3, 2), (5, 31), (70, 33), (2, 128), (9, 129), (33, 257), (4, 1000), (3, 1025), (2, 4097)]
# dtype, x format, rows, n_in, n_out, activation, bias, residual: one row, rows and columns at a tile's edges, blocks and steps that are not whole
LINEAR = [("bf16", "mx8", 1, 1, 1, "none", False, False), ("f32", "mx8", 1, 300, 70, "silu", True, True), ("f16", "mx4", 5, 33, 17, "relu", True, False),
          ("bf16", "mx4", 16, 128, 64, "square", False, True), ("f32", "mx4", 17, 129, 16, "gelu", True, True), ("f16", "mx8", 65, 257, 66, "gelu", True, True),
          ("bf16", "mx8", 64, 1100, 63, "none", True, False), ("f32", "mx8", 70, 40, 5, "square", False, False), ("bf16", "mx4", 0, 4, 4, "none", False, False),
          ("f32", "mx8", 2, 0, 5, "gelu", True, True), ("f16", "mx4", 130, 384, 129, "silu", False, True)]
