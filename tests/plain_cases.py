"""Cases of the training operators, shared by the CPU checker's tests and the device's (test helper, not collected).

A backend turns float64 arrays into arrays of a type ("f32", "f16", "bf16") and back; everything expected is computed here, in 64 bits,
from the values the arrays hold.  Bounds are derived from the number formats: u = half a unit of the last place of the type,
E = 2^-23 per operation of a 32-bit sum in any order (an fma rounds once, a split sum a few times more), and are checked number by number.
"""
import numpy as np
from scipy.special import erf

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}      # the type's smallest step
E = 2.0 ** -23
FN = 2.0 ** -20          # exponentials, erf and quotients in 32 bits: a few units of the last place
IGNORE = -100


def within(got, want, bound, what):
    got, want, bound = np.asarray(got, np.float64), np.asarray(want, np.float64), np.broadcast_to(np.asarray(bound, np.float64), np.shape(want))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if not got.size:
        return
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - bound
    worst = np.unravel_index(np.argmax(off), off.shape) if off.ndim else ()
    assert off[worst] <= 0, "%s: %r at %r, expected %r within %r" % (what, got[worst], worst, want[worst], bound[worst])


def act(z, name):
    """(value, slope)"""
    if name == "square":
        return z * z, 2 * z
    if name == "relu":
        return np.maximum(z, 0), (z > 0) * 1.0
    if name == "gelu":
        cdf = 0.5 * (1 + erf(z / np.sqrt(2)))
        return z * cdf, cdf + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    return z, np.ones_like(z)


def normal(rng, *shape, std=1.0):
    return rng.standard_normal(shape) * std


def check_linear(b, dtype, M, K, N, name="none", bias=False, residual=False, keep=False, seed=0, strides=None):
    rng = np.random.default_rng([seed, M, K, N])
    x, w = b.make(normal(rng, M, K), dtype, strides), b.make(normal(rng, N, K, std=max(K, 1) ** -0.5), dtype, strides)
    bi = b.make(normal(rng, N), dtype) if bias else None
    r = b.make(normal(rng, M, N), dtype, strides) if residual else None
    got = b.ctx.linear(x, w, bi, r, activation=name, keep=keep)
    y, z = got if keep else (got, None)
    X, W = b.values(x), b.values(w)
    Z = X @ W.T + (b.values(bi) if bias else 0)
    dz = (K + 4) * E * (np.abs(X) @ np.abs(W).T + (np.abs(b.values(bi)) if bias else 0))
    if keep:
        within(b.values(z), Z, U[dtype] * np.abs(Z) + dz + LEAST[dtype], "z")
    Y, S = act(Z, name)
    R = b.values(r) if residual else 0
    steep = 2 * np.abs(Z) + dz if name == "square" else 1.2
    err = steep * dz + (FN * (np.abs(Z) + 1e-30) * (2 + np.abs(Z)) if name in ("gelu", "silu") else 2 * E * np.abs(Y))
    within(b.values(y), Y + R, U[dtype] * np.abs(Y + R) + err + 2 * E * np.abs(R) + LEAST[dtype], "y")


def check_grad(b, dtype, M, K, N, name="none", bias=False, seed=0, strides=None, dy=None):
    rng = np.random.default_rng([seed, M, K, N, 1])
    x, w = b.make(normal(rng, M, K), dtype, strides), b.make(normal(rng, N, K, std=max(K, 1) ** -0.5), dtype, strides)
    dy = b.make(normal(rng, M, N), dtype, strides) if dy is None else dy
    z = b.make(normal(rng, M, N), dtype, strides) if name != "none" else None
    dx, dw, db = b.ctx.linear_grad(dy, x, w, z, activation=name, bias=bias)
    X, W, DY = b.values(x), b.values(w), b.values(dy)
    DZ = DY * act(b.values(z), name)[1] if name != "none" else DY
    slack = 0.0 if name == "none" else U[dtype] + 4 * E                      # dz is rounded to the type
    low = 0.0 if name == "none" else LEAST[dtype] + (np.abs(DY) * FN * 4 if name in ("gelu", "silu") else 0.0)
    dDZ = slack * np.abs(DZ) + low
    within(b.values(dx), DZ @ W, U[dtype] * np.abs(DZ @ W) + (dDZ + (N + 4) * E * np.abs(DZ)) @ np.abs(W) + LEAST[dtype], "dx")
    within(b.values(dw), DZ.T @ X, U[dtype] * np.abs(DZ.T @ X) + (dDZ + (M + 4) * E * np.abs(DZ)).T @ np.abs(X) + LEAST[dtype], "dw")
    if bias:
        D = DZ.sum(0)
        low = np.abs(DY) * FN * 4 if name in ("gelu", "silu") else np.zeros_like(DY)
        within(b.values(db), D, U[dtype] * np.abs(D) + ((M + 8) * E * np.abs(DZ) + low).sum(0) + LEAST[dtype], "db")
    else:
        assert db is None


def loss_inputs(b, dtype, M, D, V, masked=0.0, seed=0, strides=None, junk=False, std=1.0):
    rng = np.random.default_rng([seed, M, D, V, 2])
    w = normal(rng, V, D, std=max(D, 1) ** -0.5)
    t = rng.integers(0, V, size=M)
    x = normal(rng, M, D, std=std) + 3 * w[t]
    hide = rng.random(M) < masked
    if junk:                                                                 # what stands in masked rows must not be seen
        x[hide] = np.resize([np.nan, np.inf, -np.inf, 1.0], (int(hide.sum()), D))
    t[hide] = IGNORE
    return b.make(x, dtype, strides), b.make(w, dtype, strides), t


def loss_exact(X, W, t, scale=1.0):
    keep = t != IGNORE
    n = max(1, int(keep.sum()))
    X = np.where(keep[:, None], X, 0.0)
    L = X @ W.T
    top = L.max(1, keepdims=True) if L.size else np.zeros((len(t), 1))
    lse = (top + np.log(np.exp(L - top).sum(1, keepdims=True)))[:, 0]
    at = (np.arange(len(t)), np.where(keep, t, 0))
    rows = np.where(keep, lse - L[at], 0.0)
    p = np.exp(L - lse[:, None])
    p[at] -= 1
    p *= keep[:, None] * (scale / n)
    return rows.sum() / n, rows, np.where(keep, lse, 0.0), p, keep, n, L, X


def check_loss(b, dtype, M, D, V, masked=0.0, scale=1.0, wide=True, seed=0, strides=None, junk=False, std=1.0):
    x, w, t = loss_inputs(b, dtype, M, D, V, masked, seed, strides, junk, std)
    targets = b.ints(t, np.int64 if wide else np.int32)
    W = b.values(w)
    loss, rows, lse, p, keep, n, L, X = loss_exact(b.values(x), W, t, scale)
    d = (D + 4) * E * (np.abs(X) @ np.abs(W).T).max(1, initial=0.0)           # of a row's scores
    row_err = (2 * d + 8 * E * (np.abs(L).max(1, initial=0.0) + np.log(V) + 1) + FN) * keep
    got, got_rows, got_lse = b.ctx.cross_entropy(x, w, targets, ignore_index=IGNORE, rows=True)
    within(b.values(got_rows), rows, row_err, "row losses")
    within(b.values(got_lse), lse, row_err, "log sums")
    within(b.values(got), loss, row_err.sum() / n + E * abs(loss), "loss")
    assert np.array_equal(b.values(b.ctx.cross_entropy(x, w, targets, ignore_index=IGNORE)), b.values(got))
    got, dx, dw = b.ctx.cross_entropy_grad(x, w, targets, ignore_index=IGNORE, scale=scale)
    within(b.values(got), loss, row_err.sum() / n + E * abs(loss), "loss")
    q = np.abs(p) * U[dtype] + (scale / n) * (np.where(keep[:, None], np.exp(L - lse[:, None]), 0) * (row_err[:, None] * 2 + FN * (1 + np.abs(L - lse[:, None])))
                                              + LEAST[dtype] * (2.0 ** -15 if dtype == "f16" else 1.0)) * keep[:, None]
    DX, DW = p @ W, p.T @ X
    within(b.values(dx), DX, U[dtype] * np.abs(DX) + (q + (V + 8) * E * np.abs(p)) @ np.abs(W) + LEAST[dtype], "dx")
    within(b.values(dw), DW, U[dtype] * np.abs(DW) + (q + (M + 8) * E * np.abs(p)).T @ np.abs(X) + LEAST[dtype], "dw")
    assert (b.values(dx)[~keep] == 0).all()
    return dx, dw


def check_clip(b, dtypes, sizes, share, where="new", seed=0, std=0.01):
    rng = np.random.default_rng([seed, len(sizes), int(sum(sizes))])
    grads = [b.make(normal(rng, n, std=std), t) for n, t in zip(sizes, dtypes)]
    vals = [b.values(g) for g in grads]
    norm = float(np.sqrt(sum((v ** 2).sum() for v in vals)))
    max_norm = share * norm
    out = None if where == "place" else [b.make(np.full(n, 7.0), t) for n, t in zip(sizes, dtypes)]
    got = b.ctx.clip_grad_norm(grads, max_norm, out=out)
    within(b.values(got), norm, 2.0 ** -23 * norm + LEAST["f32"], "norm")
    factor = min(1.0, max_norm / (norm + 1e-6))
    for v, g, o, t in zip(vals, grads, out or grads, dtypes):
        within(b.values(o), v * factor, (U[t] + 4 * E) * np.abs(v) * factor + LEAST[t] if factor < 1 else 0.0, "gradient")
        if out is not None:
            assert np.array_equal(b.values(g), v)


# (dtype, rows, n_in, n_out, activation, bias, residual, keep): one row, one number, odd sizes, sizes at the tiles' edges
LINEAR = [("f32", 1, 1, 1, "none", False, False, False), ("bf16", 1, 200, 70, "gelu", True, True, True),
          ("f16", 5, 33, 17, "relu", True, False, True), ("f32", 130, 25, 5, "square", False, False, True),
          ("bf16", 65, 129, 130, "silu", True, True, False), ("f16", 16, 64, 128, "square", False, True, True),
          ("bf16", 17, 64, 16, "none", True, False, False), ("f32", 70, 100, 33, "gelu", True, True, True),
          ("bf16", 300, 70, 260, "square", True, False, True), ("f16", 129, 192, 257, "silu", False, False, False),
          ("f32", 257, 65, 129, "relu", False, True, False), ("bf16", 3, 1031, 9, "none", False, False, False),
          ("f32", 2, 0, 5, "gelu", True, True, True), ("bf16", 0, 4, 4, "none", False, False, True)]
GRAD = [("f32", 1, 1, 1, "none", False), ("bf16", 1, 200, 70, "gelu", True), ("f16", 5, 33, 17, "relu", True),
        ("f32", 700, 25, 5, "square", True), ("bf16", 65, 129, 130, "silu", True), ("f16", 130, 125, 50, "square", True),
        ("bf16", 300, 70, 260, "none", True), ("f32", 70, 100, 33, "gelu", False), ("f16", 257, 65, 16, "none", False),
        ("bf16", 0, 5, 7, "none", True), ("f32", 9, 3, 0, "none", False), ("f32", 6, 0, 4, "square", True)]
# (dtype, rows, n_in, classes, share of masked rows, scale)
LOSS = [("f32", 1, 1, 1, 0.0, 1.0), ("f32", 70, 40, 10, 0.0, 1.0), ("bf16", 33, 65, 300, 0.4, 1.0), ("f16", 130, 33, 129, 0.3, 1024.0),
        ("bf16", 260, 64, 17, 0.5, 1.0), ("f16", 7, 129, 515, 0.0, 64.0), ("f32", 65, 17, 130, 0.2, 2.0), ("bf16", 20, 16, 40, 1.0, 1.0),
        ("f32", 0, 8, 5, 0.0, 1.0), ("bf16", 1, 96, 1000, 0.0, 1.0)]
# for the device: every tile shape with its edges, long sums in parts, more rows than a launch's band of tiles
LINEAR_LARGE = [("bf16", 4100, 200, 4200, "gelu", True, True, True), ("f16", 3900, 129, 3800, "square", False, False, True),
                ("bf16", 2000, 1031, 1100, "silu", True, False, False), ("f32", 2100, 300, 1300, "gelu", True, True, True),
                ("bf16", 1, 4096, 4096, "none", True, True, False), ("f16", 12, 5001, 300, "relu", False, True, True),
                ("f32", 40000, 25, 5, "square", False, False, True), ("bf16", 600, 4000, 40, "none", True, False, False)]
GRAD_LARGE = [("bf16", 4100, 200, 4200, "gelu", True), ("f16", 3900, 129, 3800, "square", False), ("f32", 2100, 300, 1300, "silu", True),
              ("f32", 40000, 25, 5, "square", True), ("bf16", 16384, 125, 50, "square", True), ("f16", 2, 3000, 2000, "relu", True),
              ("bf16", 1024, 1025, 2049, "none", False)]
LOSS_LARGE = [("bf16", 2050, 128, 9001, 0.3, 1.0), ("f16", 1021, 517, 5003, 0.33, 1024.0), ("f32", 3000, 800, 10, 0.0, 1.0),
              ("f32", 700, 100, 3000, 0.1, 1.0), ("bf16", 3, 256, 40000, 0.4, 1.0), ("bf16", 5000, 64, 10, 0.9, 1.0)]
