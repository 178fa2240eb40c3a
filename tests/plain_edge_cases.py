"""Further cases of the training operators, shared by the CPU checker's tests and the device's (test helper, not collected).
Backends, bounds and definitions are plain_cases'."""
import numpy as np
from scipy.special import ndtr

import plain_cases as pc
from plain_cases import E, FN, LEAST, U, normal, within

# (dtype, rows, n_in, classes, first class of -infinity, one past the last): a class alone in a lane, all but the narrowest tile's
# columns, whole tiles in front of and behind the others, all but one class
LOW = [("f32", 9, 5, 33, 32, 33), ("bf16", 9, 5, 33, 32, 33), ("f32", 70, 40, 40, 16, 40), ("bf16", 30, 9, 300, 16, 300),
       ("f32", 20, 33, 300, 0, 290), ("bf16", 65, 64, 520, 100, 519), ("f32", 21, 7, 10, 3, 9), ("f16", 33, 20, 300, 16, 300),
       ("f16", 9, 5, 40, 0, 39)]


def check_low_classes(b, dtype, M, D, V, first, last, masked=0.2, seed=0):
    """Classes whose score is -infinity in 32 bits take no part: loss and gradients are those of the other classes, their own rows 0.
    The last number of x and w makes those scores: a product beyond the range, and in binary16, which has none, an infinite weight (dx is then
    0 times infinity, as it is by the formula, and not looked at)."""
    rng = np.random.default_rng([seed, M, D, V, first, 5])
    w = np.concatenate([normal(rng, V, D, std=D ** -0.5), np.zeros((V, 1))], 1)
    low = np.zeros(V, bool)
    low[first:last] = True
    far = -np.inf if dtype == "f16" else -1e20
    w[low, D] = far
    t = rng.choice(np.nonzero(~low)[0], size=M)
    x = np.concatenate([normal(rng, M, D) + 3 * w[t, :D], np.full((M, 1), 1.0 if dtype == "f16" else 1e20)], 1)
    hide = rng.random(M) < masked
    hide[0] = False
    t[hide] = pc.IGNORE
    x, w = b.make(x, dtype), b.make(w, dtype)
    X, W = b.values(x), b.values(w)[~low]
    place = np.cumsum(~low) - 1                                              # of a class among those that take part
    loss, rows, lse, p, keep, n, L, X = pc.loss_exact(X, W, np.where(hide, pc.IGNORE, place[np.where(hide, 0, t)]))
    d = (D + 5) * E * (np.abs(X) @ np.abs(W).T).max(1)
    row_err = (2 * d + 8 * E * (np.abs(L).max(1) + np.log(V) + 1) + FN) * keep
    targets = b.ints(t, np.int64)
    got, got_rows, got_lse = b.ctx.cross_entropy(x, w, targets, rows=True)
    within(b.values(got_rows), rows, row_err, "row losses")
    within(b.values(got_lse), lse, row_err, "log sums")
    within(b.values(got), loss, row_err.sum() / n + E * abs(loss), "loss")
    got, dx, dw = b.ctx.cross_entropy_grad(x, w, targets)
    within(b.values(got), loss, row_err.sum() / n + E * abs(loss), "loss")
    q = np.abs(p) * U[dtype] + (1.0 / n) * (np.exp(L - lse[:, None]) * (row_err[:, None] * 2 + FN * (1 + np.abs(L - lse[:, None])))
                                            + LEAST[dtype] * (2.0 ** -15 if dtype == "f16" else 1.0)) * keep[:, None]
    DX, DW = p @ W, p.T @ X
    if dtype != "f16":
        within(b.values(dx), DX, U[dtype] * np.abs(DX) + (q + (V + 8) * E * np.abs(p)) @ np.abs(W) + LEAST[dtype], "dx")
    within(b.values(dw)[~low], DW, U[dtype] * np.abs(DW) + (q + (M + 8) * E * np.abs(p)).T @ np.abs(X) + LEAST[dtype], "dw")
    assert (b.values(dw)[low] == 0).all()


# (activation, rows, n_in, n_out, sizes of z, dy, w and x): gradients of binary16 whose dz leaves that type's range on either side,
# though its operands and results do not
RANGE = [("square", 20, 20, 20, 300.0, 200.0, 1e-3, 1e-4), ("square", 20, 20, 20, 1e-4, 1e-4, 1e4, 1e4), ("square", 65, 33, 270, 30.0, 1000.0, 1e-4, 1e-4),
         ("square", 700, 9, 5, 200.0, 3000.0, 1e-4, 1e-6), ("gelu", 37, 41, 19, 1.0, 1.5e4, 1e-2, 1e-3), ("silu", 37, 41, 19, 2.0, 1e-5, 1e4, 1e4),
         ("gelu", 130, 17, 50, 1.0, 1e-6, 1.5e4, 1e4), ("relu", 20, 30, 40, 1.0, 1.5e4, 1e-2, 1e-3)]


def check_range(b, name, M, K, N, z, dy, w, x, seed=0, rows=None, cols=None):
    """linear_grad in binary16.  dz may be held with a factor for each row (dx) or column (dw), whose largest number then has room for 2^-39 of itself:
    what the type's 11 bits and smallest step leave.  rows, cols: factors of z and dy."""
    rng = np.random.default_rng([seed, M, K, N, 6])

    def sized(m, n, size):
        return np.clip(normal(rng, m, n, std=size), -4 * size, 4 * size)

    r, c = np.ones(M) if rows is None else rows, np.ones(N) if cols is None else cols
    X, W = b.make(sized(M, K, x), "f16"), b.make(sized(N, K, w), "f16")
    Z, DY = b.make(sized(M, N, z) * r[:, None] * c, "f16"), b.make(sized(M, N, dy) * r[:, None] * c, "f16")
    dx, dw, db = b.ctx.linear_grad(DY, X, W, Z, activation=name, bias=True)
    X, W, Z, DY = b.values(X), b.values(W), b.values(Z), b.values(DY)
    assert all(np.isfinite(v).all() for v in (X, W, Z, DY))
    DZ = DY * pc.act(Z, name)[1]
    curve = np.abs(DY) * FN * 4 if name in ("gelu", "silu") else np.zeros_like(DY)
    u, least = U["f16"], LEAST["f16"]
    dDZ = (u + 4 * E) * np.abs(DZ) + curve
    ex = dDZ + 2.0 ** -39 * np.abs(DZ).max(1, keepdims=True)
    ew = dDZ + 2.0 ** -39 * np.abs(DZ).max(0, keepdims=True)
    DX, DW, DB = DZ @ W, DZ.T @ X, DZ.sum(0)
    assert max(np.abs(DX).max(), np.abs(DW).max()) < 60000
    within(b.values(dx), DX, u * np.abs(DX) + (ex + (N + 4) * E * np.abs(DZ)) @ np.abs(W) + least, "dx")
    within(b.values(dw), DW, u * np.abs(DW) + (ew + (M + 4) * E * np.abs(DZ)).T @ np.abs(X) + least, "dw")
    fits = np.abs(DB) < 60000
    within(b.values(db)[fits], DB[fits], (u * np.abs(DB) + ((M + 8) * E * np.abs(DZ) + curve).sum(0) + least)[fits], "db")


def check_range_of_each_row(b):
    """rows, and columns, whose dz lie 2^40 apart"""
    far = np.where(np.arange(23) % 3 == 0, 1e3, 1e-3)
    check_range(b, "square", 23, 31, 17, 1.0, 1.0, 1e-4, 1e-4, rows=far)
    check_range(b, "square", 23, 31, 17, 1.0, 1.0, 1e-4, 1e-4, cols=far[:17])
    check_range(b, "square", 300, 31, 290, 1.0, 1.0, 1e-4, 1e-4, rows=np.where(np.arange(300) % 7, 1e-2, 1e2), cols=np.where(np.arange(290) % 5, 1.0, 10.0))


def check_rows_that_are_not_finite(b, M=70, K=20, N=270):
    """an infinity or NaN among dy or z is its own row's affair in dx, and its own column's in dw and db"""
    rng = np.random.default_rng(11)
    x, w, z, dy = (normal(rng, *s) for s in ((M, K), (N, K), (M, N), (M, N)))
    clean = b.ctx.linear_grad(b.make(dy, "f16"), b.make(x, "f16"), b.make(w, "f16"), b.make(z, "f16"), activation="square", bias=True)
    dy[3, 5], dy[69, 200], z[40, 269] = np.inf, np.nan, -np.inf
    got = b.ctx.linear_grad(b.make(dy, "f16"), b.make(x, "f16"), b.make(w, "f16"), b.make(z, "f16"), activation="square", bias=True)
    rows, cols = np.ones(M, bool), np.ones(N, bool)
    rows[[3, 40, 69]] = cols[[5, 200, 269]] = False
    for g, c, fine in zip(got, clean, (rows, cols, cols)):
        g, c = b.values(g), b.values(c)
        assert np.isfinite(g[fine]).all() and not np.isfinite(g[~fine]).any()
        if fine is not rows:
            assert np.array_equal(g[fine], c[fine])


# (dtype, rows, n_in, n_out) for the device: products that take the largest tile in all three of a layer's products, every edge ragged
WIDE = [("bf16", 4091, 4088, 4072), ("f16", 4005, 4080, 4064)]
# ... and ones whose odd rows are worth copying
COPIED = [("bf16", 2501, 2503, 2507), ("f16", 2503, 2601, 2705)]
COPIED_LOSS = [("bf16", 2051, 1021, 7001), ("f16", 1021, 517, 30011)]


# (size of the numbers, largest norm): factors below the smallest normal 32-bit number
TINY = [(1e30, 1e-9), (2e30, 1e-12), (3e37, 1.0), (1e25, 1e-16)]


def check_tiny_factor(b, std, max_norm, where):
    """32-bit gradients so large, or a norm so small, that the factor has few bits left as a 32-bit number: the scaled numbers have theirs"""
    rng = np.random.default_rng(15)
    for sizes in ((50, 7), (40000, 3)):
        grads = [b.make(np.clip(normal(rng, n, std=std), -3e38, 3e38), "f32") for n in sizes]
        vals = [b.values(g) for g in grads]
        norm = float(np.sqrt(sum((v ** 2).sum() for v in vals)))
        factor = max_norm / (norm + 1e-6)
        assert factor < 2.0 ** -120
        out = None if where == "place" else [b.make(np.full(n, 7.0), "f32") for n in sizes]
        b.ctx.clip_grad_norm(grads, max_norm, out=out)
        for v, o in zip(vals, out or grads):
            within(b.values(o), v * factor, (U["f32"] + 4 * E) * np.abs(v) * factor + LEAST["f32"], "gradient")


def check_gelu_tail(b):
    """gelu's own digits, where its value is far below its argument: 1e-6 + 1e-7 z^2 of it, and a rounding of the product"""
    z = np.concatenate([-np.linspace(0.001, 12.8, 3001), np.linspace(0.001, 12.8, 501)])[:, None]
    x, one = b.make(z, "f32"), b.make(np.ones((1, 1)), "f32")
    Z = b.values(x)
    want = Z * ndtr(Z)
    within(b.values(b.ctx.linear(x, one, activation="gelu")), want, np.abs(want) * (1e-6 + 1e-7 * Z * Z + U["f32"]), "gelu")


def check_some_of_the_gradients(b, dtype, name):
    """any of dx, dw and db by itself is what it is among the others"""
    rng = np.random.default_rng(16)
    for M, K, N in ((70, 40, 33), (9, 300, 270)):
        x, w, dy, z = (b.make(normal(rng, *s), dtype) for s in ((M, K), (N, K), (M, N), (M, N)))
        z = None if name == "none" else z
        all_three = b.ctx.linear_grad(dy, x, w, z, activation=name, bias=True)
        for wanted in range(8):
            need = [bool(wanted >> i & 1) for i in range(3)]
            got = b.ctx.linear_grad(dy, x, w, z, activation=name, need_dx=need[0], need_dw=need[1], bias=need[2])
            for g, a, n in zip(got, all_three, need):
                assert (g is None) == (not n)
                if n:
                    assert np.array_equal(b.values(g), b.values(a)), (M, K, N, need)


def check_some_of_the_loss(b, dtype, M, D, V):
    """the loss' gradients by themselves, and the loss alone, are what they are together"""
    x, w, t = pc.loss_inputs(b, dtype, M, D, V, 0.3)
    targets = b.ints(t, np.int64)
    loss, dx, dw = (b.values(v) for v in b.ctx.cross_entropy_grad(x, w, targets, scale=3.0))
    for need_dx, need_dw in ((True, False), (False, True), (False, False)):
        got = b.ctx.cross_entropy_grad(x, w, targets, scale=3.0, need_dx=need_dx, need_dw=need_dw)
        assert np.array_equal(b.values(got[0]), loss)
        assert (got[1] is None) == (not need_dx) and (got[2] is None) == (not need_dw)
        assert not need_dx or np.array_equal(b.values(got[1]), dx)
        assert not need_dw or np.array_equal(b.values(got[2]), dw)
