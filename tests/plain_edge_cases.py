"""Further cases of the training operators, shared by the CPU checker's tests and the device's (test helper, not collected).
Backends, bounds and definitions are plain_cases'."""
import numpy as np

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
