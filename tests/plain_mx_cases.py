"""Operands of the microscaled product whose sums 32 bits hold whatever their order, shared by the CPU checker's tests and the device's (test helper, not collected).

Results are then those of the definition rounded once to their type, and are compared number by number: nothing may be cut on the way.
"""
import numpy as np

import plain_rows_cases as rc


def exact_codes(rng, M, K, N, form):
    """(x's codes, x's exponents, w's codes, w's exponents): numbers of the formats [rows][K up to whole 128] (0 behind K) and of the blocks [blocks][rows], 0 or 1.

    Four bits: any codes.  Products are multiples of 2^-2 up to 36, times scales up to 4: sums of K <= 2^13 stay below 2^24 of those steps.
    Eight bits: numbers up to 7 2^-9, and in every group of eight neighbours a pair x, -x of any size whose two weights are equal.  A pair cancels: what is left of a group is
    below 8 * 6 * 7 * 2^-9 = 2^-0.6, in multiples of 2^-10, but a sum that drops what lies far below its largest product loses it.  Times scales up to 4, sums of
    K <= 2^11 with one pair open stay below 2^8 * 0.66 * 4 + 448 * 6 * 4 < 2^14."""
    assert K <= (1 << 13 if form == "mx4" else 1 << 11)
    wide = -(-K // 128) * 128
    w = rng.integers(0, 16, size=(N, wide))
    if form == "mx4":
        x = rng.integers(0, 16, size=(M, wide))
    else:
        x = rng.integers(0, 8, size=(M, wide)) + 128 * rng.integers(0, 2, size=(M, wide))
        at = np.arange(0, K - K % 8, 8) + 2 * rng.integers(0, 4, size=K // 8)          # the first of each group's pair
        big = rng.integers(0, 127, size=(M, len(at)))
        x[:, at], x[:, at + 1] = big, big + 128
        w[:, at + 1] = w[:, at]
    x[:, K:] = w[:, K:] = 0
    blocks = -(-K // 32)
    ex, ew = np.zeros((wide // 32, M), int), np.zeros((wide // 32, N), int)
    ex[:blocks], ew[:blocks] = rng.integers(0, 2, size=(blocks, M)), rng.integers(0, 2, size=(blocks, N))
    return x, ex, w, ew


def check_exact(b, dtype, form, M, K, N, seed=0):
    rng = np.random.default_rng([seed, M, K, N, 21])
    x, ex, w, ew = exact_codes(rng, M, K, N, form)
    X, W = (rc.decode(rc.packed(c, f), e + 127, f) for c, e, f in ((x, ex, form), (w, ew, "mx4")))
    scale = 2.0 ** -6 if form == "mx4" else 1.0                      # (binary16's range)
    ex = ex + int(np.log2(scale))
    a, c = (b.microscaled(rc.packed(v, f), (e + 127).astype(np.uint8), K, f) for v, e, f in ((x, ex, form), (w, ew, "mx4")))
    want = X @ W.T * scale
    assert np.abs(want).max(initial=0) < 65504
    y = b.ctx.linear_mx(a, c, dtype=b.type(dtype))
    got, want = b.values(y), b.values(b.make(want, dtype))
    assert got.shape == (M, N)
    assert np.array_equal(got, want), (int((got != want).sum()), np.argwhere(got != want)[:5].tolist())
    return y
