"""Operands of the microscaled product whose sums 32 bits hold whatever their order, shared by the CPU checker's tests and the device's (test helper, not collected).

Results are then those of the definition rounded once to their type, and are compared number by number: nothing may be cut on the way.
"""
import numpy as np

import plain_rows_cases as rc


# Sizes for every form of the product: (format, kernel, parts of k, (rows, n_in, n_out)).  Which form the library takes on 256 compute units is asserted by the checker's tests: a
# change of its rule that moves a size elsewhere fails there, and the device's tests go on reaching every form.
STRIP_16_16, STRIP_16_64, STRIP_64_16, STRIP_64_64, TILE_128, TILE_256 = range(6)
FORMS = [(form, kind, parts, size) for form in ("mx4", "mx8") for kind, parts, size in (
    (STRIP_16_16, 1, (1, 2000, 3000)), (STRIP_16_16, 1, (3, 2040, 2100)),
    (STRIP_16_64, 1, (1, 4096, 16384)), (STRIP_16_64, 1, (13, 1100, 8200)),
    (STRIP_64_16, 1, (32, 4096, 4096)), (STRIP_64_16, 1, (65, 257, 66)),
    (STRIP_64_64, 1, (64, 4096, 16384)), (STRIP_64_64, 1, (60, 1990, 16300)),
    (TILE_128, 1, (1100, 700, 1200)), (TILE_128, 1, (1100, 1300, 4090)), (TILE_128, 2, (8190, 8000, 250)),
    (TILE_256, 1, (4096, 700, 4096)), (TILE_256, 1, (4090, 1300, 4090)))]
FORMS += [("mx8", STRIP_64_64, 1, (1024, 1024, 1024)), ("mx8", TILE_128, 4, (3000, 2000, 100)), ("mx8", TILE_256, 3, (1500, 6000, 3000)), ("mx4", TILE_256, 3, (2060, 20000, 2060))]


def exact_codes(rng, M, K, N, form):
    """(x's codes, x's exponents, w's codes, w's exponents): numbers of the formats [rows][K up to whole 128] (0 behind K) and of the blocks [blocks][rows], 0 or 1.

    Four bits: any codes.  Products are multiples of 2^-2 up to 36, times scales up to 4: sums of K <= 29000 stay below 2^24 of those steps.
    Eight bits: numbers up to 7 2^-9, and in every group of eight neighbours a pair x, -x of any size whose two weights are equal.  A pair cancels: what is left of a group is
    below 8 * 6 * 7 * 2^-9 = 2^-0.6, in multiples of 2^-10, but a sum that drops what lies far below its largest product loses it.  Times scales up to 4, sums of
    K <= 2^13 with one pair open stay below 2^10 * 0.66 * 4 + 448 * 6 * 4 < 2^14."""
    assert K <= (29000 if form == "mx4" else 1 << 13)
    wide = -(-K // 128) * 128
    w = rng.integers(0, 16, size=(N, wide), dtype=np.uint8)
    if form == "mx4":
        x = rng.integers(0, 16, size=(M, wide), dtype=np.uint8)
    else:
        x = rng.integers(0, 8, size=(M, wide), dtype=np.uint8) + 128 * rng.integers(0, 2, size=(M, wide), dtype=np.uint8)
        at = np.arange(0, K - K % 8, 8) + 2 * rng.integers(0, 4, size=K // 8)          # the first of each group's pair
        big = rng.integers(0, 127, size=(M, len(at)), dtype=np.uint8)
        x[:, at], x[:, at + 1] = big, big + 128
        w[:, at + 1] = w[:, at]
    x[:, K:] = w[:, K:] = 0
    blocks = -(-K // 32)
    ex, ew = np.zeros((wide // 32, M), int), np.zeros((wide // 32, N), int)
    ex[:blocks], ew[:blocks] = rng.integers(0, 2, size=(blocks, M)), rng.integers(0, 2, size=(blocks, N))
    return x, ex, w, ew


def exact_operands(b, form, M, K, N, seed=0):
    """(x, w, x w^T in 64 bits)"""
    rng = np.random.default_rng([seed, M, K, N, 21])
    x, ex, w, ew = exact_codes(rng, M, K, N, form)
    X, W = (rc.decode(rc.packed(c, f), e + 127, f) for c, e, f in ((x, ex, form), (w, ew, "mx4")))
    down = 6 if form == "mx4" else 0                                 # (binary16's range)
    a, c = (b.microscaled(rc.packed(v, f), (e + 127).astype(np.uint8), K, f) for v, e, f in ((x, ex - down, form), (w, ew, "mx4")))
    want = X @ W.T * 2.0 ** -down
    assert np.abs(want).max(initial=0) < 65504
    return a, c, want


def check_exact(b, dtypes, form, M, K, N, seed=0):
    a, c, exact = exact_operands(b, form, M, K, N, seed)
    for dtype in dtypes:
        got, want = b.values(b.ctx.linear_mx(a, c, dtype=b.type(dtype))), b.values(b.make(exact, dtype))
        assert got.shape == (M, N)
        assert np.array_equal(got, want), (dtype, int((got != want).sum()), np.argwhere(got != want)[:5].tolist())
