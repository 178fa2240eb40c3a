"""The product of microscaled matrices on the device, number by number: operands whose sums 32 bits hold in any order."""
import numpy as np
import pytest

import plain_mx_cases as mx
import plain_rows_cases as rc
from test_gpu_plain_rows import RowsBackend, TYPES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    return RowsBackend()


def say(*a):
    print("[mx]", *a, flush=True)


# rows, n_in, n_out: one row, few rows or columns, and tiles, of whole and odd sizes
EXACT = [(1, 300, 70), (3, 2040, 2100), (40, 130, 700), (257, 1024, 258), (1100, 300, 1200), (4090, 700, 4100)]


@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", EXACT, ids=str)
def test_nothing_is_cut(b, dtype, form, size):
    """small products beside large ones that cancel, in every type of result"""
    say("exact", dtype, form, size)
    mx.check_exact(b, [dtype], form, *size)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_ends_of_the_eight_bits(b, dtype):
    """448 and 3.75 beside the smallest number, cancelled and not: each number of x with its opposite, the smallest one, and weights of 6 and 0.5"""
    codes = [c for c in range(2, 127)]
    x = np.zeros((len(codes), 128), np.uint8)
    w = np.zeros((2, 128), int)
    for i, c in enumerate(codes):
        x[i, :3] = c, c + 128, 1
    w[0, :3] = 7, 7, 1                                               # 6 a - 6 a + 0.5 * 2^-9
    w[1, :3] = 1, 1, 7
    a = b.microscaled(x, np.full((4, len(codes)), 127, np.uint8), 128, "mx8")
    c = b.microscaled(rc.packed(w, "mx4"), np.full((4, 2), 127, np.uint8), 128, "mx4")
    y = b.values(b.ctx.linear_mx(a, c, dtype=b.type(dtype)))
    assert np.array_equal(y, np.tile([2.0 ** -10, 6 * 2.0 ** -9], (len(codes), 1)))
    # not cancelled, 22.5 + 2^-10 and the largest: 32 bits hold them
    if dtype == "f32":
        x[:, 1] = 0
        a = b.microscaled(x, np.full((4, len(codes)), 127, np.uint8), 128, "mx8")
        y = b.values(b.ctx.linear_mx(a, c, dtype=b.type(dtype)))
        v = rc.GRID["mx8"][codes]
        assert np.array_equal(y[:, 0], 6 * v + 2.0 ** -10) and y[codes.index(0x47), 0] == 22.5 + 2.0 ** -10
