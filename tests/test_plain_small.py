"""The norm into eight bits where its results lie below the normal 32-bit numbers, on the CPU checker."""
import pytest

import plain_small_cases as small
from test_plain_rows import b  # noqa: F401  (the fixture)


@pytest.mark.parametrize("power", small.POWERS)
@pytest.mark.parametrize("n", [2048, 17000])
def test_norm_mx(b, n, power):
    small.check_norm_mx(b, "f32", 100 if n < 16384 else 3, n, power)


def test_norm_mx_of_what_vanishes(b):
    """weights of 2^-149, the least 32-bit number: blocks that hold anything but zeros have the least scale"""
    small.check_norm_mx(b, "f32", 5, 200, -147)
