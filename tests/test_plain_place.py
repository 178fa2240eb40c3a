"""The norm and its gradient in the memory of their inputs, on the CPU checker."""
import pytest

import plain_place_cases as place
from test_plain_rows import TYPES, b  # noqa: F401  (the fixture)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", place.SIZES, ids=str)
def test_norm(b, dtype, size):
    place.check_norm(b, dtype, *size)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", place.SIZES, ids=str)
def test_norm_grad(b, dtype, size):
    place.check_norm_grad(b, dtype, *size)
