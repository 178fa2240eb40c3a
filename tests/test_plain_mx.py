"""The product of microscaled matrices on the CPU checker, number by number: operands whose sums 32 bits hold in any order."""
import pytest

import plain_mx_cases as mx
from test_plain_rows import TYPES, b  # noqa: F401  (the fixture)


@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 300, 70), (3, 300, 260), (40, 130, 100), (130, 384, 129)], ids=str)
def test_nothing_is_cut(b, dtype, form, size):
    mx.check_exact(b, dtype, form, *size)
