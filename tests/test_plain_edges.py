"""The training operators on the CPU checker, at the edges of their numbers, memory and arguments."""
import pytest

import emu
import plain_edge_cases as pe
from test_plain_ops import Backend


@pytest.fixture(scope="module", params=[1, 256], ids=["one-unit", "256-units"])
def b(request):
    with emu.device(emu.lib(), units=request.param):
        yield Backend()


@pytest.mark.parametrize("case", pe.LOW, ids=str)
def test_classes_of_minus_infinity(b, case):
    pe.check_low_classes(b, *case)


@pytest.mark.parametrize("case", pe.RANGE, ids=str)
def test_range_of_binary16_gradients(b, case):
    pe.check_range(b, *case)


def test_range_of_each_row_and_column(b):
    pe.check_range_of_each_row(b)


def test_rows_that_are_not_finite(b):
    pe.check_rows_that_are_not_finite(b)
