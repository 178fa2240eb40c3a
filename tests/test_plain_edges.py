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
