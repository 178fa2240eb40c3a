"""The training operators on the device, at the edges of their numbers, memory and arguments."""
import pytest

import plain_edge_cases as pe
from test_gpu_plain_ops import Backend, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    return Backend()


@pytest.mark.parametrize("case", pe.LOW, ids=str)
def test_classes_of_minus_infinity(b, case):
    say("minus infinity", case)
    pe.check_low_classes(b, *case)
