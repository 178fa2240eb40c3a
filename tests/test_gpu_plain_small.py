"""The norm into eight bits where its results lie below the normal 32-bit numbers, on the device."""
import pytest

import plain_small_cases as small
from test_gpu_plain_rows import RowsBackend

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    return RowsBackend()


@pytest.mark.parametrize("power", small.POWERS + [-147])
@pytest.mark.parametrize("size", [(5, 200), (100, 2048), (3, 17000)], ids=str)
def test_norm_mx(b, size, power):
    print("[small]", size, power, flush=True)
    small.check_norm_mx(b, "f32", *size, power)
