"""The norm and its gradient in the memory of their inputs, on the device."""
import pytest

import plain_place_cases as place
from test_gpu_plain_rows import RowsBackend, TYPES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    return RowsBackend()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", place.SIZES + [(3000, 256), (700, 4096)], ids=str)
def test_norm(b, dtype, size):
    print("[place] norm", dtype, size, flush=True)
    place.check_norm(b, dtype, *size)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", place.SIZES + [(3000, 256), (700, 4096)], ids=str)
def test_norm_grad(b, dtype, size):
    print("[place] norm_grad", dtype, size, flush=True)
    place.check_norm_grad(b, dtype, *size)
