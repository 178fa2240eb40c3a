"""The product of microscaled matrices on the CPU checker, number by number: operands whose sums 32 bits hold in any order."""
import ctypes

import pytest

import emu
import plain_mx_cases as mx
from test_plain_rows import EmuRows, TYPES, b  # noqa: F401  (the fixture)


@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 300, 70), (3, 300, 260), (40, 130, 100), (130, 384, 129)], ids=str)
def test_nothing_is_cut(b, dtype, form, size):
    mx.check_exact(b, [dtype], form, *size)


def test_the_forms_of_the_device_s_tests():
    """the form that each of those sizes takes on 256 compute units"""
    lib = emu.lib()
    lib.hcnn_emu_mx_choice.argtypes, lib.hcnn_emu_mx_choice.restype = [ctypes.c_void_p, ctypes.c_int] + [ctypes.c_size_t] * 3, ctypes.c_uint32
    with emu.device(lib, units=256):
        ctx = EmuRows()
        for form, kind, parts, size in mx.FORMS:
            choice = lib.hcnn_emu_mx_choice(ctx.raw.handle, {"mx4": 4, "mx8": 8}[form], *size)
            assert (choice & 255, choice >> 8) == (kind, parts), (form, size)
    assert {(form, kind, parts > 1) for form, kind, parts, _ in mx.FORMS} == {(form, kind, many) for form in ("mx4", "mx8") for kind in range(6) for many in ((False, True) if kind >= mx.TILE_128 else (False,))}
