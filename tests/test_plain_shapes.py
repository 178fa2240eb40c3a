"""Every shape of the training operators' products on the CPU checker: tiles, parts of k, ways to LDS and copies of operands are forced, and
what was launched is looked at.  And what the device's larger cases take, by the rules."""
import ctypes

import numpy as np
import pytest

import emu
import plain_cases as pc
import plain_edge_cases as pe
from paper_1811_00778_amd import _capi
from test_plain_ops import Backend

T256, T128, T64, TALL, FLAT = range(5)
OUT, SUMS, STATS, DELTA = range(4)
TILES = [(t, tile) for t in ("f32", "f16", "bf16") for tile in (T256, T128, T64, TALL, FLAT) if t != "f32" or tile != T256]   # (the largest: 16 bits)


class forced:
    """Products in this tile and number of parts, copies of every unaligned operand, while the block runs."""

    def __init__(self, tile, parts=1, copies=False):
        self.lib, self.args = emu.lib(), (tile, parts, int(copies))
        self.lib.hcnn_emu_shape.argtypes, self.lib.hcnn_emu_shape.restype = [ctypes.c_int, ctypes.c_uint32, ctypes.c_int], None
        self.lib.hcnn_emu_taken.argtypes, self.lib.hcnn_emu_taken.restype = [ctypes.POINTER(ctypes.c_uint64)] * 2, None

    def __enter__(self):
        self.lib.hcnn_emu_shape(*self.args)
        return self

    def taken(self):
        """({(ending, tile, past the registers)}, copies launched)"""
        bits, copied = ctypes.c_uint64(), ctypes.c_uint64()
        self.lib.hcnn_emu_taken(ctypes.byref(bits), ctypes.byref(copied))
        return {(i // 16, i % 16 // 2, i % 2 == 1) for i in range(64) if bits.value >> i & 1}, copied.value

    def __exit__(self, *_):
        self.lib.hcnn_emu_shape(-1, 1, 0)


@pytest.fixture(scope="module")
def b():
    return Backend()


# (rows, n_in, n_out): more than a tile in every direction, ragged; the last stage of k is not whole; rows that start on 16 bytes, and ones that do not
ALIGNED, ODD = (280, 200, 264), (277, 197, 261)


@pytest.mark.parametrize("dtype,tile", TILES)
def test_whole_stages_past_the_registers(b, dtype, tile):
    with forced(tile) as f:
        pc.check_linear(b, dtype, *ALIGNED, "gelu", bias=True, residual=True, keep=True)
        pc.check_grad(b, dtype, *ALIGNED, "square", bias=True)
        pc.check_loss(b, dtype, *ALIGNED, 0.3, scale=64.0)
        pc.check_loss(b, dtype, *ALIGNED, 0.0)
        taken, copied = f.taken()
    assert {(e, tile, True) for e in (OUT, STATS, DELTA)} <= taken and not copied


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tile", [T128, T64, TALL, FLAT])
def test_through_the_registers(b, dtype, tile):
    with forced(tile) as f:
        pc.check_linear(b, dtype, *ODD, "silu", bias=True, residual=True, keep=True, strides=(3, 1))
        pc.check_grad(b, dtype, *ODD, "none", bias=True, strides=(3, 1))
        pc.check_loss(b, dtype, *ODD, 0.3, scale=64.0, strides=(3, 1))
        taken, _ = f.taken()
    assert {(e, tile, False) for e in (OUT, STATS, DELTA)} <= taken


@pytest.mark.parametrize("dtype,tile", TILES)
def test_parts_of_k(b, dtype, tile):
    for parts in (2, 9):
        with forced(tile, parts) as f:
            pc.check_linear(b, dtype, 40, 2000, 72, "square", bias=True, residual=True, keep=True)
            pc.check_grad(b, dtype, 1400, 72, 40, "square", bias=True)
            pc.check_loss(b, dtype, 1200, 72, 40, 0.5)
            taken, _ = f.taken()
        assert (SUMS, tile, True) in taken


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tile", [T256, T128, T64])
@pytest.mark.parametrize("strides", [None, (3, 1)])
def test_copied_operands(b, dtype, tile, strides):
    """operands of odd rows are copied to rows that end in zeros: NaN between the rows must not come along, masked rows neither"""
    with forced(tile, copies=True) as f:
        pc.check_linear(b, dtype, *ODD, "gelu", bias=True, residual=True, keep=True, strides=strides)
        taken, copied = f.taken()
        assert (OUT, tile, True) in taken and copied == 2                   # x and w
    with forced(tile, copies=True) as f:
        pc.check_grad(b, dtype, *ODD, "none", bias=True, strides=strides)
        taken, copied = f.taken()
        assert (OUT, tile, True) in taken and copied == 3                   # dy, x and w
    with forced(tile, copies=True) as f:
        pc.check_grad(b, dtype, *ODD, "square", bias=True, strides=strides)
        assert f.taken()[1] == 2
    with forced(tile, copies=True) as f:
        pc.check_loss(b, dtype, *ODD, 0.3, strides=strides, junk=True)
        taken, copied = f.taken()
        assert {(e, tile, True) for e in (OUT, STATS, DELTA)} <= taken and copied == 3      # w in each of three calls; x by the rows that take part
    with forced(tile, copies=True):
        pc.check_loss(b, dtype, *ODD, 0.0, strides=strides)


def test_the_largest_tiles_narrow_operand():
    """one operand copied, the other in place: the sum then ends at its last number, not at the copy's"""
    b = Backend()
    with forced(T256, copies=True) as f:
        rng = np.random.default_rng(3)
        M, K, N = ODD
        x = b.make(pc.normal(rng, M, K), "bf16", (3, 0))                     # rows of 200 numbers: aligned, NaN behind each
        w = b.make(pc.normal(rng, N, K), "bf16")
        want = b.values(x) @ b.values(w).T
        got = b.values(b.ctx.linear(x, w))
        taken, copied = f.taken()
        assert (OUT, T256, True) in taken and copied == 1
    pc.within(got, want, pc.U["bf16"] * np.abs(want) + (K + 4) * pc.E * (np.abs(b.values(x)) @ np.abs(b.values(w)).T), "y")


def _choice(h, dtype, M, N, K, split, direct):
    f = emu.lib().hcnn_emu_choice
    f.argtypes, f.restype = [ctypes.c_void_p, ctypes.c_int] + [ctypes.c_size_t] * 3 + [ctypes.c_int] * 2, ctypes.c_uint32
    v = f(h, {"f32": _capi.F32, "f16": _capi.F16, "bf16": _capi.BF16}[dtype], M, N, K, split, direct)
    return v & 255, v >> 8


def _copies(rows, cols, work):
    f = emu.lib().hcnn_emu_copies
    f.argtypes, f.restype = [ctypes.c_size_t, ctypes.c_size_t, ctypes.c_double], ctypes.c_int
    return bool(f(rows, cols, work))


def test_what_the_devices_cases_take():
    """the device's cases of plain_edge_cases reach what they are there for, on 256 compute units"""
    with emu.device(emu.lib(), units=256):
        held = Backend()                                         # (owns the handle)
        h = held.ctx.raw.handle
        for dtype, M, K, N in pe.WIDE:
            assert _choice(h, dtype, M, N, K, True, True)[0] == T256, (dtype, M, K, N)
            assert _choice(h, dtype, M, K, N, True, True)[0] == T256 and _choice(h, dtype, N, K, M, True, True)[0] == T256
        for dtype, M, K, N in pe.COPIED:
            work = float(M) * K * N
            assert all(n % 8 for n in (K, N)) and all(_copies(r, c, work) for r, c in ((M, K), (N, K), (M, N)))
        for dtype, M, K, V in pe.COPIED_LOSS:
            assert K % 8 and _copies(M, K, 3.0 * M * K * V) and _copies(V, K, 3.0 * M * K * V)


class thread_limit:
    """The most threads of one launch, while the block runs."""

    def __init__(self, most):
        self.set, self.most = emu.lib().hcnn_emu_threads, most
        self.set.argtypes, self.set.restype = [ctypes.c_uint64], None

    def __enter__(self):
        self.set(self.most)

    def __exit__(self, *_):
        self.set(2 ** 32 - 1)


def test_rows_and_copies_beyond_one_threads_each(b):
    """a launch has fewer than 2^32 threads: the kernels whose threads follow rows (64 each) and copied bytes go round instead"""
    with thread_limit(2 ** 14):
        pc.check_loss(b, "f32", 700, 3, 5, 0.3, junk=True)
        pc.check_loss(b, "bf16", 600, 7, 20, 0.9)
        with forced(T128, copies=True) as f:
            pc.check_linear(b, "bf16", 600, 197, 40, strides=(3, 1))
            pc.check_loss(b, "f16", 600, 197, 40, 0.3, junk=True)
            assert f.taken()[1] == 5


def test_offsets_of_rows_that_take_part_stay_in_32_bits(b):
    """x and w of broadcast rows have a stride of 0, the copy of the rows that take part has their length: at 4.2 million numbers a row, a tile's rows are
    more than 2^32 bytes apart there, and its loads past the registers would reach other ones"""
    x, w = (np.broadcast_to(b.make(np.ones((1, 4200000)), "f32"), (n, 4200000)) for n in (2, 1000))
    with forced(FLAT) as f, thread_limit(1024):               # (the products' launches are refused: only their shape is looked at)
        with pytest.raises(_capi.HcnnError):
            b.ctx.cross_entropy(x, w, b.ints([3, pc.IGNORE], np.int64))
        taken, _ = f.taken()
    assert taken == {(STATS, FLAT, False)}
