"""The training operators on the CPU checker, at the edges of their numbers, memory and arguments."""
import ctypes
import glob
import os
import re

import numpy as np
import pytest
from scipy.special import erfcx

import emu
import plain_cases as pc
import plain_edge_cases as pe
from paper_1811_00778_amd import _capi
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


def _recording(on):
    """Whether streams count as being recorded from now on; the frees of the checker's device memory so far."""
    f = emu.lib().hcnn_emu_record
    f.argtypes, f.restype = [ctypes.c_int], ctypes.c_size_t
    return f(int(on))


def test_work_memory_that_a_recording_has_seen_stays():
    """a recorded graph reads the work memory of its calls: a later call that needs more must not free it before the handle goes"""
    b = Backend()

    def loss(rows):
        x, w, t = pc.loss_inputs(b, "f32", rows, 20, 40)
        return [v.copy() for v in b.ctx.cross_entropy_grad(x, w, b.ints(t, np.int64))]

    small = loss(30)
    _recording(True)
    for u, v in zip(small, loss(30)):
        assert np.array_equal(u, v)
    frees, held = _recording(False), b.ctx.scratch_bytes()
    loss(300)
    assert b.ctx.scratch_bytes() > held
    assert _recording(False) == frees                    # the recorded block is still there
    loss(900)
    assert _recording(False) == frees + 1                # the one between, which no recording has seen, is not
    _recording(True)
    loss(1500)                                           # grows while it is recorded: its old block may be in use
    assert _recording(False) == frees + 1
    b.ctx.close()
    assert _recording(False) == frees + 5                # three blocks, the one in use, the counter


def test_clipping_refuses_numbers_named_twice(b):
    """a number in two tensors of the list would be scaled by two workgroups, once or twice"""
    g = b.make(np.linspace(-3, 3, 200), "f32")
    before = g.copy()
    for grads, out in (([g, g], None), ([g, g[:-1]], None), ([g[:100], g[99:]], None), ([g, g], [g, g]), ([g[:100], g[50:150]], [g[:100], g[50:150]]),
                       ([g[10:20], g], [g[10:20], g])):
        with pytest.raises(ValueError):
            b.ctx.clip_grad_norm(grads, 1.0, out=out)
        assert np.array_equal(g, before)
    norm = b.ctx.clip_grad_norm([g[:100], g[100:], g[:0]], 1.0)          # side by side: no overlap
    pc.within(b.values(norm), np.linalg.norm(b.values(before)), 1e-6 * np.linalg.norm(b.values(before)), "norm")
    pc.within(b.values(b.ctx.clip_grad_norm([g, g], 1.0, out=[b.make(np.zeros(200), "f32") for _ in range(2)])), 2 ** 0.5, 1e-5, "norm of a tensor read twice")


def test_output_in_other_columns_of_the_inputs_array(b):
    """columns of one array: what a layer writes beside what it reads is no overlap, what reaches into it is"""
    rng = np.random.default_rng(12)
    w = b.make(pc.normal(rng, 5, 6), "f32")
    big = b.make(pc.normal(rng, 11, 24), "f32")
    x = big[:, 4:10]
    want = b.ctx.linear(x.copy(), w)
    for at in (10, 19):
        b.ctx.linear(x, w, out=big[:, at:at + 5])
        assert np.array_equal(big[:, at:at + 5], want)
    kept = big.copy()
    for at in (0, 5, 9):
        with pytest.raises(ValueError):
            b.ctx.linear(x, w, out=big[:, at:at + 5])
    with pytest.raises(ValueError):                             # rows of another pitch
        b.ctx.linear(x, w, out=np.lib.stride_tricks.as_strided(big[:, 10:], (11, 5), (23 * 4, 4)))
    assert np.array_equal(big, kept)
    # the residual's array, in other columns too
    r = big[:, 10:15]
    want = b.ctx.linear(x.copy(), w, residual=r.copy())
    b.ctx.linear(x, w, residual=r, out=big[:, 15:20])
    assert np.array_equal(big[:, 15:20], want)


def test_output_of_one_row_with_any_stride(b):
    """a single row has no next one: its stride says nothing"""
    rng = np.random.default_rng(13)
    x, w, r = (b.make(pc.normal(rng, *s), "f32") for s in ((1, 9), (6, 9), (1, 6)))
    want = b.ctx.linear(x, w, residual=r)
    for stride in (0, 4, 5 * 4, 400):
        out = np.lib.stride_tricks.as_strided(b.make(np.zeros(6), "f32"), (1, 6), (stride, 4))
        assert b.ctx.linear(x, w, residual=r, out=out) is out and np.array_equal(out, want)
    place = np.lib.stride_tricks.as_strided(r, (1, 6), (4, 4))           # the residual's own memory
    b.ctx.linear(x, w, residual=r, out=place)
    assert np.array_equal(r, want)


def test_assembly_names_the_registers_it_writes():
    """every asm statement of the kernels that sets m0 or vcc names it as clobbered"""
    found = 0
    for path in glob.glob(os.path.join(os.path.dirname(_capi.__file__), "csrc", "*")):
        with open(path) as f:
            for statement in re.findall(r"\basm\b[^;]*;", f.read()):
                for register in ("m0", "vcc"):
                    if re.search(r"\b[sv]_\w+ (?:%\d, )?" + register + r"\b", statement):
                        found += 1
                        assert '"%s"' % register in statement, (os.path.basename(path), statement)
    assert found >= 3


@pytest.mark.parametrize("where", ["new", "place"])
@pytest.mark.parametrize("case", pe.TINY, ids=str)
def test_factors_below_the_normal_numbers(b, case, where):
    pe.check_tiny_factor(b, *case, where)


def test_tail_of_gelu(b):
    pe.check_gelu_tail(b)


def test_polynomial_of_the_normal_distribution():
    """the coefficients themselves, in 64 bits: 1.5e-7 of the tail"""
    with open(os.path.join(os.path.dirname(_capi.__file__), "csrc", "plain_kernels.h")) as f:
        body = f.read().split("HCNN_HD float normal_cdf")[1].split("*bell = e")[0]
    c = float(re.search(r"1\.0f \+ ([\d.]+)f \* fabsf", body).group(1))
    q = [float(re.search(r"float q = (-?[\d.]+)f", body).group(1))] + [float(v.replace(" ", "")) for v in re.findall(r"q = q \* t ([+-] [\d.]+)f", body)]
    assert len(q) == 8
    a = np.linspace(0, 14, 20001)
    t, p = 1 / (1 + c * a), 0.0
    for v in q:
        p = p * t + v
    assert np.abs(p * t / (erfcx(a / np.sqrt(2)) / 2) - 1).max() < 1.5e-7


@pytest.mark.parametrize("name", ["none", "square", "relu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_some_of_the_gradients(b, dtype, name):
    pe.check_some_of_the_gradients(b, dtype, name)


@pytest.mark.parametrize("shape", [(50, 20, 9), (70, 33, 300), (3, 0, 20), (1, 40, 1000)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_some_of_the_loss(b, dtype, shape):
    pe.check_some_of_the_loss(b, dtype, *shape)


@pytest.mark.parametrize("V", [9, 300])
def test_outputs_of_the_losses_entry_points(b, V):
    """each of the optional outputs by itself, as C calls them"""
    x, w, t = pc.loss_inputs(b, "f32", 70, 33, V, 0.3)
    loss, rows, lse = b.ctx.cross_entropy(x, w, b.ints(t, np.int64), rows=True)
    dx, dw = b.ctx.cross_entropy_grad(x, w, b.ints(t, np.int64))[1:]
    given = (_capi.F32, 70, 33, V, x.ctypes.data, 33, w.ctypes.data, 33, t.ctypes.data, 8, pc.IGNORE)
    for wanted in range(8):
        out = [np.full_like(v, np.nan) for v in (rows, lse, loss)]
        b.ctx.raw.call("hcnn_cross_entropy", *given, *[o.ctypes.data if wanted >> i & 1 else None for i, o in enumerate(out)])
        for i, (o, v) in enumerate(zip(out, (rows, lse, loss))):
            assert np.array_equal(o, v) if wanted >> i & 1 else np.isnan(o).all()
    for wanted in range(16):
        out = [np.full_like(v, np.nan) for v in (rows, loss, dx, dw)]
        p = [o.ctypes.data if wanted >> i & 1 else None for i, o in enumerate(out)]
        b.ctx.raw.call("hcnn_cross_entropy_grad", *given, 1.0, p[0], p[1], p[2], 33, p[3], 33)
        for i, (o, v) in enumerate(zip(out, (rows, loss, dx, dw))):
            assert np.array_equal(o, v) if wanted >> i & 1 else np.isnan(o).all()
