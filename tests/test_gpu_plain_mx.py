"""The product of microscaled matrices on the device, number by number: operands whose sums 32 bits hold in any order."""
import numpy as np
import pytest

import plain_mx_cases as mx
import plain_rows_cases as rc
from test_gpu_plain_rows import RowsBackend, TYPES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    return RowsBackend()


def say(*a):
    print("[mx]", *a, flush=True)


# rows, n_in, n_out: one row, few rows or columns, and tiles, of whole and odd sizes
EXACT = [(1, 300, 70), (3, 2040, 2100), (40, 130, 700), (257, 1024, 258), (1100, 300, 1200), (4090, 700, 4100)]


@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", EXACT, ids=str)
def test_nothing_is_cut(b, dtype, form, size):
    """small products beside large ones that cancel, in every type of result"""
    say("exact", dtype, form, size)
    mx.check_exact(b, [dtype], form, *size)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_ends_of_the_eight_bits(b, dtype):
    """448 and 3.75 beside the smallest number, cancelled and not: each number of x with its opposite, the smallest one, and weights of 6 and 0.5"""
    codes = [c for c in range(2, 127)]
    x = np.zeros((len(codes), 128), np.uint8)
    w = np.zeros((2, 128), int)
    for i, c in enumerate(codes):
        x[i, :3] = c, c + 128, 1
    w[0, :3] = 7, 7, 1                                               # 6 a - 6 a + 0.5 * 2^-9
    w[1, :3] = 1, 1, 7
    a = b.microscaled(x, np.full((4, len(codes)), 127, np.uint8), 128, "mx8")
    c = b.microscaled(rc.packed(w, "mx4"), np.full((4, 2), 127, np.uint8), 128, "mx4")
    y = b.values(b.ctx.linear_mx(a, c, dtype=b.type(dtype)))
    assert np.array_equal(y, np.tile([2.0 ** -10, 6 * 2.0 ** -9], (len(codes), 1)))
    # not cancelled, 22.5 + 2^-10 and the largest: 32 bits hold them
    if dtype == "f32":
        x[:, 1] = 0
        a = b.microscaled(x, np.full((4, len(codes)), 127, np.uint8), 128, "mx8")
        y = b.values(b.ctx.linear_mx(a, c, dtype=b.type(dtype)))
        v = rc.GRID["mx8"][codes]
        assert np.array_equal(y[:, 0], 6 * v + 2.0 ** -10) and y[codes.index(0x47), 0] == 22.5 + 2.0 ** -10


# ---------------------------------------------------------------- every form of the product
def test_the_device_is_the_one_that_the_forms_are_named_for(b):
    assert torch.cuda.get_device_properties(0).multi_processor_count == 256


@pytest.mark.parametrize("form,kind,parts,size", mx.FORMS, ids=str)
def test_forms(b, form, kind, parts, size):
    """each strip and tile, one slot and many, an odd number of steps, parts of k, edges that are not whole: number by number in every type of result"""
    say("form", kind, parts, form, size)
    mx.check_exact(b, TYPES, form, *size)


@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype,size", [("bf16", (4090, 700, 4090)), ("f32", (4090, 400, 4090)), ("f16", (8190, 2000, 250))], ids=str)
def test_endings_of_the_tiles(b, dtype, form, size):
    """activation, bias and residual behind sums of several slots, and behind joined parts"""
    say("ending", dtype, form, size)
    rc.check_linear(b, dtype, form, *size, "gelu", True, True)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_tiles_into_place(b, dtype):
    """the residual's memory as the output of the 256 x 256 tiles; what lies between the rows stays"""
    M, K, N = 4090, 700, 4090
    say("place", dtype)
    for form in ("mx4", "mx8"):
        x, w, exact = mx.exact_operands(b, form, M, K, N)
        exact = torch.from_numpy(exact).cuda()
        wide = torch.full((M, N + 13), 7.0, dtype=b.type(dtype), device="cuda")
        place = wide[:, 5:N + 5]
        place.zero_()
        b.ctx.linear_mx(x, w, residual=place, out=place)
        # (a double rounded to 32 bits, which hold it, and then to the type)
        assert torch.equal(place, exact.float().to(b.type(dtype)))
        assert bool((wide[:, :5] == 7).all()) and bool((wide[:, N + 5:] == 7).all())


def test_parts_recorded_and_replayed(b):
    """parts of k share the handle's work memory with larger ones that run between the replays"""
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    (x, w, exact), (big_x, big_w, big) = mx.exact_operands(b, "mx8", 3000, 2000, 100), mx.exact_operands(b, "mx8", 8190, 8000, 250)
    exact, big = (torch.from_numpy(v).cuda().float() for v in (exact, big))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ctx.use_stream()
        ctx.linear_mx(x, w, dtype=torch.float32)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = ctx.linear_mx(x, w, dtype=torch.float32)
        for turn in range(3):
            y.zero_()
            graph.replay()
            assert torch.equal(ctx.linear_mx(big_x, big_w, dtype=torch.float32), big), turn
            torch.cuda.synchronize()
            assert torch.equal(y, exact), turn
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    del graph, y
    ctx.close()
