"""The operators between the plain network's layers on the device: the CPU checker's cases and larger ones against 64-bit definitions, streams and graphs, offsets
beyond 32 bits, the same bits on every call."""
import numpy as np
import pytest

import plain_cases as pc
import plain_rows_cases as rc
from test_gpu_plain_ops import _DT, Backend

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = ["f32", "f16", "bf16"]


class RowsBackend(Backend):
    cuts = True

    def type(self, dtype):
        return _DT[dtype]

    def raw(self, a):
        return a.cpu().numpy()

    def microscaled(self, codes, scales, columns, form, pitch=None):
        from paper_1811_00778_amd.binding import Microscaled
        rows = codes.shape[0]
        room = torch.full((scales.shape[0], pitch or -(-rows // 64) * 64), 255, dtype=torch.uint8, device="cuda")
        room[:, :rows] = torch.from_numpy(np.ascontiguousarray(scales)).cuda()
        return Microscaled(torch.from_numpy(np.ascontiguousarray(codes)).cuda(), room[:, :rows], columns, form)


@pytest.fixture(scope="module")
def b():
    return RowsBackend()


def say(*a):
    print("[rows]", *a, flush=True)


# ---------------------------------------------------------------- the checker's cases, and larger ones
LARGE = [(8192, 77), (700, 1031), (300, 4096), (33, 8200), (5, 16384), (3, 20001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES + LARGE, ids=str)
def test_dropout(b, dtype, size):
    say("dropout", dtype, size)
    rc.check_dropout(b, dtype, *size, 0.3, True)
    rc.check_dropout(b, dtype, *size, 0.9, False, seed=2 ** 64 - 1, stream=2 ** 32 - 1, strides=(5, 1), junk=True)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -33, 0.5, 1 - 2.0 ** -33, 1.0])
def test_dropout_at_the_ends(b, p):
    rc.check_dropout(b, "f32", 9, 30, p, True, junk=p > 0.4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES + LARGE, ids=str)
def test_norm(b, dtype, size):
    say("norm", dtype, size)
    rc.check_norm(b, dtype, *size, residual=True)
    rc.check_norm(b, dtype, *size, weight=False, strides=(3, 1))
    rc.check_norm_mx(b, dtype, *size)
    rc.check_norm_mx(b, dtype, *size, residual=True, weight=False, strides=(3, 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES + LARGE, ids=str)
def test_norm_grad(b, dtype, size):
    say("norm_grad", dtype, size)
    rc.check_norm_grad(b, dtype, *size, ds=True)
    rc.check_norm_grad(b, dtype, *size, weight=False, strides=(3, 1))


def test_norm_of_large_and_small_numbers(b):
    for std in (1e25, 1e37, 1e-30):
        rc.check_norm(b, "f32", 4, 300, std=std, eps=1e-30)
        rc.check_norm(b, "bf16", 4, 300, std=std, eps=1e-30)
    rc.check_norm_grad(b, "f32", 4, 300, std=1e25)


@pytest.mark.parametrize("form", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", rc.SIZES + LARGE, ids=str)
def test_quantize(b, dtype, form, size):
    say("quantize", dtype, form, size)
    rc.check_quantize(b, dtype, form, *size)
    rc.check_quantize(b, dtype, form, *size, strides=(3, 1))


@pytest.mark.parametrize("form", ["mx4", "mx8"])
def test_quantize_ties_and_ends(b, form):
    from test_plain_rows import edge_numbers
    rows = edge_numbers(form)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows * 2.0 ** -120)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows * 2.0 ** -140)
    rc.check_quantize(b, "f32", form, *rows.shape, x=rows * 2.0 ** (127 - rc.TOP[form]))
    rc.check_quantize(b, "bf16", form, *rows.shape, x=rows)
    rc.check_quantize(b, "f16", form, *rows.shape, x=rows * 2.0 ** -10)


def test_what_is_not_finite(b):
    x = pc.normal(np.random.default_rng(3), 4, 200)
    x[1, 7], x[2, 150] = np.inf, np.nan
    rc.check_quantize(b, "bf16", "mx4", 4, 200, x=x)
    rc.check_quantize(b, "f32", "mx8", 4, 200, x=x)
    a = b.make(x, "f32")
    y = b.values(b.ctx.rms_norm(a))
    assert np.isfinite(y[[0, 3]]).all() and np.isnan(y[1, 7]) and (np.delete(y[1], 7) == 0).all() and np.isnan(y[2]).all()
    s = b.raw(b.ctx.rms_norm(a, format="mx8").scales)
    assert (s[0, 1] == 255) and (s[1:, 1] == 127).all() and (s[:7, 2] == 255).all() and (s[:, [0, 3]] < 255).all()


# ---------------------------------------------------------------- the product
LINEAR_LARGE = [("bf16", "mx8", 1, 4096, 4096, "silu", True, True), ("f16", "mx4", 3, 1000, 16400, "none", True, False), ("f32", "mx8", 16, 2000, 300, "none", False, False),
                ("bf16", "mx4", 517, 1031, 777, "gelu", True, True), ("f16", "mx8", 300, 640, 520, "relu", True, True), ("f32", "mx4", 1000, 25, 5, "square", False, False),
                ("bf16", "mx8", 1100, 300, 1200, "silu", True, False), ("f16", "mx4", 2300, 640, 2180, "square", True, True), ("bf16", "mx8", 4100, 1300, 4360, "gelu", True, True),
                ("bf16", "mx4", 4100, 1300, 4360, "none", False, False), ("f32", "mx8", 4000, 140, 4100, "none", True, False), ("f16", "mx8", 4096, 100, 4096, "relu", False, False), ("f32", "mx8", 257, 1024, 258, "gelu", True, True), ("bf16", "mx4", 600, 4000, 40, "none", True, False)]


@pytest.mark.parametrize("case", rc.LINEAR + LINEAR_LARGE, ids=str)
def test_linear_mx(b, case):
    say("linear_mx", case)
    rc.check_linear(b, *case)


def test_linear_mx_wide_scales_and_nan(b):
    rng = np.random.default_rng(4)
    X = pc.normal(rng, 20, 300) * np.exp2(rng.integers(-20, 20, size=(20, 10)).repeat(30, 1))
    rc.check_linear(b, "f32", "mx8", 20, 300, 40, X=X)
    rc.check_linear(b, "bf16", "mx4", 20, 300, 40, X=X)
    rc.check_linear(b, "bf16", "mx8", 20, 300, 40, X=X)
    X[3, 77] = np.nan
    x, _ = rc.microscaled(b, X, "mx8")
    w, _ = rc.microscaled(b, pc.normal(rng, 40, 300), "mx4")
    y = b.values(b.ctx.linear_mx(x, w, dtype=torch.float32))
    assert np.isnan(y[3]).all() and np.isfinite(np.delete(y, 3, 0)).all()


def test_products_of_eight_bits_into_32_are_exact(b):
    """every code of both formats beside one another: sums of 128 products whose range is the formats' whole one, which 32 bits hold exactly where few terms are large"""
    rng = np.random.default_rng(5)
    code = rng.integers(0, 256, size=(40, 128)).astype(np.uint8)
    code[code % 128 == 127] = 0
    scales = np.full((4, 40), 127, np.uint8)
    x = b.microscaled(code, scales, 128, "mx8")
    wc = rng.integers(0, 256, size=(70, 64)).astype(np.uint8)
    w = b.microscaled(wc, np.full((4, 70), 127, np.uint8), 128, "mx4")
    X, W = rc.decode(code, scales, "mx8"), rc.decode(wc, np.full((4, 70), 127), "mx4")
    y = b.values(b.ctx.linear_mx(x, w, dtype=torch.float32))
    # products are multiples of 2^-10; both halves' 16 sums of eight, and those of the instruction, are rounded to 32 bits
    pc.within(y, X @ W.T, 40 * 2.0 ** -24 * (np.abs(X) @ np.abs(W).T), "y")
    half = b.values(b.ctx.linear_mx(x, w, dtype=torch.float16))
    pc.within(half, np.clip(X @ W.T, -65000, 65000), 2.0 ** -11 * np.abs(X @ W.T) + rc.cut_of(X, W) + 40 * 2.0 ** -24 * (np.abs(X) @ np.abs(W).T), "y")


def test_linear_mx_into_place(b):
    rng = np.random.default_rng(6)
    x, _ = rc.microscaled(b, pc.normal(rng, 130, 140), "mx8", pitch=192)
    w, _ = rc.microscaled(b, pc.normal(rng, 50, 140), "mx4")
    r = pc.normal(rng, 130, 50)
    want = b.ctx.linear_mx(x, w, residual=b.make(r, "bf16"), activation="relu")
    place = b.make(r, "bf16", (6, 1))
    assert b.ctx.linear_mx(x, w, residual=place, activation="relu", out=place) is place
    assert np.array_equal(b.values(place), b.values(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1100, 300, 1200), (4100, 300, 4160)], ids=str)
def test_tiles_into_place(b, dtype, size):
    """the residual's own memory as the output of tiles whose lanes exchange what they store; what lies between the rows stays"""
    say("place", dtype, size)
    rng = np.random.default_rng(8)
    M, K, N = size
    x, _ = rc.microscaled(b, pc.normal(rng, M, K), "mx8")
    w, _ = rc.microscaled(b, pc.normal(rng, N, K), "mx4")
    r = b.make(pc.normal(rng, M, N), dtype)
    want = b.ctx.linear_mx(x, w, residual=r, activation="silu")
    wide = torch.full((M, N + 13), 7.0, dtype=_DT[dtype], device="cuda")
    place = wide[:, 5:N + 5]
    place.copy_(r)
    b.ctx.linear_mx(x, w, residual=place, activation="silu", out=place)
    assert torch.equal(place, want)
    assert bool((wide[:, :5] == 7).all()) and bool((wide[:, N + 5:] == 7).all())
    assert torch.equal(b.ctx.linear_mx(x, w, residual=r[:1].expand(M, N), activation="none", dtype=_DT[dtype])[3], b.ctx.linear_mx(x, w, residual=r[:1].repeat(M, 1))[3])


# ---------------------------------------------------------------- runs of them
def chain(ctx, x, r, w, w4, bias):
    """A layer's way in training and back, and its answer from few bits"""
    h = ctx.dropout(x, 0.2, 11, 1, residual=r)
    y, s = ctx.rms_norm(h, w, x, keep=True)
    dx, dw = ctx.rms_norm_grad(y, s, w, h)
    d = ctx.dropout_grad(dx, 0.2, 11, 1)
    m = ctx.rms_norm(h, w, format="mx8")
    out = ctx.linear_mx(m, w4, bias, activation="gelu")
    q, values = ctx.quantize_mx(out, "mx4", values=True)
    return [h, y, s, dx, dw, d, m.codes, m.scales, out, q.codes, q.scales, values]


def chain_inputs(seed, rows=530, n=520, n_out=700):
    from paper_1811_00778_amd import binding
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, r, w = (torch.randn(s, generator=g, device="cuda").to(torch.bfloat16) for s in ((rows, n), (rows, n), (n,)))
    w4 = binding.PlainContext().quantize_mx(torch.randn((n_out, n), generator=g, device="cuda"), "mx4")
    return x, r, w, w4, torch.randn(n_out, generator=g, device="cuda")


def equal(a, c):
    return all(torch.equal(u, v) for u, v in zip(a, c))


def test_the_same_bits_on_every_call(b):
    ins = chain_inputs(1)
    first = [v.clone() for v in chain(b.ctx, *ins)]
    for _ in range(3):
        assert equal(first, chain(b.ctx, *ins))


def test_recorded_and_replayed(b):
    """a graph of the whole run, replayed between the program's own calls of other sizes; two graphs share the handle's work memory"""
    from paper_1811_00778_amd import binding
    ctx = binding.PlainContext()
    ins, other = chain_inputs(2), chain_inputs(3, rows=1200, n=1040, n_out=300)
    want, want_other = [v.clone() for v in chain(ctx, *ins)], [v.clone() for v in chain(ctx, *other)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(stream):
        ctx.use_stream()
        for i in (ins, other):
            chain(ctx, *i)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                outs.append(chain(ctx, *i))
            graphs.append(graph)
        big = chain_inputs(4, rows=3000, n=2000, n_out=100)
        for turn in range(3):
            for graph, out, expected in zip(graphs, outs, (want, want_other)):
                for v in out:
                    v.zero_()
                graph.replay()
                chain(ctx, *big)
                torch.cuda.synchronize()
                assert equal(expected, out), turn
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    del graphs, outs
    ctx.close()


def test_another_stream_is_refused(b):
    x = torch.ones((4, 8), device="cuda")
    with torch.cuda.stream(torch.cuda.Stream()):
        for call in (lambda: b.ctx.dropout(x, 0.5, 1), lambda: b.ctx.rms_norm(x), lambda: b.ctx.rms_norm_grad(x, x), lambda: b.ctx.quantize_mx(x)):
            with pytest.raises(RuntimeError):
                call()


def test_other_devices_and_types_are_refused(b):
    x = torch.ones((4, 8))
    for call in (lambda: b.ctx.dropout(x, 0.5, 1), lambda: b.ctx.rms_norm(x), lambda: b.ctx.quantize_mx(x), lambda: b.ctx.dropout(x.double().cuda(), 0.5, 1)):
        with pytest.raises(TypeError):
            call()
    m = b.ctx.quantize_mx(x.cuda())
    with pytest.raises(TypeError):
        b.ctx.linear_mx(m, m, dtype=torch.float64)


def test_offsets_beyond_32_bits(b):
    """rows that lie more than 2^32 bytes apart, and more than 2^31 numbers in one matrix"""
    rows, n = 3, 200
    gap = (1 << 31) + 64
    big = torch.empty(2 * gap + n, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((rows, n), (gap, 1))
    x.copy_(torch.randn((rows, n), device="cuda"))
    near = x.contiguous()
    assert torch.equal(b.ctx.dropout(x, 0.5, 1, residual=x), b.ctx.dropout(near, 0.5, 1, residual=near))
    assert torch.equal(b.ctx.rms_norm(x), b.ctx.rms_norm(near))
    assert torch.equal(b.ctx.rms_norm_grad(x, x)[0], b.ctx.rms_norm_grad(near, near)[0])
    assert torch.equal(b.ctx.quantize_mx(x).codes, b.ctx.quantize_mx(near).codes)
    del big, x
    rows, n = 600_000, 4096
    x = torch.ones((rows, n), dtype=torch.bfloat16, device="cuda")
    y = b.ctx.dropout(x, 0.5, 9)
    tail = torch.from_numpy(rc.kept(rows, 8, 0.5, 9, 0)[-5:]).cuda()
    assert torch.equal(y[-5:, :8] > 0, tail)
    m = b.ctx.quantize_mx(y, "mx4")
    assert torch.equal(m.codes[-1], b.ctx.quantize_mx(y[-1:], "mx4").codes[0])
    # one row in 64 of the result is compared: each is a sum of ones and twos
    w = b.ctx.quantize_mx(torch.ones((3, n), device="cuda"), "mx4")
    got = b.ctx.linear_mx(m, w, dtype=torch.float32)
    assert torch.equal(got[::64], y[::64].float().sum(1, keepdim=True).expand(-1, 3))
    torch.cuda.empty_cache()
